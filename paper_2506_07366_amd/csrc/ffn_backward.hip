// Gradient of the grouped expert FFN (grouped_ffn.hip).  For the rows of an expert, with their inputs x (one row per token,
// in the layer's type or as an 8-bit checkpoint) and the gradient dy of their results:
//     a = x W1, b = x W3, s = 1 / (1 + exp(-a)), h = a s b        worked out again, nothing of it was kept
//     dh = dy W2^T,  db = dh a s,  da = dh b s (1 + a (1 - s))
//     dx = da W1^T + db W3^T,  dW1 = x^T da,  dW3 = x^T db,  dW2 = h^T dy
// and in the ReLU form h = max(a, 0), da = dh where a > 0, dx = da W1^T, dW1 = x^T da, dW2 = h^T dy.
//
// bf16: sums in fp32.  Rounded to bf16 on the way are h, da and db, which are operands of further matrix products
// (as h is in the forward pass): a half step of 2^-8 each, on the terms of a long sum.  dh is not (with it rounded too, the
// gradients' error grows by a fifth, and the bytes that halving it saves are 1 to 2 % of a call).  Rows are worked on in the order of the
// forward pass's row list (by expert, replicas together):
//   1. dh = dy W2^T             tiles of ffn_tiles.h, weights packed for it (moe_pack_weights_backward)
//   2. a, b and from them and dh: h, and da and db side by side in the packed order of the columns of a and b
//                               tiles of ffn_tiles.h, the forward pass's packed weights
//   3. dW1, dW3 and dW2         ffn_weight_grad.h
//   4. dx                       tiles of ffn_tiles.h, one sum over da's and db's columns
// fp32: three launches of plain LDS tiles (below), from the forward pass's packed weights alone.
#include "ffn_device.h"
#include "checkpoint.h"
#include "../../include/moegps_train.h"

namespace moegps {

#include "ffn_tiles.h"
#include "ffn_weight_grad.h"

// The first product again, and what follows from it and dh.
template <int EPI>
__global__ __launch_bounds__(512, 2) void hidden_grad_kernel(
    const bf16_t* __restrict__ X, int d, const bf16_t* __restrict__ P13, size_t b_stride, bf16_t* __restrict__ dab,
    const MTile* __restrict__ mtiles, const int32_t* __restrict__ counts, int32_t* __restrict__ queues, int N,
    bool past_caches, RowMap rm, const float* __restrict__ dhidden, bf16_t* __restrict__ hidden) {
    tile_product<EPI, kAlone>(X, d, P13, b_stride, dab, N, mtiles, counts, queues, N, d, kTileGroup, past_caches, rm, nullptr,
                              RowCopy{}, nullptr, dhidden, hidden);
}

// dh = dy W2^T, in fp32.
__global__ __launch_bounds__(512, 2) void dhidden_kernel(
    const bf16_t* __restrict__ dy, int d, const bf16_t* __restrict__ P2, size_t b_stride, float* __restrict__ dhidden,
    const MTile* __restrict__ mtiles, const int32_t* __restrict__ counts, int32_t* __restrict__ queues, int N,
    bool past_caches, RowMap rm) {
    tile_product<kEpiFloat, kAlone>(dy, d, P2, b_stride, nullptr, N, mtiles, counts, queues, N, d, kTileGroup, past_caches, rm,
                                    dhidden, RowCopy{}, nullptr);
}

// ---------------------------------------------------------------------------
// weights packed for the backward pass
// ---------------------------------------------------------------------------
// Both products sum over the rows' own direction of the matrices as they are given, so nothing is transposed: 16-byte pieces go to
// their place in the packed form, n the output column of the product, k the index summed over.  in [rows][len] of an expert
// (blockIdx.y): row -> n, column -> k; interleave: columns of W1 / W3 to the blocks of 32 that da / db have.  One thread per
// piece of the packed form; zeros past the matrix.
__global__ __launch_bounds__(256) void pack_rows_kernel(const bf16_t* __restrict__ in, bf16_t* __restrict__ out, int rows,
                                                        int len, int rows_out, int len_out, int K_out, size_t out_stride,
                                                        int interleave, int sel) {
    const bf16_t* src = in + (size_t)blockIdx.y * rows * len;
    bf16_t* dst = out + (size_t)blockIdx.y * out_stride;
    const int pieces = len_out / 8;
    const bool vec = len % 8 == 0 && (uintptr_t)in % 16 == 0;
    const int64_t total = (int64_t)rows_out * pieces;
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < total; i += (int64_t)gridDim.x * blockDim.x) {
        // 64 threads: 16 rows by four pieces, a fragment of the packed form
        const int64_t frag = i >> 6;
        const int quads = pieces / 4;
        const int n = (int)(frag / quads) * 16 + (int)(i & 15), c = ((int)(frag % quads) * 4 + (int)((i >> 4) & 3)) * 8;
        alignas(16) bf16_t v[8];
        if (vec && n < rows && c < len) {
            *(uint4*)v = *(const uint4*)(src + (size_t)n * len + c);
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q) v[q] = n < rows && c + q < len ? src[(size_t)n * len + c + q] : (bf16_t)0;
        }
        const int k = interleave ? (c / 32) * 64 + sel * 32 + c % 32 : c;
        *(uint4*)(dst + packed_index(n, k, K_out)) = *(const uint4*)v;
    }
}

// elements of one expert: W2 with ffn as columns of the product, [W1 W3] with d
static inline size_t packed_back2(int d, int fp) { return packed_rows((size_t)fp) * d; }
static inline size_t packed_back13(int n1, int d, int fp) { return packed_rows((size_t)d) * n1 * fp; }

// ---------------------------------------------------------------------------
// fp32
// ---------------------------------------------------------------------------
// 64 x 64 tiles, 32 of the sum at a time through LDS, four wavefronts of 16 rows each on the fp32 matrix instruction.
// The layers are small; what a tile costs is waiting, so the next step's values are requested before this one is multiplied, and
// steps are long (512 rows of 8 experts of 128 x 256: with steps of 16, rows looked up for every value, the two kernels take 35.4 and 23.5
// us instead of 25.4 and 23.2).
constexpr int kF32Tile = 64, kF32Step = 32, kF32Pitch = kF32Tile + 4;
struct F32Stage {
    float a[2][kF32Step][kF32Pitch], b[2][kF32Step][kF32Pitch];
};

// acc[j] += sum_k A(m, k) B(n, k) for the wavefront's 16 m and the four groups of 16 n; A_ALONG / B_ALONG: neighbouring
// k are neighbours in memory (else neighbouring m or n).  a(m), along: where the values of m begin, asked once, as its row may have
// to be looked up; else a(m, k): the value.
template <bool A_ALONG, bool B_ALONG, class FA, class FB>
__device__ __forceinline__ void f32_sum(F32Stage& sh, int K, FA&& a, FB&& b, f32x4 (&acc)[4]) {
    const int tid = threadIdx.x, lane = tid & 63, wave = tid >> 6, l16 = lane & 15, g16 = lane >> 4;
    constexpr int N = kF32Tile * kF32Step / 256;  // values of a thread
    float ra[N], rb[N];
    auto place = [&](bool along, int i, int& m, int& k) {
        const int v = tid + i % 4 * 256;  // of 64 x 16 values, which a wavefront stores to as many banks
        if (along) {
            k = v & 15;
            m = v >> 4;
        } else {
            m = v & 63;
            k = v >> 6;
        }
        k += i / 4 * 16;
    };
    const float *pa[N], *pb[N];
#pragma unroll
    for (int i = 0; i < N; ++i) {
        int m, k;
        place(A_ALONG, i, m, k);
        if constexpr (A_ALONG) pa[i] = a(m);
        place(B_ALONG, i, m, k);
        if constexpr (B_ALONG) pb[i] = b(m);
    }
    auto fetch = [&](int k0) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int m, k;
            place(A_ALONG, i, m, k);
            if constexpr (A_ALONG) ra[i] = k0 + k < K ? pa[i][k0 + k] : 0.f;
            else ra[i] = k0 + k < K ? a(m, k0 + k) : 0.f;
            place(B_ALONG, i, m, k);
            if constexpr (B_ALONG) rb[i] = k0 + k < K ? pb[i][k0 + k] : 0.f;
            else rb[i] = k0 + k < K ? b(m, k0 + k) : 0.f;
        }
    };
    fetch(0);
    for (int k0 = 0, u = 0; k0 < K; k0 += kF32Step, u ^= 1) {
#pragma unroll
        for (int i = 0; i < N; ++i) {
            int m, k;
            place(A_ALONG, i, m, k);
            sh.a[u][k][m] = ra[i];
            place(B_ALONG, i, m, k);
            sh.b[u][k][m] = rb[i];
        }
        __syncthreads();  // (the other buffer is written next, by wavefronts that are past this: one barrier a step)
        if (k0 + kF32Step < K) fetch(k0 + kF32Step);
#pragma unroll
        for (int s = 0; s < kF32Step / 4; ++s) {
            const float av = sh.a[u][4 * s + g16][wave * 16 + l16];
#pragma unroll
            for (int j = 0; j < 4; ++j)
                acc[j] = __builtin_amdgcn_mfma_f32_16x16x4f32(sh.b[u][4 * s + g16][j * 16 + l16], av, acc[j], 0, 0, 0);
        }
    }
    __syncthreads();
}

struct F32Backward {
    const float *x, *dy, *w1, *w3, *w2;  // w3: null in the ReLU form
    const int32_t *tokens, *rows;        // token and row of x_perm of every list position
    const MTile* tiles;
    const int32_t *counts, *bases;       // bases: null when there are no rows
    float *h, *da, *db, *dx, *dW1, *dW3, *dW2;
    int d, ffn, E;
};

__device__ __forceinline__ void zero(f32x4 (&v)[4]) {
#pragma unroll
    for (int j = 0; j < 4; ++j) v[j] = f32x4{0.f, 0.f, 0.f, 0.f};
}

// h, da and db of the listed rows
__global__ __launch_bounds__(256) void f32_hidden_kernel(F32Backward p) {
    __shared__ F32Stage sh;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g16 = lane >> 4;
    const int n_tiles = ceil_div(p.ffn, kF32Tile);
    const int64_t total = (int64_t)p.counts[kCntEntries] * n_tiles;
    for (int64_t t = blockIdx.x; t < total; t += gridDim.x) {
        const MTile mt = p.tiles[t / n_tiles];
        const int f0 = (int)(t % n_tiles) * kF32Tile;
        const size_t we = (size_t)mt.expert * p.d * p.ffn;
        f32x4 dh[4], a[4], b[4];
        zero(dh);
        zero(a);
        zero(b);
        auto row = [&](int m) { return mt.list0 + (m < mt.rows ? m : mt.rows - 1); };
        auto xv = [&](int m) { return p.x + (size_t)p.tokens[row(m)] * p.d; };
        auto col = [&](int n) { return f0 + n < p.ffn ? f0 + n : p.ffn - 1; };
        f32_sum<true, true>(sh, p.d, [&](int m) { return p.dy + (size_t)p.rows[row(m)] * p.d; },
                            [&](int n) { return p.w2 + we + (size_t)col(n) * p.d; }, dh);
        f32_sum<true, false>(sh, p.d, xv, [&](int n, int k) { return p.w1[we + (size_t)k * p.ffn + col(n)]; }, a);
        if (p.w3)
            f32_sum<true, false>(sh, p.d, xv, [&](int n, int k) { return p.w3[we + (size_t)k * p.ffn + col(n)]; }, b);
        const int m = wave * 16 + l16;
        if (m >= mt.rows) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j)
#pragma unroll
            for (int c = 0; c < 4; ++c) {
                const int f = f0 + j * 16 + 4 * g16 + c;
                if (f >= p.ffn) continue;
                const size_t at = (size_t)(mt.list0 + m) * p.ffn + f;
                const float g = a[j][c], dhv = dh[j][c];
                if (p.w3) {
                    const float s = 1.0f / (1.0f + expf(-g)), gs = g * s;
                    p.h[at] = gs * b[j][c];
                    p.db[at] = dhv * gs;
                    p.da[at] = dhv * b[j][c] * (s + gs * (1.0f - s));
                } else {
                    p.h[at] = fmaxf(g, 0.f);
                    p.da[at] = g > 0.f ? dhv : 0.f;
                }
            }
    }
}

// dx, dW1, dW3 and dW2, side by side in one launch
__global__ __launch_bounds__(256) void f32_grads_kernel(F32Backward p) {
    __shared__ F32Stage sh;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6, l16 = lane & 15, g16 = lane >> 4;
    const int d_tiles = ceil_div(p.d, kF32Tile), f_tiles = ceil_div(p.ffn, kF32Tile);
    const int64_t n_dx = p.dx && p.bases ? (int64_t)p.counts[kCntEntries] * d_tiles : 0;
    const int64_t per = (int64_t)d_tiles * f_tiles;             // tiles of one matrix
    const int matrices = !p.dW1 ? 0 : p.w3 ? 3 : 2;
    const int64_t total = n_dx + (int64_t)p.E * per * matrices;
    for (int64_t t = blockIdx.x; t < total; t += gridDim.x) {
        f32x4 acc[4];
        zero(acc);
        const int mm = wave * 16 + l16;
        float* out;
        int n0, n_out;
        bool on;
        if (t < n_dx) {
            const MTile mt = p.tiles[t / d_tiles];
            n0 = (int)(t % d_tiles) * kF32Tile;
            n_out = p.d;
            const size_t we = (size_t)mt.expert * p.d * p.ffn;
            auto row = [&](int m) { return (size_t)(mt.list0 + (m < mt.rows ? m : mt.rows - 1)) * p.ffn; };
            auto col = [&](int n) { return (size_t)(n0 + n < p.d ? n0 + n : p.d - 1) * p.ffn; };
            f32_sum<true, true>(sh, p.ffn, [&](int m) { return p.da + row(m); },
                                [&](int n) { return p.w1 + we + col(n); }, acc);
            if (p.w3)
                f32_sum<true, true>(sh, p.ffn, [&](int m) { return p.db + row(m); },
                                    [&](int n) { return p.w3 + we + col(n); }, acc);
            on = mm < mt.rows;
            out = p.dx + (size_t)p.rows[mt.list0 + (on ? mm : 0)] * p.d;
        } else {
            const int64_t v = t - n_dx;
            const int e = (int)(v / (per * matrices));
            const int64_t in_e = v - (int64_t)e * per * matrices;
            const int which = (int)(in_e / per), at = (int)(in_e % per);  // 0: dW1, 1: dW2, 2: dW3
            const int first = p.bases ? p.bases[e] : 0, n = p.bases ? p.bases[e + 1] - first : 0;
            const bool second = which == 1;
            const int tiles = second ? d_tiles : f_tiles;
            const int M = second ? p.ffn : p.d;
            n_out = second ? p.d : p.ffn;
            n0 = at % tiles * kF32Tile;
            const int m0 = at / tiles * kF32Tile;
            auto mc = [&](int m) { return m0 + m < M ? m0 + m : M - 1; };
            auto nc = [&](int c) { return n0 + c < n_out ? n0 + c : n_out - 1; };
            if (second) {
                f32_sum<false, false>(sh, n, [&](int m, int k) { return p.h[(size_t)(first + k) * p.ffn + mc(m)]; },
                                      [&](int c, int k) { return p.dy[(size_t)p.rows[first + k] * p.d + nc(c)]; }, acc);
            } else {
                const float* g = which == 0 ? p.da : p.db;
                f32_sum<false, false>(sh, n, [&](int m, int k) { return p.x[(size_t)p.tokens[first + k] * p.d + mc(m)]; },
                                      [&](int c, int k) { return g[(size_t)(first + k) * p.ffn + nc(c)]; }, acc);
            }
            on = m0 + mm < M;
            out = (second ? p.dW2 : which == 0 ? p.dW1 : p.dW3) + (size_t)e * p.d * p.ffn + (size_t)(m0 + (on ? mm : 0)) * n_out;
        }
        if (!on) continue;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const int c = n0 + j * 16 + 4 * g16;  // (d and ffn are multiples of four)
            if (c < n_out) *(f32x4_any*)(out + c) = acc[j];
        }
    }
}

// ---------------------------------------------------------------------------
// host side
// ---------------------------------------------------------------------------
struct BackwardWs {
    void* x;             // [T, d] rows of x, from a checkpoint
    float* dhidden;      // [A, fp] dh (bf16)
    void *hidden, *dab;  // [A, fp] h; [A, n1 * fp] da (and db)
    int32_t *rows, *tokens, *bases;
    MTile *tiles1, *tiles2;
    int32_t *counts, *queues;
    int capacity;
};
constexpr int kBackwardQueues = 5 * 8;  // claim counters of the three products and of the weight gradients

static size_t backward_layout(int64_t T, int k, int d, int ffn, int E, int nseg, int dtype, int relu, char* base,
                              BackwardWs* ws) {
    size_t off = 0;
    auto take = [&](size_t bytes) {
        void* p = base ? (void*)(base + off) : nullptr;
        off += align_up(bytes, 256);
        return p;
    };
    const int64_t A = T * k, A1 = A > 0 ? A : 1, T1 = T > 0 ? T : 1;
    const size_t size = (size_t)dtype_size(dtype), fp = (size_t)padded_ffn(ffn, dtype);
    BackwardWs w;
    w.capacity = (int)(ceil_div64(A1, kMinBM) + nseg);
    w.x = take((size_t)T1 * d * size);
    w.dhidden = (float*)take(dtype == MOE_DTYPE_BF16 ? (size_t)A1 * fp * sizeof(float) : 0);
    w.hidden = take((size_t)A1 * fp * size);
    w.dab = take((size_t)A1 * fp * size * (relu ? 1 : 2));
    w.rows = (int32_t*)take((size_t)A1 * sizeof(int32_t));
    w.tokens = (int32_t*)take((size_t)A1 * sizeof(int32_t));
    w.bases = (int32_t*)take(((size_t)E + 1) * sizeof(int32_t));
    w.tiles1 = (MTile*)take((size_t)w.capacity * sizeof(MTile));
    w.tiles2 = (MTile*)take((size_t)w.capacity * sizeof(MTile));
    w.counts = (int32_t*)take((2 * kCntStride + kBackwardQueues) * sizeof(int32_t));
    w.queues = w.counts ? w.counts + 2 * kCntStride : nullptr;
    if (ws) *ws = w;
    return off;
}

static bool backward_in_range(int T, int k, int d, int ffn, int E, int nseg, int dtype) {
    return T >= 0 && k >= 1 && k <= MOE_MAX_TOPK && E >= 1 && E <= MOE_MAX_EXPERTS &&
           ffn_shape_in_range((int64_t)T * k, d, ffn, nseg, dtype);
}

// workgroups of a launch that goes round its tiles
static unsigned tile_grid(int64_t tiles) { return (unsigned)(tiles < 1 ? 1 : tiles < (1 << 20) ? tiles : 1 << 20); }

// Rows per expert, on average, up to which the gradients of the weights are made by small tiles.  Whole calls, us, large tiles -> small,
// popularity 10 / 0.1: 128 experts of 4096 x 1536, 0.1 rows per expert 1368 -> 1066 / 1337 -> 1064, 8 2686 -> 2141 / 1632 -> 1328, 32
// 2925 -> 2668 / 1927 -> 1712, 128 3462 -> 3713 / 2544 -> 2993; 8 of 4096 x 14336, 8 1745 -> 1430 / 1255 -> 1007, 32 1838 -> 1592 /
// 1258 -> 1120, 128 2122 -> 2046 / 1595 -> 1591; 64 of 2048 x 1408, 12 575 -> 505 / 561 -> 491, 48 747 -> 726 / 763 -> 732, 96 879 ->
// 887 / 862 -> 903; 64 of 768 x 3072 (ReLU), 8 378 -> 310 / 257 -> 239, 32 439 -> 418 / 316 -> 351, 64 474 -> 487 / 368 -> 452.
// The mean is all that the host knows; at the rule's edge either side can be up to 11 % the slower, as widths and popularity have it.
// The results are the same bits: either sums an expert's rows 32 at a time in their order.
constexpr int kFewRows = 32;

template <bool PAIR>
static int launch_weight_grads(const WeightGrad& w13, const WeightGrad& w2, const int32_t* bases, int32_t* queues, int64_t A, int E,
                               hipStream_t st) {
    if (A <= (int64_t)kFewRows * E) {
        const int64_t tiles13 = few_rows_tiles(w13, E), tiles = tiles13 + few_rows_tiles(w2, E);
        hipLaunchKernelGGL(few_rows_grads_kernel<PAIR>, dim3(tile_grid(tiles)), dim3(256), 0, st, w13, w2, bases, tiles13, tiles);
        return check_launch();
    }
    const auto kern = weight_grads_kernel<PAIR>;
    static std::atomic<unsigned long long> raised{0};
    if (const int rc = raise_lds((const void*)kern, grad_lds(MOE_MAX_EXPERTS), raised); rc != MOE_OK) return rc;
    hipLaunchKernelGGL(kern, dim3(kGemmGrid), dim3(512), grad_lds(E), st, w13, w2, bases, queues, E);
    return check_launch();
}

template <int EPI>
static int launch_hidden_grad(const bf16_t* x, int d, const bf16_t* p13, size_t stride, int E, const BackwardWs& ws, int N,
                              const RowMap& rm, hipStream_t st) {
    const auto kern = hidden_grad_kernel<EPI>;
    static std::atomic<unsigned long long> raised{0};
    if (const int rc = raise_lds((const void*)kern, kTileLds<EPI>, raised); rc != MOE_OK) return rc;
    hipLaunchKernelGGL(kern, dim3(kGemmGrid), dim3(512), kTileLds<EPI>, st, x, d, p13, stride, (bf16_t*)ws.dab, ws.tiles1,
                       ws.counts, ws.queues + 8, N, past_caches(E, stride), rm, ws.dhidden, (bf16_t*)ws.hidden);
    return check_launch();
}

static int launch_dhidden(const bf16_t* dy, int d, const bf16_t* p2, size_t stride, int E, const BackwardWs& ws, int N,
                          const RowMap& rm, hipStream_t st) {
    static std::atomic<unsigned long long> raised{0};
    if (const int rc = raise_lds((const void*)dhidden_kernel, kTileLds<kEpiFloat>, raised); rc != MOE_OK) return rc;
    hipLaunchKernelGGL(dhidden_kernel, dim3(kGemmGrid), dim3(512), kTileLds<kEpiFloat>, st, dy, d, p2, stride, ws.dhidden,
                       ws.tiles1, ws.counts, ws.queues, N, past_caches(E, stride), rm);
    return check_launch();
}

static int backward_f32(const moe_ffn_backward_args& a, const float* x, const BackwardWs& ws, hipStream_t st) {
    const size_t per = (size_t)a.E * a.d * a.ffn;
    const float* w1 = (const float*)a.packed;
    const float* w3 = a.relu ? nullptr : w1 + per;
    const bool any = a.T > 0;
    float* da = (float*)ws.dab;
    const F32Backward p{x, (const float*)a.dy_perm, w1, w3, w1 + (a.relu ? 1 : 2) * per, ws.tokens, ws.rows, ws.tiles1, ws.counts,
                        any ? ws.bases : nullptr, (float*)ws.hidden, da, da + (size_t)a.T * a.k * a.ffn, (float*)a.dx_perm,
                        (float*)a.dW1, (float*)a.dW3, (float*)a.dW2, a.d, a.ffn, a.E};
    const int64_t rows64 = ceil_div64((int64_t)a.T * a.k, kF32Tile) + (a.nseg < a.E ? a.nseg : a.E);  // most tiles of rows
    const int64_t dt = ceil_div(a.d, kF32Tile), ft = ceil_div(a.ffn, kF32Tile);
    if (any) {
        hipLaunchKernelGGL(f32_hidden_kernel, dim3(tile_grid(rows64 * ft)), dim3(256), 0, st, p);
        if (const int rc = check_launch(); rc != MOE_OK) return rc;
    }
    const int64_t tiles = (any && a.dx_perm ? rows64 * dt : 0) + (a.dW1 ? (int64_t)a.E * dt * ft * (a.relu ? 2 : 3) : 0);
    if (tiles == 0) return MOE_OK;
    hipLaunchKernelGGL(f32_grads_kernel, dim3(tile_grid(tiles)), dim3(256), 0, st, p);
    return check_launch();
}

static int backward_bf16(const moe_ffn_backward_args& a, const bf16_t* x, const BackwardWs& ws, hipStream_t st) {
    const int n1 = a.relu ? 1 : 2, fp = padded_ffn(a.ffn, MOE_DTYPE_BF16), d = a.d;
    const bf16_t* p13 = (const bf16_t*)a.packed;
    const bf16_t* back2 = (const bf16_t*)a.packed_backward;
    const bf16_t* back13 = back2 + (size_t)a.E * packed_back2(d, fp);
    bf16_t *hidden = (bf16_t*)ws.hidden, *dab = (bf16_t*)ws.dab;
    int rc = MOE_OK;
    const RowMap by_row{ws.rows, nullptr, 1, nullptr, nullptr, nullptr}, by_token{ws.tokens, nullptr, 1, nullptr, nullptr, nullptr};
    if (a.T > 0) {
        rc = launch_dhidden((const bf16_t*)a.dy_perm, d, back2, packed_back2(d, fp), a.E, ws, fp, by_row, st);
        if (rc == MOE_OK)
            rc = a.relu ? launch_hidden_grad<kEpiReluGrad>(x, d, p13, packed_elems1(1, d, fp), a.E, ws, fp, by_token, st)
                        : launch_hidden_grad<kEpiSwigluGrad>(x, d, p13, packed_elems1(2, d, fp), a.E, ws, 2 * fp, by_token, st);
    }
    if (rc == MOE_OK && a.dW1) {
        const WeightGrad w13{x, dab, ws.tokens, d, n1 * fp, {(bf16_t*)a.dW1, (bf16_t*)a.dW3}, d, n1 * fp, d, a.ffn};
        const WeightGrad w2{hidden, (const bf16_t*)a.dy_perm, ws.rows, fp, d, {(bf16_t*)a.dW2, nullptr}, fp, d, a.ffn, d};
        const int32_t* bases = a.T > 0 ? ws.bases : nullptr;
        const int64_t A = (int64_t)a.T * a.k;
        rc = a.relu ? launch_weight_grads<false>(w13, w2, bases, ws.queues + 24, A, a.E, st)
                    : launch_weight_grads<true>(w13, w2, bases, ws.queues + 24, A, a.E, st);
    }
    if (rc == MOE_OK && a.T > 0 && a.dx_perm) {
        const RowMap to_row{nullptr, nullptr, 1, ws.rows, nullptr, nullptr};
        rc = launch_product(dab, n1 * fp, back13, packed_back13(n1, d, fp), a.E, (bf16_t*)a.dx_perm, d, ws.tiles2,
                            ws.counts + kCntStride, ws.queues + 16, d, n1 * fp, to_row, st);
    }
    return rc;
}

}  // namespace moegps

extern "C" size_t moe_packed_weights_backward_bytes(int E, int d, int ffn, int dtype, int relu) {
    using namespace moegps;
    if (E < 1 || E > MOE_MAX_EXPERTS || !ffn_shape_in_range(0, d, ffn, 1, dtype)) return 0;
    if (dtype != MOE_DTYPE_BF16) return 0;
    const int fp = padded_ffn(ffn, dtype);
    return (size_t)E * (packed_back2(d, fp) + packed_back13(relu ? 1 : 2, d, fp)) * sizeof(bf16_t);
}

extern "C" int moe_pack_weights_backward(const void* W1, const void* W3, const void* W2, int dtype, int E, int d, int ffn,
                                         void* packed, void* stream) {
    using namespace moegps;
    if (dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_INVALID_ARG;
    if (E < 1 || d < 1 || ffn < 1) return MOE_ERR_INVALID_ARG;
    if (E > MOE_MAX_EXPERTS || d > kMaxWidth || ffn > kMaxWidth) return MOE_ERR_UNSUPPORTED;
    if (dtype == MOE_DTYPE_F32) return MOE_OK;  // the forward pass's packed form serves both
    if (d % 64 != 0) return MOE_ERR_UNSUPPORTED;
    if (!W1 || !W2 || !packed) return MOE_ERR_INVALID_ARG;
    const int fp = padded_ffn(ffn, dtype), n1 = W3 ? 2 : 1;
    bf16_t* back2 = (bf16_t*)packed;
    bf16_t* back13 = back2 + (size_t)E * packed_back2(d, fp);
    auto pack = [&](const void* W, bf16_t* out, int rows, int len, int len_out, int K_out, size_t stride, int interleave, int sel) {
        const int rows_out = (int)packed_rows((size_t)rows);
        const int64_t blocks = ceil_div64((int64_t)rows_out * (len_out / 8), 256);
        hipLaunchKernelGGL(pack_rows_kernel, dim3((unsigned)(blocks < 4096 ? blocks : 4096), (unsigned)E), dim3(256), 0,
                           (hipStream_t)stream, (const bf16_t*)W, out, rows, len, rows_out, len_out, K_out, stride, interleave,
                           sel);
        return check_launch();
    };
    int rc = pack(W2, back2, ffn, d, d, d, packed_back2(d, fp), 0, 0);
    if (rc == MOE_OK) rc = pack(W1, back13, d, ffn, fp, n1 * fp, packed_back13(n1, d, fp), W3 ? 1 : 0, 0);
    if (rc == MOE_OK && W3) rc = pack(W3, back13, d, ffn, fp, n1 * fp, packed_back13(n1, d, fp), 1, 1);
    return rc;
}

extern "C" size_t moe_grouped_ffn_backward_workspace_bytes(int T, int k, int d, int ffn, int E, int nseg, int dtype, int relu) {
    using namespace moegps;
    if (!backward_in_range(T, k, d, ffn, E, nseg, dtype)) return 0;
    return backward_layout(T, k, d, ffn, E, nseg, dtype, relu, nullptr, nullptr);
}

extern "C" int moe_grouped_ffn_backward(const moe_ffn_backward_args* args, void* stream) {
    using namespace moegps;
    if (!args) return MOE_ERR_INVALID_ARG;
    const moe_ffn_backward_args a = *args;
    if (a.dtype != MOE_DTYPE_F32 && a.dtype != MOE_DTYPE_BF16) return MOE_ERR_INVALID_ARG;
    if (a.T < 0 || a.k < 1 || a.d < 1 || a.ffn < 1 || a.E < 1 || a.nseg < 1) return MOE_ERR_INVALID_ARG;
    if (!backward_in_range(a.T, a.k, a.d, a.ffn, a.E, a.nseg, a.dtype)) return MOE_ERR_UNSUPPORTED;
    const bool bf16 = a.dtype == MOE_DTYPE_BF16;
    if (bf16 ? a.d % 64 != 0 : a.d % 4 != 0 || a.ffn % 4 != 0) return MOE_ERR_UNSUPPORTED;
    if ((int64_t)256 * (a.d > a.ffn + 63 ? a.d : a.ffn + 63) * 2 >= (1ll << 31)) return MOE_ERR_UNSUPPORTED;  // 32-bit tile offsets
    // the product for dx sums over da's and db's columns: no more of them than the widest matrix has (a panel's 32-bit offsets)
    if (bf16 && a.dx_perm && (int64_t)(a.relu ? 1 : 2) * padded_ffn(a.ffn, a.dtype) > kMaxWidth) return MOE_ERR_UNSUPPORTED;
    const int64_t A = (int64_t)a.T * a.k;
    if (bf16 && A * a.d >= (1ll << 31)) return MOE_ERR_UNSUPPORTED;  // 32-bit row offsets
    if (!a.packed || (bf16 && !a.packed_backward) || !a.workspace) return MOE_ERR_INVALID_ARG;
    if (!a.dW1 != !a.dW2 || (a.relu ? a.dW3 != nullptr : !a.dW3 != !a.dW1)) return MOE_ERR_INVALID_ARG;
    if (a.T > 0 && (!a.x || !a.assign_of_row || !a.seg_offsets || !a.slot_expert || !a.dy_perm)) return MOE_ERR_INVALID_ARG;
    BackwardWs ws;
    const size_t need = backward_layout(a.T, a.k, a.d, a.ffn, a.E, a.nseg, a.dtype, a.relu, (char*)a.workspace, &ws);
    if (a.workspace_bytes < need) return MOE_ERR_WORKSPACE_TOO_SMALL;
    if (!a.dW1 && (a.T == 0 || !a.dx_perm)) return MOE_OK;  // nothing is wanted
    hipStream_t st = (hipStream_t)stream;
    const void* x = a.x;
    if (a.T > 0) {
        if (a.x_scales) {
            if (const int rc = checkpoint_load((const uint8_t*)a.x, a.x_scales, a.T, a.d, ws.x, a.dtype, st); rc != MOE_OK) return rc;
            x = ws.x;
        }
        const int n1 = a.relu ? 1 : 2, fp = padded_ffn(a.ffn, a.dtype);
        const TableSpec t1{ws.tiles1, ws.counts, nullptr, bf16 ? 0 : kF32Tile, ws.capacity, a.d / kPackK, 0,
                           ceil_div(n1 * fp, kPackN), 0, 0};
        const TableSpec t2{bf16 ? ws.tiles2 : nullptr, ws.counts + kCntStride, nullptr, 0, ws.capacity, n1 * fp / kPackK, 0,
                           ceil_div(a.d, kPackN), 0, 0};
        const RowLists lists{ws.rows, ws.tokens, a.assign_of_row, a.k};
        const TableJob job{a.E, 0, a.nseg, t1, t2, lists, ws.queues, kBackwardQueues, nullptr, ws.bases};
        if (const int rc = launch_tables(A, a.seg_offsets, a.slot_expert, job, st); rc != MOE_OK) return rc;
    }
    return bf16 ? backward_bf16(a, (const bf16_t*)x, ws, st) : backward_f32(a, (const float*)x, ws, st);
}
