// Gradient of the weighted un-permute (combine.hip), out[t] = sum_j w[t, j] y[row(t, j)]:
//     dy[row(t, j)] = w[t, j] dout[t],   dw[t, j] = <dout[t], y[row(t, j)]>
// and of the gate behind it, w[t] = softmax of the k selected logits of token t:
//     dlogits[t, e_j] = w[t, j] (dw[t, j] - sum_i w[t, i] dw[t, i]),   0 for the other experts.
// Stands where the gradients of the return all-to-all are (Background, communication paragraph).
//
// Bound by memory: dout once, the k rows of y (as they are, or as an 8-bit checkpoint), the k rows of dy.  The
// wavefronts of a token deal its row among them in pieces of 8 values per lane; a piece of dout serves all k rows, whose
// loads are under way together.  The k products are summed in fp32: lane by lane, over the wavefront by DPP and LDS, over
// the token's wavefronts in LDS in their order.
#include "checkpoint.h"

namespace moegps {

enum Saved { kSavedNone, kSavedPlain, kSavedCodes };  // what is there of y

struct CombineBackward {
    const void* dout;
    const void* y;                  // rows of y in the layer's type, or their codes
    const uint8_t* scales;
    const int32_t *row_of_assign, *topk_idx;
    const float* topk_w;
    void* dy;
    float *dtopk_w, *dlogits;
    int T, d, k, E, pieces;
};

// sum over the wavefront, in every lane
__device__ __forceinline__ float wave_sum(float v) {
#pragma unroll
    for (int m = 32; m > 0; m >>= 1) v += __shfl_xor(v, m, kWave);
    return v;
}

// A piece as it lies in memory, and its values.
template <bool BF16>
struct Piece {
    u32x4 w[BF16 ? 1 : 2];
    // row: the row's first value, the same in all lanes; p: the lane's piece
    __device__ __forceinline__ void load(const char* row, unsigned p, bool whole) {
        const u32x4* q = (const u32x4*)(row + p * (kPiece * (BF16 ? 2u : 4u)));
        w[0] = __builtin_nontemporal_load(q);
        if constexpr (!BF16) {
            w[1] = u32x4{0, 0, 0, 0};
            if (whole) w[1] = __builtin_nontemporal_load(q + 1);
        }
    }
    __device__ __forceinline__ float value(int i) const {
        if constexpr (BF16) {
            const unsigned bits = w[0][i >> 1];
            return i & 1 ? bf16_hi(bits) : bf16_lo(bits);
        } else {
            const unsigned bits = w[i >> 2][i & 3];
            return __builtin_bit_cast(float, bits);
        }
    }
};

// KMAX: k rounded up.  A workgroup serves one token at a time.
template <bool BF16, int SAVED, int KMAX>
__global__ __launch_bounds__(1024) void combine_backward_kernel(CombineBackward a) {
    __shared__ float part[16][KMAX];
    const int lane = threadIdx.x & (kWave - 1);
    const int wave = __builtin_amdgcn_readfirstlane((int)(threadIdx.x / kWave));
    const int n_waves = blockDim.x / kWave;
    const int groups = groups_of(a.d);
    const size_t row_bytes = (size_t)a.d * (BF16 ? 2 : 4);
    for (int t = blockIdx.x; t < a.T; t += gridDim.x) {
        int rows[KMAX];
        float w[KMAX], dot[KMAX];
#pragma unroll
        for (int j = 0; j < KMAX; ++j) {
            if constexpr (KMAX <= 8) {  // all asked for at once: one token 9.2 -> 8.5 us (with 16 of them they leave the registers)
                const size_t at = (size_t)t * a.k + (j < a.k ? j : a.k - 1);
                rows[j] = a.row_of_assign[at];
                w[j] = a.topk_w[at];
            } else {
                rows[j] = j < a.k ? a.row_of_assign[(size_t)t * a.k + j] : 0;
                w[j] = j < a.k ? a.topk_w[(size_t)t * a.k + j] : 0.f;
            }
            dot[j] = 0.f;
        }
        for (int p = (int)threadIdx.x; p < a.pieces; p += blockDim.x) {
            const bool whole = BF16 || p * kPiece + 4 < a.d;  // (fp32 rows are multiples of four values)
            Piece<BF16> raw;
            raw.load((const char*)a.dout + (size_t)t * row_bytes, p, whole);
            // rows under way together: more of them would not leave the registers for a workgroup of 16 wavefronts
            constexpr int JW = KMAX < 8 ? KMAX : 8;
#pragma unroll
            for (int j0 = 0; j0 < KMAX; j0 += JW) {
                Piece<BF16> y[SAVED == kSavedPlain ? JW : 1];
                u32x2 codes[JW];
                int biased[JW];
#pragma unroll
                for (int jj = 0; jj < JW; ++jj) {
                    const int j = j0 + jj;
                    if (j >= a.k) continue;
                    if constexpr (SAVED == kSavedPlain) y[jj].load((const char*)a.y + (size_t)rows[j] * row_bytes, p, whole);
                    if constexpr (SAVED == kSavedCodes) {
                        const uint8_t* from = (const uint8_t*)a.y + (size_t)rows[j] * a.d + (unsigned)p * kPiece;
                        if (BF16) {
                            codes[jj] = __builtin_nontemporal_load((const u32x2*)from);
                        } else {
                            codes[jj][0] = *(const unsigned*)from;
                            codes[jj][1] = whole ? *(const unsigned*)(from + 4) : 0u;
                        }
                        biased[jj] = (a.scales + (size_t)rows[j] * groups)[(unsigned)p / 4];
                    }
                }
                float g[kPiece];
#pragma unroll
                for (int i = 0; i < kPiece; ++i) g[i] = raw.value(i);
#pragma unroll
                for (int jj = 0; jj < JW; ++jj) {
                    const int j = j0 + jj;
                    if (j >= a.k) continue;
                    if constexpr (SAVED == kSavedPlain) {
#pragma unroll
                        for (int i = 0; i < kPiece; ++i) dot[j] = fmaf(g[i], y[jj].value(i), dot[j]);
                    }
                    if constexpr (SAVED == kSavedCodes) {
                        // the scale is a power of two: taken out of the sum of a piece
                        float lo[4], hi[4], s = 0.f;
                        codes_to_float(codes[jj][0], 1.f, lo);
                        codes_to_float(codes[jj][1], 1.f, hi);
#pragma unroll
                        for (int i = 0; i < 4; ++i) s = fmaf(g[i], lo[i], s);
#pragma unroll
                        for (int i = 0; i < 4; ++i) s = fmaf(g[4 + i], hi[i], s);
                        dot[j] = fmaf(s, exp2_biased(biased[jj]), dot[j]);
                    }
                    float v[kPiece];
#pragma unroll
                    for (int i = 0; i < kPiece; ++i) v[i] = g[i] * w[j];
                    char* to = (char*)a.dy + (size_t)rows[j] * row_bytes + (unsigned)p * (kPiece * (BF16 ? 2u : 4u));
                    if constexpr (BF16) {
                        const u32x4 o = {bf16_pair(v[0], v[1]), bf16_pair(v[2], v[3]), bf16_pair(v[4], v[5]),
                                         bf16_pair(v[6], v[7])};
                        __builtin_nontemporal_store(o, (u32x4*)to);
                    } else {
                        typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f4;
                        f4* q = (f4*)to;
                        __builtin_nontemporal_store(f4{v[0], v[1], v[2], v[3]}, q);
                        if (whole) __builtin_nontemporal_store(f4{v[4], v[5], v[6], v[7]}, q + 1);
                    }
                }
            }
        }
        if constexpr (SAVED != kSavedNone) {
#pragma unroll
            for (int j = 0; j < KMAX; ++j)
                if (j < a.k) dot[j] = wave_sum(dot[j]);
            if (n_waves > 1) {
                if (lane == 0)
#pragma unroll
                    for (int j = 0; j < KMAX; ++j) part[wave][j] = dot[j];
                __syncthreads();
#pragma unroll
                for (int j = 0; j < KMAX; ++j) {
                    dot[j] = part[0][j];
                    for (int v = 1; v < n_waves; ++v) dot[j] += part[v][j];
                }
            }
            float mean = 0.f;
#pragma unroll
            for (int j = 0; j < KMAX; ++j)
                if (j < a.k) {
                    if (threadIdx.x == 0) a.dtopk_w[(size_t)t * a.k + j] = dot[j];
                    mean = fmaf(w[j], dot[j], mean);
                }
            if (a.dlogits) {
                int id[KMAX];
#pragma unroll
                for (int j = 0; j < KMAX; ++j) id[j] = j < a.k ? a.topk_idx[(size_t)t * a.k + j] : -1;
                for (int e = (int)threadIdx.x; e < a.E; e += blockDim.x) {
                    float v = 0.f;
#pragma unroll
                    for (int j = 0; j < KMAX; ++j) v = id[j] == e ? w[j] * (dot[j] - mean) : v;
                    a.dlogits[(size_t)t * a.E + e] = v;
                }
            }
            if (n_waves > 1) __syncthreads();  // (the next token's products go to the same place)
        }
    }
}

template <bool BF16, int SAVED>
static int launch_combine_backward(const CombineBackward& a, hipStream_t st) {
    // wavefronts of a token: one for every two pieces of a lane, more where there are few tokens
    int waves = ceil_div(a.pieces, 2 * kWave);
    if (a.T < 1024) waves = ceil_div(a.pieces, kWave);
    waves = waves < 1 ? 1 : waves > 16 ? 16 : waves;
    auto go = [&](auto kern) {
        // (a launch counts fewer than 2^32 threads; beyond that the workgroups go round)
        hipLaunchKernelGGL(kern, dim3((unsigned)(a.T < 1 << 21 ? a.T : 1 << 21)), dim3((unsigned)(waves * kWave)), 0, st, a);
        return check_launch();
    };
    if (a.k <= 2) return go(combine_backward_kernel<BF16, SAVED, 2>);
    if (a.k <= 4) return go(combine_backward_kernel<BF16, SAVED, 4>);
    if (a.k <= 8) return go(combine_backward_kernel<BF16, SAVED, 8>);
    return go(combine_backward_kernel<BF16, SAVED, 16>);
}

}  // namespace moegps

extern "C" int moe_combine_backward(const void* dout, int dtype, int T, int d, int k, int E, const int32_t* row_of_assign,
                                    const float* topk_w, const int32_t* topk_idx, const void* y_perm,
                                    const uint8_t* y_scales, void* dy_perm, float* dtopk_w, float* dlogits, void* stream) {
    using namespace moegps;
    if (dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_INVALID_ARG;
    if (T < 0 || d < 1 || k < 1) return MOE_ERR_INVALID_ARG;
    if (k > MOE_MAX_TOPK || (size_t)d * dtype_size(dtype) % 16 != 0 || d > (1 << 22)) return MOE_ERR_UNSUPPORTED;
    if ((int64_t)T * k >= (1ll << 31)) return MOE_ERR_UNSUPPORTED;
    if (dlogits) {
        if (!dtopk_w || E < k) return MOE_ERR_INVALID_ARG;
        if (E > MOE_MAX_EXPERTS) return MOE_ERR_UNSUPPORTED;
        if (T > 0 && !topk_idx) return MOE_ERR_INVALID_ARG;
    }
    if (y_scales && !y_perm) return MOE_ERR_INVALID_ARG;
    if (T == 0) return MOE_OK;
    if (!dout || !row_of_assign || !topk_w || !dy_perm) return MOE_ERR_INVALID_ARG;
    if ((dtopk_w != nullptr) != (y_perm != nullptr)) return MOE_ERR_INVALID_ARG;
    const CombineBackward a{dout, y_perm, y_scales, row_of_assign, topk_idx, topk_w, dy_perm, dtopk_w, dlogits, T, d, k, E,
                            ceil_div(d, kPiece)};
    hipStream_t st = (hipStream_t)stream;
    if (dtype == MOE_DTYPE_BF16)
        return !y_perm ? launch_combine_backward<true, kSavedNone>(a, st)
                       : y_scales ? launch_combine_backward<true, kSavedCodes>(a, st)
                                  : launch_combine_backward<true, kSavedPlain>(a, st);
    return !y_perm ? launch_combine_backward<false, kSavedNone>(a, st)
                   : y_scales ? launch_combine_backward<false, kSavedCodes>(a, st)
                              : launch_combine_backward<false, kSavedPlain>(a, st);
}
