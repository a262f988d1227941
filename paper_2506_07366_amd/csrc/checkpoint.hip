// Activation checkpoints in 8 bits: rows kept between the forward and the backward pass as e4m3 codes with a
// power-of-two scale for every 32 values of a row,
//     s = 2^e, e the smallest with max|x| <= 448 * 2^e;   code = e4m3(x / s);   back = code * s.
// A power of two makes the division, the way back and the bf16 that comes of it exact: the one rounding is that to
// four significant bits (half a step, 2^-4 of a value at most; values below 2^-6 s have the step 2^-9 s).  With a full scale
// max|x| / 448 a value would be rounded again to bf16 on the way back, for half a bit of range on average.
//
// Bound by memory: 2 (fp32: 4) bytes of a value one way and 1 + 1/32 the other.  A lane takes 8 values as one or two 16-byte
// loads and stores their 8 codes, four neighbouring lanes make a group (two DPP steps give its maximum), a few pieces per
// lane are under way at a time.
#include "checkpoint.h"

namespace moegps {

// maximum over four neighbouring lanes of non-negative ints
__device__ __forceinline__ int quad_max(int v) {
    int o = __builtin_amdgcn_update_dpp(0, v, 0xb1, 0xf, 0xf, true);  // quad_perm [1, 0, 3, 2]
    v = o > v ? o : v;
    o = __builtin_amdgcn_update_dpp(0, v, 0x4e, 0xf, 0xf, true);      // quad_perm [2, 3, 0, 1]
    return o > v ? o : v;
}

// Biased exponent of the scale of a group whose largest finite magnitude has the bits `top`: 448 = 1.75 * 2^8, so
// the exponent of `top` less 8, one more above 1.75; 1 for nothing but zeros.
__device__ __forceinline__ int scale_of(int top) {
    const int b = ((top + 0x1fffff) >> 23) - 8;
    return top == 0 ? 127 : b < 1 ? 1 : b;
}

// One pass over the rows: f(row, piece, lanes) for pieces piece + u * lanes, u < UNROLL, of a row, called by all lanes that
// share the row, also past its end and past the last row.
template <int UNROLL, class F>
__device__ __forceinline__ void walk_rows(const RowWalk& w, F&& f) {
    const int lane = threadIdx.x & (kWave - 1);
    const int lanes = 1 << w.log_lanes;
    const int per_wave = kWave >> w.log_lanes;  // rows
    const int64_t n_waves = (int64_t)gridDim.x * (blockDim.x / kWave);
    for (int64_t wave = (int64_t)blockIdx.x * (blockDim.x / kWave) + (threadIdx.x / kWave);
         wave / w.slices * per_wave < w.rows; wave += n_waves) {
        const int slice = (int)(wave % w.slices);
        const int64_t row = (wave / w.slices) * per_wave + (lane >> w.log_lanes);
        for (int p0 = slice * lanes * UNROLL; p0 < w.pieces; p0 += lanes * UNROLL * w.slices)
            f(row, p0 + (lane & (lanes - 1)), lanes);
    }
}

template <bool BF16, int UNROLL>
__global__ __launch_bounds__(256) void checkpoint_store_kernel(const void* __restrict__ x, uint8_t* __restrict__ codes,
                                                                uint8_t* __restrict__ scales, int d, RowWalk w) {
    const int groups = groups_of(d);
    walk_rows<UNROLL>(w, [&](int64_t row, int piece0, int lanes) {
        u32x4 raw[UNROLL][BF16 ? 1 : 2];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int piece = piece0 + u * lanes;
            const bool in = row < w.rows && piece < w.pieces;
            const size_t at = (size_t)row * d + (size_t)piece * kPiece;
#pragma unroll
            for (int h = 0; h < (BF16 ? 1 : 2); ++h) {
                // (fp32 rows are multiples of four values: a row's last piece may be half a one)
                const bool on = in && (BF16 || piece * kPiece + h * 4 < d);
                raw[u][h] = u32x4{0, 0, 0, 0};
                if (on)
                    raw[u][h] = __builtin_nontemporal_load(
                        (const u32x4*)((const char*)x + at * (BF16 ? 2 : 4) + h * 16));
            }
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int piece = piece0 + u * lanes;
            const bool in = row < w.rows && piece < w.pieces;
            unsigned v[kPiece];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                if constexpr (BF16) {
                    const unsigned bits = raw[u][0][i];
                    v[2 * i] = bits << 16;
                    v[2 * i + 1] = bits & 0xffff0000u;
                } else {
                    v[i] = raw[u][0][i];
                    v[4 + i] = raw[u][1][i];
                }
            }
            int top = 0;  // the largest finite magnitude; what is infinite or not a number becomes that of the codes
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                const int m = (int)(v[i] & 0x7fffffffu);
                top = m < 0x7f800000 && m > top ? m : top;
            }
            const int biased = scale_of(quad_max(top));
            const float inv = exp2_biased(254 - biased);  // (biased is 247 at most: its reciprocal is a normal number)
            const float most = biased == 247 ? 240.f : 448.f;  // 256 * 2^120 would be infinite on the way back
            float f[kPiece];
#pragma unroll
            for (int i = 0; i < kPiece; ++i) {
                const float q = fminf(fmaxf(__builtin_bit_cast(float, v[i]) * inv, -most), most);
                f[i] = (v[i] & 0x7f800000u) == 0x7f800000u ? __builtin_nanf("") : q;  // e4m3 has no infinity
            }
            u32x2 c;
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                int word = __builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h], f[4 * h + 1], 0, false);
                c[h] = (unsigned)__builtin_amdgcn_cvt_pk_fp8_f32(f[4 * h + 2], f[4 * h + 3], word, true);
            }
            if (in) {
                uint8_t* to = codes + (size_t)row * d + (size_t)piece * kPiece;
                if (BF16) {
                    __builtin_nontemporal_store(c, (u32x2*)to);
                } else {  // rows of codes start at multiples of four bytes
                    *(unsigned*)to = c[0];
                    if (piece * kPiece + 4 < d) *(unsigned*)(to + 4) = c[1];
                }
                if ((piece & 3) == 0) scales[(size_t)row * groups + piece / 4] = (uint8_t)biased;
            }
        }
    });
}

template <bool BF16, int UNROLL>
__global__ __launch_bounds__(256) void checkpoint_load_kernel(const uint8_t* __restrict__ codes,
                                                               const uint8_t* __restrict__ scales, void* __restrict__ x,
                                                               int d, RowWalk w) {
    const int groups = groups_of(d);
    walk_rows<UNROLL>(w, [&](int64_t row, int piece0, int lanes) {
        u32x2 c[UNROLL];
        int biased[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int piece = piece0 + u * lanes;
            c[u] = u32x2{0, 0};
            biased[u] = 127;
            if (row >= w.rows || piece >= w.pieces) continue;
            const uint8_t* from = codes + (size_t)row * d + (size_t)piece * kPiece;
            if (BF16) {
                c[u] = __builtin_nontemporal_load((const u32x2*)from);
            } else {
                c[u][0] = *(const unsigned*)from;
                if (piece * kPiece + 4 < d) c[u][1] = *(const unsigned*)(from + 4);
            }
            biased[u] = scales[(size_t)row * groups + piece / 4];
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            const int piece = piece0 + u * lanes;
            if (row >= w.rows || piece >= w.pieces) continue;
            const float s = exp2_biased(biased[u]);
            float lo[4], hi[4];
            codes_to_float(c[u][0], s, lo);
            codes_to_float(c[u][1], s, hi);
            const size_t at = (size_t)row * d + (size_t)piece * kPiece;
            if constexpr (BF16) {
                const u32x4 o = {bf16_pair(lo[0], lo[1]), bf16_pair(lo[2], lo[3]), bf16_pair(hi[0], hi[1]),
                                 bf16_pair(hi[2], hi[3])};
                __builtin_nontemporal_store(o, (u32x4*)((char*)x + at * 2));
            } else {
                typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f4;
                *(f4*)((char*)x + at * 4) = f4{lo[0], lo[1], lo[2], lo[3]};
                if (piece * kPiece + 4 < d) *(f4*)((char*)x + at * 4 + 16) = f4{hi[0], hi[1], hi[2], hi[3]};
            }
        }
    });
}

static int check_rows(int dtype, int64_t rows, int d) {
    if (dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) return MOE_ERR_INVALID_ARG;
    if (rows < 0 || d < 1) return MOE_ERR_INVALID_ARG;
    if ((size_t)d * dtype_size(dtype) % 16 != 0 || rows >= (1ll << 31) || d > (1 << 22)) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

static int walk_unroll(int pieces) { return pieces >= 4 * kWave ? 4 : pieces >= 2 * kWave ? 2 : 1; }

int checkpoint_load(const uint8_t* codes, const uint8_t* scales, int64_t rows, int d, void* x, int dtype, hipStream_t st) {
    const int pieces = ceil_div(d, kPiece), unroll = walk_unroll(pieces);
    const RowWalk w = row_walk(rows, pieces, unroll);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(row_walk_blocks(w)), dim3(256), 0, st, codes, scales, x, d, w);
        return check_launch();
    };
    if (dtype == MOE_DTYPE_BF16)
        return unroll == 4 ? go(checkpoint_load_kernel<true, 4>)
                           : unroll == 2 ? go(checkpoint_load_kernel<true, 2>) : go(checkpoint_load_kernel<true, 1>);
    return unroll == 4 ? go(checkpoint_load_kernel<false, 4>)
                       : unroll == 2 ? go(checkpoint_load_kernel<false, 2>) : go(checkpoint_load_kernel<false, 1>);
}

}  // namespace moegps

extern "C" int moe_checkpoint_store(const void* x, int dtype, int64_t rows, int d, uint8_t* codes, uint8_t* scales,
                                    void* stream) {
    using namespace moegps;
    if (const int rc = check_rows(dtype, rows, d); rc != MOE_OK) return rc;
    if (rows == 0) return MOE_OK;
    if (!x || !codes || !scales) return MOE_ERR_INVALID_ARG;
    const int pieces = ceil_div(d, kPiece), unroll = walk_unroll(pieces);
    const RowWalk w = row_walk(rows, pieces, unroll);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(row_walk_blocks(w)), dim3(256), 0, (hipStream_t)stream, x,
                           codes, scales, d, w);
        return check_launch();
    };
    if (dtype == MOE_DTYPE_BF16)
        return unroll == 4 ? go(checkpoint_store_kernel<true, 4>)
                           : unroll == 2 ? go(checkpoint_store_kernel<true, 2>) : go(checkpoint_store_kernel<true, 1>);
    return unroll == 4 ? go(checkpoint_store_kernel<false, 4>)
                       : unroll == 2 ? go(checkpoint_store_kernel<false, 2>) : go(checkpoint_store_kernel<false, 1>);
}

extern "C" int moe_checkpoint_load(const uint8_t* codes, const uint8_t* scales, int64_t rows, int d, void* x, int dtype,
                                   void* stream) {
    using namespace moegps;
    if (const int rc = check_rows(dtype, rows, d); rc != MOE_OK) return rc;
    if (rows == 0) return MOE_OK;
    if (!x || !codes || !scales) return MOE_ERR_INVALID_ARG;
    return checkpoint_load(codes, scales, rows, d, x, dtype, (hipStream_t)stream);
}
