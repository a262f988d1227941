// Rows kept in 8 bits (checkpoint.hip): what the kernels that read them share.
#pragma once
#include "common.h"
#include "../../include/moegps_train.h"

namespace moegps {

constexpr int kGroup = MOE_CHECKPOINT_GROUP;  // values that share a scale
constexpr int kPiece = 8;                     // values a lane holds at a time; four lanes hold a group

typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
typedef __attribute__((__vector_size__(2 * sizeof(unsigned)))) unsigned u32x2;
typedef __attribute__((__vector_size__(4 * sizeof(unsigned)))) unsigned u32x4;

__host__ __device__ inline int groups_of(int d) { return ceil_div(d, kGroup); }

// 2^(b - 127) for b in [1, 254]
__device__ __forceinline__ float exp2_biased(int b) { return __builtin_bit_cast(float, (unsigned)b << 23); }

// four codes -> the values they stand for
__device__ __forceinline__ void codes_to_float(unsigned codes, float scale, float (&v)[4]) {
    const f32x2 lo = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, false);
    const f32x2 hi = __builtin_amdgcn_cvt_pk_f32_fp8((int)codes, true);
    v[0] = lo[0] * scale;
    v[1] = lo[1] * scale;
    v[2] = hi[0] * scale;
    v[3] = hi[1] * scale;
}

// two bf16 of a word as floats, and back (nearest even)
__device__ __forceinline__ float bf16_lo(unsigned w) { return __builtin_bit_cast(float, w << 16); }
__device__ __forceinline__ float bf16_hi(unsigned w) { return __builtin_bit_cast(float, w & 0xffff0000u); }
__device__ __forceinline__ unsigned bf16_pair(float lo, float hi) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}

// How a wavefront goes over rows of `pieces` pieces: `lanes` lanes (a power of two, four at least) side by side on a
// row, 64 / lanes rows at a time; long rows of a small batch are cut into slices, a wavefront each.
struct RowWalk {
    int64_t rows;
    int pieces, log_lanes, slices;
};
inline RowWalk row_walk(int64_t rows, int pieces, int unroll) {
    RowWalk w{rows, pieces, 2, 1};
    while (w.log_lanes < 6 && (1 << w.log_lanes) < pieces) ++w.log_lanes;
    if (w.log_lanes == 6)
        while (w.slices < 16 && rows * w.slices < 4096 && pieces >= 2 * w.slices * kWave * unroll) w.slices *= 2;
    return w;
}
// workgroups of four wavefronts (a launch counts fewer than 2^32 threads; beyond that they go round)
inline unsigned row_walk_blocks(const RowWalk& w) {
    const int64_t blocks = ceil_div64(ceil_div64(w.rows, kWave >> w.log_lanes) * w.slices, 4);
    return (unsigned)(blocks < (1 << 22) ? blocks : 1 << 22);
}

int checkpoint_load(const uint8_t* codes, const uint8_t* scales, int64_t rows, int d, void* x, int dtype, hipStream_t st);

}  // namespace moegps
