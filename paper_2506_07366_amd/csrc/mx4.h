// Weights in 4 bits (include/moegps_mx4.h): how they are laid out, and what the kernels that read them share.
//
// What a product wants to find is a panel: 32 output columns, all of the contracted dimension, cut into k-tiles of 64.  A k-tile's
// codes are one contiguous kilobyte, which a wavefront loads as 16 bytes per lane:
//   lane 16 g + c holds columns c (word 2 s) and 16 + c (word 2 s + 1), k = 16 g + 8 s .. + 7 of the k-tile, s = 0, 1.
// Eight codes are one operand of v_mfma_f32_16x16x32_bf16; the order of k inside an instruction is free as long as both operands
// have the same, and this one gives a lane 16 neighbours, so that one scale does for its two words and a row's 128 bytes are one cache
// line for the four lanes that read them.  Ahead of every four k-tiles (or what is left) are their scales, 256 bytes:
//   bytes 128 h + 8 c + 2 i + j: k-tile i, column 16 j + c, k = 32 h .. 32 h + 31.
// In the first product of a SwiGLU FFN a panel is 16 hidden columns: the gate's as columns 0 .. 15, the up projection's as 16 .. 31, so
// that a lane has both sums of a hidden value.  Padding (k past the end, columns past the end) is zeros.
#pragma once
#include "../../include/moegps_mx4.h"
#include "ffn_device.h"

namespace moegps {

constexpr int kMx4K = 64, kMx4N = 32;      // of a k-tile's block
constexpr int kMx4Block = kMx4K * kMx4N / 2;  // bytes of its codes
constexpr int kMx4Scales = 256;            // bytes of the scales of four
static_assert(MOE_MX4_GROUP == 32 && kMx4Block == 64 * 16, "a block is 16 bytes for every lane");

__host__ __device__ inline size_t mx4_panel_bytes(int kt) {
    return (size_t)kt * kMx4Block + (size_t)ceil_div(kt, 4) * kMx4Scales;
}
// bytes from a panel's start to the codes of k-tile i, and to the scales of its four
__host__ __device__ inline unsigned mx4_codes_at(int i) { return (unsigned)i * kMx4Block + (unsigned)((i >> 2) + 1) * kMx4Scales; }
__host__ __device__ inline unsigned mx4_scales_at(int i) { return (unsigned)(i >> 2) * (4 * kMx4Block + kMx4Scales); }

// One matrix per expert: k-tiles, panels, bytes of an expert.
struct Mx4Matrix {
    const unsigned char* at;
    int kt, panels;
    size_t expert;
};
inline Mx4Matrix mx4_matrix(const void* at, int K, int panels) {
    Mx4Matrix m{(const unsigned char*)at, ceil_div(K, kMx4K), panels, 0};
    m.expert = (size_t)panels * mx4_panel_bytes(m.kt);
    return m;
}
// The two of an FFN: the hidden width is padded to whole k-tiles of the second.
inline int mx4_hidden(int ffn) { return (int)align_up((size_t)ffn, kMx4K); }
inline Mx4Matrix mx4_first(const void* packed, int d, int ffn, int relu) {
    return mx4_matrix(packed, d, mx4_hidden(ffn) / (relu ? 32 : 16));
}
inline Mx4Matrix mx4_second(const void* packed, int E, int d, int ffn, int relu) {
    const Mx4Matrix first = mx4_first(packed, d, ffn, relu);
    return mx4_matrix((const char*)packed + (size_t)E * first.expert, mx4_hidden(ffn), ceil_div(d, kMx4N));
}

// Eight codes of a word as bf16 values: four conversions, each of two codes.  `scale` is a float whose exponent field is b; its sign and
// mantissa are not looked at, so a byte of a word need only be shifted there.  Exponent field 255 makes NaN.
__device__ __forceinline__ bf16x8 mx4_values(unsigned codes, float scale) {
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    struct {
        bf16x2 v[4];
    } r;
    r.v[0] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 0);
    r.v[1] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 1);
    r.v[2] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 2);
    r.v[3] = __builtin_amdgcn_cvt_scalef32_pk_bf16_fp4(codes, scale, 3);
    return __builtin_bit_cast(bf16x8, r);
}
// byte j (0, 1) of the low half of a word, as such a scale
template <int J>
__device__ __forceinline__ float mx4_scale(unsigned bytes) {
    return __builtin_bit_cast(float, bytes << (23 - 8 * J));
}

// moe_grouped_ffn_mx4, or the part of it that `stage` names (ffn_tables.h).
int mx4_ffn_call(const moe_ffn_mx4_args& a, hipStream_t st, const FfnOptions& opt, FfnStage stage, TableJob* job_out);

}  // namespace moegps
