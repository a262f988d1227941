// Weights to 4 bits and back (mx4.h, include/moegps_mx4.h).
//
//     s = 2^(b - 127), b the smallest with max|w| <= 6 s over 32 neighbours along k;   code = e2m1(w / s);   back = code * s
//
// Division and way back are exact, the one rounding is that to the code.  With a scale that may cut off (max|w| below 8 s) the largest weight
// of a group would be off by up to a quarter instead of a fifth.
//
// Bound by memory: 2 (fp32: 4) bytes of a weight one way and 0.53 the other.  A workgroup of four wavefronts turns a k-tile of eight
// panels: a lane takes two neighbouring columns of a matrix and 32 of k, a row's pieces of a wavefront being 256 (512) contiguous
// bytes, all of its 32 rows under way at once; a group's maximum is then the lane's own.  The codes meet in LDS in the order of the
// layout and leave as whole kilobytes.  8 experts of 4096 x 14336 680 us there, 659 back (5.3 TB/s); 8 of 128 x 256 10 and 11, two launches each.
#include "mx4.h"

namespace moegps {

typedef __attribute__((__vector_size__(2 * sizeof(unsigned)))) unsigned u32x2;
typedef __attribute__((__vector_size__(4 * sizeof(unsigned)))) unsigned u32x4;

constexpr int kPackPanels = 8;   // panels of a workgroup
constexpr int kPartCols = 128;   // columns of a wavefront

// What a launch goes over: `two`: panels of 16 columns of both matrices, else of 32 of the first.
struct Mx4Pack {
    const void* W[2];
    int K, N, two, E;
    int kt, panels;
    size_t expert;
};

struct Mx4PackAt {
    int e, kt, p0, n0, half, part, lane;
    const char* W;
};

// Where item `item` of a launch and this lane of its workgroup are.
__device__ __forceinline__ Mx4PackAt pack_at(const Mx4Pack& p, int64_t item, int size) {
    Mx4PackAt a;
    const int blocks = ceil_div(p.panels, kPackPanels);
    // (k-tiles run fastest: workgroups side by side write neighbouring kilobytes of the same panels)
    const int64_t rest = item / p.kt;
    a.kt = (int)(item - rest * p.kt);
    a.e = (int)(rest / blocks);
    a.p0 = (int)(rest - (int64_t)a.e * blocks) * kPackPanels;
    const int wave = threadIdx.x / kWave;
    a.lane = threadIdx.x & (kWave - 1);
    a.half = wave & 1;
    a.part = wave >> 1;
    a.n0 = (p.two ? a.p0 * 16 : a.p0 * 32 + a.part * kPartCols) + 2 * a.lane;
    a.W = (const char*)(p.two && a.part ? p.W[1] : p.W[0]);
    if (a.W) a.W += (size_t)a.e * p.K * p.N * size;
    return a;
}
// panel (of the workgroup's eight), word's column half, column in it, of column c (0, 1) of this lane
__device__ __forceinline__ void column_of(const Mx4Pack& p, const Mx4PackAt& a, int c, int& panel, int& j, int& l16) {
    const int col = 2 * a.lane + c;
    l16 = col & 15;
    panel = p.two ? col >> 4 : a.part * 4 + (col >> 5);
    j = p.two ? a.part : (col >> 4) & 1;
}

// VEC: rows of an even number of values, a lane's two at once
template <bool BF16, bool VEC>
__global__ __launch_bounds__(256) void mx4_pack_kernel(Mx4Pack p, unsigned char* __restrict__ out, int64_t items) {
    constexpr int SIZE = BF16 ? 2 : 4;
    __shared__ __align__(16) unsigned codes[kPackPanels * kMx4Block / 4];
    __shared__ unsigned char scales[kPackPanels * 64];
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const Mx4PackAt a = pack_at(p, item, SIZE);
        // the bits of the values as floats: [column][k]
        unsigned v[2][32];
        const int k0 = a.kt * kMx4K + a.half * 32;
#pragma unroll
        for (int r = 0; r < 32; ++r) {
            const char* row = a.W + ((size_t)(k0 + r) * p.N + a.n0) * SIZE;
            const bool in = k0 + r < p.K;
            v[0][r] = v[1][r] = 0;
            if constexpr (VEC) {
                if (in && a.n0 < p.N) {
                    if constexpr (BF16) {
                        v[0][r] = __builtin_nontemporal_load((const unsigned*)row);
                    } else {
                        const u32x2 w = __builtin_nontemporal_load((const u32x2*)row);
                        v[0][r] = w[0];
                        v[1][r] = w[1];
                    }
                }
            } else {
#pragma unroll
                for (int c = 0; c < 2; ++c)
                    if (in && a.n0 + c < p.N) {
                        if constexpr (BF16) v[c][r] = ((const unsigned short*)row)[c];
                        else v[c][r] = ((const unsigned*)row)[c];
                    }
            }
        }
        if constexpr (BF16) {
#pragma unroll
            for (int r = 0; r < 32; ++r) {
                if constexpr (VEC) {
                    v[1][r] = v[0][r] & 0xffff0000u;
                    v[0][r] <<= 16;
                } else {
                    v[0][r] <<= 16;
                    v[1][r] <<= 16;
                }
            }
        }
        __syncthreads();  // (the previous item's codes have been read)
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            unsigned top = 0;
#pragma unroll
            for (int r = 0; r < 32; ++r) {
                const unsigned m = v[c][r] & 0x7fffffffu;
                top = m > top ? m : top;
            }
            // 6 = 1.5 * 2^2: the exponent of `top` less 2, one more above 1.5
            int b = (int)((top + 0x3fffffu) >> 23) - 2;
            b = top == 0 ? 127 : b < 2 ? 2 : b > 253 ? 253 : b;
            const float s = __builtin_bit_cast(float, (unsigned)b << 23);
            if (b == 253)  // 4 * 2^126 would be infinite
#pragma unroll
                for (int r = 0; r < 32; ++r)
                    v[c][r] = __builtin_bit_cast(unsigned, fminf(fmaxf(__builtin_bit_cast(float, v[c][r]), -0x3p126f), 0x3p126f));
            if (top >= 0x7f800000u) b = 255;
            int panel, j, l16;
            column_of(p, a, c, panel, j, l16);
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                unsigned w = 0;
                auto f = [&](int i) { return __builtin_bit_cast(float, v[c][q * 8 + i]); };
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f(0), f(1), s, 0);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f(2), f(3), s, 1);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f(4), f(5), s, 2);
                w = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(w, f(6), f(7), s, 3);
                const int g = a.half * 2 + (q >> 1);
                codes[panel * (kMx4Block / 4) + (g * 16 + l16) * 4 + (q & 1) * 2 + j] = w;
            }
            scales[panel * 64 + a.half * 32 + l16 * 2 + j] = (unsigned char)b;
        }
        __syncthreads();
        unsigned char* to = out + (size_t)a.e * p.expert;
        const size_t panel_bytes = mx4_panel_bytes(p.kt);
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int panel = i * 4 + threadIdx.x / kWave;
            if (a.p0 + panel < p.panels)
                *(u32x4*)(to + (a.p0 + panel) * panel_bytes + mx4_codes_at(a.kt) + a.lane * 16) =
                    ((const u32x4*)codes)[panel * kWave + a.lane];
        }
        const int panel = threadIdx.x / 32, at = threadIdx.x % 32;  // a panel's 32 pairs of scales
        if (a.p0 + panel < p.panels) {
            unsigned char* s = to + (a.p0 + panel) * panel_bytes + mx4_scales_at(a.kt) + at * 8;
            const unsigned pair = ((const unsigned short*)scales)[panel * 32 + at];
            ((unsigned short*)s)[a.kt & 3] = (unsigned short)pair;
            if (a.kt == p.kt - 1)  // k-tiles that the last four do not have
                for (int i = (a.kt & 3) + 1; i < 4; ++i) ((unsigned short*)s)[i] = 0;
        }
    }
}

template <bool BF16, bool VEC>
__global__ __launch_bounds__(256) void mx4_unpack_kernel(Mx4Pack p, const unsigned char* __restrict__ in, int64_t items) {
    constexpr int SIZE = BF16 ? 2 : 4;
    __shared__ __align__(16) unsigned codes[kPackPanels * kMx4Block / 4];
    for (int64_t item = blockIdx.x; item < items; item += gridDim.x) {
        const Mx4PackAt a = pack_at(p, item, SIZE);
        const unsigned char* from = in + (size_t)a.e * p.expert;
        const size_t panel_bytes = mx4_panel_bytes(p.kt);
        __syncthreads();  // (the previous item's codes have been read)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const int panel = i * 4 + threadIdx.x / kWave;
            if (a.p0 + panel < p.panels)
                ((u32x4*)codes)[panel * kWave + a.lane] = __builtin_nontemporal_load(
                    (const u32x4*)(from + (a.p0 + panel) * panel_bytes + mx4_codes_at(a.kt) + a.lane * 16));
        }
        int panel[2], j[2], l16[2];
        float s[2];
#pragma unroll
        for (int c = 0; c < 2; ++c) {
            column_of(p, a, c, panel[c], j[c], l16[c]);
            s[c] = 1.f;
            if (a.p0 + panel[c] < p.panels) {
                const unsigned char* at = from + (a.p0 + panel[c]) * panel_bytes + mx4_scales_at(a.kt);
                s[c] = __builtin_bit_cast(float, (unsigned)at[a.half * 128 + l16[c] * 8 + (a.kt & 3) * 2 + j[c]] << 23);
            }
        }
        __syncthreads();
        const int k0 = a.kt * kMx4K + a.half * 32;
        char* W = const_cast<char*>(a.W);
        if (W && a.n0 < p.N) {
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                u32x4 v[2];  // eight values of a column, two to a word
#pragma unroll
                for (int c = 0; c < 2; ++c) {
                    const int g = a.half * 2 + (q >> 1);
                    v[c] = __builtin_bit_cast(u32x4, mx4_values(
                        codes[panel[c] * (kMx4Block / 4) + (g * 16 + l16[c]) * 4 + (q & 1) * 2 + j[c]], s[c]));
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const int k = k0 + q * 8 + i;
                    if (k >= p.K) continue;
                    const unsigned w0 = i & 1 ? v[0][i / 2] >> 16 : v[0][i / 2] & 0xffffu;
                    const unsigned w1 = i & 1 ? v[1][i / 2] >> 16 : v[1][i / 2] & 0xffffu;
                    char* row = W + ((size_t)k * p.N + a.n0) * SIZE;
                    if constexpr (BF16 && VEC) {
                        __builtin_nontemporal_store(w0 | w1 << 16, (unsigned*)row);
                    } else if constexpr (BF16) {
                        ((unsigned short*)row)[0] = (unsigned short)w0;
                        if (a.n0 + 1 < p.N) ((unsigned short*)row)[1] = (unsigned short)w1;
                    } else if constexpr (VEC) {
                        __builtin_nontemporal_store(u32x2{w0 << 16, w1 << 16}, (u32x2*)row);
                    } else {
                        ((unsigned*)row)[0] = w0 << 16;
                        if (a.n0 + 1 < p.N) ((unsigned*)row)[1] = w1 << 16;
                    }
                }
            }
        }
    }
}

static bool mx4_width(int w) { return w >= 1 && w <= kMaxWidth; }

static int64_t pack_items(const Mx4Pack& p) { return (int64_t)p.E * p.kt * ceil_div(p.panels, kPackPanels); }
static unsigned pack_grid(int64_t items) { return (unsigned)(items < (1 << 22) ? items : 1 << 22); }

static int launch_pack(const Mx4Pack& p, int dtype, void* out, hipStream_t st) {
    const int64_t items = pack_items(p);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(pack_grid(items)), dim3(256), 0, st, p, (unsigned char*)out, items);
        return check_launch();
    };
    if (dtype == MOE_DTYPE_BF16) return go(p.N % 2 == 0 ? mx4_pack_kernel<true, true> : mx4_pack_kernel<true, false>);
    return go(p.N % 2 == 0 ? mx4_pack_kernel<false, true> : mx4_pack_kernel<false, false>);
}

static int launch_unpack(const Mx4Pack& p, int dtype, const void* in, hipStream_t st) {
    const int64_t items = pack_items(p);
    auto go = [&](auto kern) {
        hipLaunchKernelGGL(kern, dim3(pack_grid(items)), dim3(256), 0, st, p, (const unsigned char*)in, items);
        return check_launch();
    };
    if (dtype == MOE_DTYPE_BF16) return go(p.N % 2 == 0 ? mx4_unpack_kernel<true, true> : mx4_unpack_kernel<true, false>);
    return go(p.N % 2 == 0 ? mx4_unpack_kernel<false, true> : mx4_unpack_kernel<false, false>);
}

static Mx4Pack pack_of(const Mx4Matrix& m, const void* W0, const void* W1, int two, int E, int K, int N) {
    return Mx4Pack{{W0, W1}, K, N, two, E, m.kt, m.panels, m.expert};
}

static int pack_args(int dtype, int E, int K, int N) {
    if ((dtype != MOE_DTYPE_F32 && dtype != MOE_DTYPE_BF16) || E < 1 || K < 1 || N < 1) return MOE_ERR_INVALID_ARG;
    if (E > MOE_MAX_EXPERTS || !mx4_width(K) || !mx4_width(N)) return MOE_ERR_UNSUPPORTED;
    return MOE_OK;
}

}  // namespace moegps

extern "C" size_t moe_packed_weights_mx4_bytes(int E, int d, int ffn, int relu) {
    using namespace moegps;
    if (E < 1 || E > MOE_MAX_EXPERTS || !mx4_width(d) || !mx4_width(ffn)) return 0;
    return (size_t)E * (mx4_first(nullptr, d, ffn, relu).expert + mx4_second(nullptr, E, d, ffn, relu).expert);
}

extern "C" int moe_pack_weights_mx4(const void* W1, const void* W3, const void* W2, int dtype, int E, int d, int ffn,
                                    void* packed, void* stream) {
    using namespace moegps;
    if (const int rc = pack_args(dtype, E, d, ffn); rc != MOE_OK) return rc;
    if (!W1 || !W2 || !packed) return MOE_ERR_INVALID_ARG;
    const int relu = W3 == nullptr;
    hipStream_t st = (hipStream_t)stream;
    const Mx4Matrix m1 = mx4_first(packed, d, ffn, relu), m2 = mx4_second(packed, E, d, ffn, relu);
    if (const int rc = launch_pack(pack_of(m1, W1, W3, !relu, E, d, ffn), dtype, (void*)m1.at, st); rc != MOE_OK) return rc;
    return launch_pack(pack_of(m2, W2, nullptr, 0, E, ffn, d), dtype, (void*)m2.at, st);
}

extern "C" int moe_unpack_weights_mx4(const void* packed, int E, int d, int ffn, int relu, void* W1, void* W3, void* W2, int dtype,
                                      void* stream) {
    using namespace moegps;
    if (const int rc = pack_args(dtype, E, d, ffn); rc != MOE_OK) return rc;
    if (!packed || (relu && W3)) return MOE_ERR_INVALID_ARG;
    hipStream_t st = (hipStream_t)stream;
    const Mx4Matrix m1 = mx4_first(packed, d, ffn, relu), m2 = mx4_second(packed, E, d, ffn, relu);
    if (W1 || W3)
        if (const int rc = launch_unpack(pack_of(m1, W1, W3, !relu, E, d, ffn), dtype, m1.at, st); rc != MOE_OK) return rc;
    return W2 ? launch_unpack(pack_of(m2, W2, nullptr, 0, E, ffn, d), dtype, m2.at, st) : MOE_OK;
}

extern "C" size_t moe_packed_matrix_mx4_bytes(int E, int K, int N) {
    using namespace moegps;
    if (E < 1 || E > MOE_MAX_EXPERTS || !mx4_width(K) || !mx4_width(N)) return 0;
    return (size_t)E * mx4_matrix(nullptr, K, ceil_div(N, kMx4N)).expert;
}

extern "C" int moe_pack_matrix_mx4(const void* W, int dtype, int E, int K, int N, void* packed, void* stream) {
    using namespace moegps;
    if (const int rc = pack_args(dtype, E, K, N); rc != MOE_OK) return rc;
    if (!W || !packed) return MOE_ERR_INVALID_ARG;
    const Mx4Matrix m = mx4_matrix(packed, K, ceil_div(N, kMx4N));
    return launch_pack(pack_of(m, W, nullptr, 0, E, K, N), dtype, packed, (hipStream_t)stream);
}

extern "C" int moe_unpack_matrix_mx4(const void* packed, int E, int K, int N, void* W, int dtype, void* stream) {
    using namespace moegps;
    if (const int rc = pack_args(dtype, E, K, N); rc != MOE_OK) return rc;
    if (!W || !packed) return MOE_ERR_INVALID_ARG;
    const Mx4Matrix m = mx4_matrix(packed, K, ceil_div(N, kMx4N));
    return launch_unpack(pack_of(m, W, nullptr, 0, E, K, N), dtype, packed, (hipStream_t)stream);
}
