// Products with 4-bit weights for a few rows per expert: weights go from memory into registers, a wavefront's k-tiles at a time.
// Included by mx4.hip inside namespace moegps.
//
// A unit is an M-tile of up to 64 rows by NG panels (32 packed columns each).  The wavefronts of a workgroup share the unit's
// columns and split K between them; each reads its own activation fragments and nothing synchronises until the fp32 sums are
// added up through LDS, wavefront 0 first, so the result does not depend on timing.
//
// fp32 rows are taken as three bf16 parts, x = hi + mid + lo, by cutting off 8 significant bits at a time: exact, and so are
// the products with the weights, which are exact in bf16.
#pragma once

// eight fp32 values as three bf16 operands that add up to them; an infinity or a NaN is all in the first
__device__ __forceinline__ void split_f32(const f32x4 (&v)[2], bf16x8& hi, bf16x8& mid, bf16x8& lo) {
    typedef __attribute__((__vector_size__(4 * sizeof(unsigned)))) unsigned u32x4;
    u32x4 w[3];
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        unsigned part[2][3];
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const float x = v[p >> 1][(p & 1) * 2 + h];
            unsigned bits = __builtin_bit_cast(unsigned, x);
            const bool finite = (bits & 0x7f800000u) != 0x7f800000u;
            if (!finite && (bits & 0x007fffffu) != 0) bits |= 0x00400000u;  // a NaN stays one
            const unsigned a = bits & 0xffff0000u;
            const float r = finite ? x - __builtin_bit_cast(float, a) : 0.f;
            const unsigned b = __builtin_bit_cast(unsigned, r) & 0xffff0000u;
            const float s = r - __builtin_bit_cast(float, b);
            part[h][0] = a;
            part[h][1] = b;
            part[h][2] = __builtin_bit_cast(unsigned, s) & 0xffff0000u;
        }
#pragma unroll
        for (int i = 0; i < 3; ++i) w[i][p] = part[0][i] >> 16 | part[1][i];
    }
    hi = __builtin_bit_cast(bf16x8, w[0]);
    mid = __builtin_bit_cast(bf16x8, w[1]);
    lo = __builtin_bit_cast(bf16x8, w[2]);
}

// A product's operands and where its rows live (RowMap).  K: true width of a row, a multiple of 16 bytes; N: output columns.
struct Mx4Product {
    const void* A;
    int lda, K;
    Mx4Matrix B;
    void* C;
    int ldc, N;
    const MTile* mtiles;
    const int32_t* counts;
    RowMap rm;
};

constexpr int kMx4StreamRows = 64;  // rows of an M-tile

template <int NG, int NW, int EPI, bool F32>
__global__ __launch_bounds__(NW * 64) void mx4_stream_kernel(Mx4Product p) {
    constexpr bool SWIGLU = EPI == kEpiSwiglu;
    constexpr int UC = NG * kMx4N;              // packed columns of a unit
    constexpr int OC = SWIGLU ? UC / 2 : UC;    // output columns
    constexpr int PITCH = UC + 4;
    constexpr int PARTS = F32 ? 3 : 1;
    constexpr int SIZE = F32 ? 4 : 2;
    __shared__ __align__(16) float xch[NW * 16 * PITCH];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g16 = lane >> 4;
    const int KT = p.B.kt;
    const int n_units = ceil_div(p.B.panels, NG);
    const int total = p.counts[kCntEntries] * n_units;
    const int kt0 = (int)((long long)KT * wave / NW), kt1 = (int)((long long)KT * (wave + 1) / NW);
    const size_t panel_bytes = mx4_panel_bytes(KT);

    for (int u = blockIdx.x; u < total; u += gridDim.x) {
        const int entry = u / n_units, nu = u - entry * n_units;
        const MTile mt = p.mtiles[entry];
        const unsigned char* panel[NG];
#pragma unroll
        for (int n = 0; n < NG; ++n) {  // (panels past the last repeat it, their columns are dropped)
            const int at = nu * NG + n < p.B.panels ? nu * NG + n : p.B.panels - 1;
            panel[n] = p.B.at + (size_t)mt.expert * p.B.expert + at * panel_bytes;
        }
        auto unit = [&](auto MT_tag) {
            constexpr int MT = decltype(MT_tag)::value;  // 16-row groups of the M-tile that hold rows, rounded up
            const char* arow[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                int r = i * 16 + l16;
                r = mt.list0 + (r < mt.rows ? r : mt.rows - 1);
                if (p.rm.a_rows) {
                    r = p.rm.a_rows[r];
                    if (p.rm.a_rows2) r = p.rm.a_rows2[r] / p.rm.a_div;
                }
                arow[i] = (const char*)p.A + (size_t)r * p.lda * SIZE;
            }
            f32x4 acc[MT][NG][2];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][n][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            struct Tile {
                uint4 codes[NG];
                unsigned scales[NG];
                f32x4 a[MT][2][F32 ? 2 : 1];
            };
            // 16 bytes of a row from element k on, zeros past its end (what lies there is not this row's)
            auto piece = [&](const char* row, int k) {
                const bool in = k < p.K;
                f32x4 v = *(const f32x4*)(row + (size_t)(in ? k : 0) * SIZE);
                if (!in) v = f32x4{0.f, 0.f, 0.f, 0.f};
                return v;
            };
            auto load = [&](int kt, Tile& t) {
#pragma unroll
                for (int n = 0; n < NG; ++n) {
                    t.codes[n] = *(const uint4*)(panel[n] + mx4_codes_at(kt) + lane * 16);
                    t.scales[n] = *(const unsigned short*)(panel[n] + mx4_scales_at(kt) + (g16 >> 1) * 128 + l16 * 8 +
                                                           (kt & 3) * 2);
                }
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const int k = kt * kMx4K + g16 * 16 + s * 8;
                        t.a[i][s][0] = piece(arow[i], k);
                        if constexpr (F32) t.a[i][s][1] = piece(arow[i], k + 4);
                    }
            };
            auto multiply = [&](const Tile& t) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    bf16x8 b[NG][2];
#pragma unroll
                    for (int n = 0; n < NG; ++n) {
                        b[n][0] = mx4_values(s ? t.codes[n].z : t.codes[n].x, mx4_scale<0>(t.scales[n]));
                        b[n][1] = mx4_values(s ? t.codes[n].w : t.codes[n].y, mx4_scale<1>(t.scales[n]));
                    }
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        bf16x8 a[PARTS];
                        if constexpr (F32) split_f32(t.a[i][s], a[2], a[1], a[0]);  // (smallest parts first)
                        else a[0] = __builtin_bit_cast(bf16x8, t.a[i][s][0]);
#pragma unroll
                        for (int q = 0; q < PARTS; ++q)
#pragma unroll
                            for (int n = 0; n < NG; ++n)
#pragma unroll
                                for (int j = 0; j < 2; ++j)
                                    acc[i][n][j] =
                                        __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[n][j], a[q], acc[i][n][j], 0, 0, 0);
                    }
                }
            };
            if (kt0 < kt1) {
                Tile t;
                load(kt0, t);
                for (int kt = kt0; kt < kt1; ++kt) {
                    Tile next;
                    load(kt + 1 < kt1 ? kt + 1 : kt, next);
                    multiply(t);
                    t = next;
                }
            }
            // the parts of K added up, 16 rows at a time
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                if (i * 16 >= mt.rows) continue;  // (uniform)
                __syncthreads();
#pragma unroll
                for (int n = 0; n < NG; ++n)
#pragma unroll
                    for (int j = 0; j < 2; ++j)
                        *(f32x4*)&xch[(wave * 16 + l16) * PITCH + n * kMx4N + j * 16 + g16 * 4] = acc[i][n][j];
                __syncthreads();
                for (int at = tid; at < 16 * OC / 2; at += NW * 64) {
                    const int row = at / (OC / 2), c = at % (OC / 2) * 2;
                    const int mrow = i * 16 + row;
                    // packed column of the first: with SwiGLU 16 gate columns and their 16 up columns alternate
                    const int pc = SWIGLU ? (c >> 4) * kMx4N + (c & 15) : c;
                    const int col = nu * OC + c;
                    if (mrow >= mt.rows || col >= p.N) continue;
                    float v[2] = {0.f, 0.f}, g[2] = {0.f, 0.f};
#pragma unroll
                    for (int w = 0; w < NW; ++w)
#pragma unroll
                        for (int q = 0; q < 2; ++q) {
                            v[q] += xch[(w * 16 + row) * PITCH + pc + q];
                            if (SWIGLU) g[q] += xch[(w * 16 + row) * PITCH + pc + 16 + q];
                        }
                    int crow = mt.list0 + mrow;
                    float sc = 1.f;
                    if (EPI == kEpiNone) {
                        if (p.rm.c_rows) crow = p.rm.c_rows[crow];
                        if (p.rm.scale) sc = p.rm.scale[p.rm.scale_idx[crow]];
                    }
#pragma unroll
                    for (int q = 0; q < 2; ++q) {
                        if constexpr (SWIGLU) v[q] = (F32 ? v[q] / (1.0f + expf(-v[q])) : silu_f(v[q])) * g[q];
                        else if constexpr (EPI == kEpiRelu) v[q] = fmaxf(v[q], 0.f);
                        else v[q] *= sc;
                    }
                    if constexpr (F32) *(float2*)((float*)p.C + (size_t)crow * p.ldc + col) = make_float2(v[0], v[1]);
                    else *(unsigned*)((bf16_t*)p.C + (size_t)crow * p.ldc + col) = pack_bf16x2(v[0], v[1]);
                }
            }
            __syncthreads();  // (the next unit's sums go to the same place)
        };
        if (mt.rows <= 16) unit(std::integral_constant<int, 1>{});
        else if (mt.rows <= 32) unit(std::integral_constant<int, 2>{});
        else unit(std::integral_constant<int, 4>{});
    }
}
