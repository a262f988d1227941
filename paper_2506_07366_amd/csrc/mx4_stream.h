// Products with 4-bit weights that go along the panels' bytes.  Included by mx4.hip inside namespace moegps.
//
//   mx4_split_kernel  bf16 rows, M-tiles of up to 32: the finest units, for batches whose tiles would not fill the chip
//   mx4_wide_kernel   bf16 rows, M-tiles of up to 32: eight panels side by side, for many units of few rows
//   mx4_f32_kernel    fp32 rows, any number: x = hi + mid + lo by cutting off 8 significant bits at a time, exact, and so are
//                     the products with the weights, which are exact in bf16
//
// In the first and the last a unit is an M-tile by one panel.  The eight wavefronts of a workgroup split K between them, and nothing
// synchronises until their fp32 sums are added up through LDS, wavefront 0 first, so the result does not depend on timing.  In the wide
// form a wavefront has a panel and all of K to itself, the rows are everybody's, and there is a barrier for every step of 256 of K.
#pragma once

typedef __attribute__((__vector_size__(2 * sizeof(unsigned)))) unsigned u32x2;

// eight fp32 values as three bf16 operands that add up to them; an infinity or a NaN is all in the first
__device__ __forceinline__ void split_f32(const f32x4 (&v)[2], bf16x8& hi, bf16x8& mid, bf16x8& lo) {
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
    RowMap rm;           // (without rows to look up twice)
    const float* gates;  // of the rows, by list position; null: none
};

constexpr int kMx4SplitWaves = 8;
constexpr int kMx4SplitRows = 32, kMx4F32Rows = 64;  // rows of an M-tile

// Adds up what the wavefronts have of rows list0 + row0 .. of an M-tile with `rows` from there on (16 at most are there) and stores
// the results.  Starts and ends with a barrier's worth of order: xch may be anything that all wavefronts are done with.
template <int EPI, bool F32>
__device__ __forceinline__ void add_parts(const Mx4Product& p, float* xch, int wave, const f32x4 (&acc)[2], int list0, int rows,
                                          int panel) {
    constexpr bool SWIGLU = EPI == kEpiSwiglu;
    constexpr int OC = SWIGLU ? kMx4N / 2 : kMx4N;  // output columns
    constexpr int PITCH = kMx4N + 4;
    const int lane = threadIdx.x & 63, l16 = lane & 15, g16 = lane >> 4;
    __syncthreads();
    if (l16 < rows)
#pragma unroll
        for (int j = 0; j < 2; ++j) *(f32x4*)&xch[(wave * 16 + l16) * PITCH + j * 16 + g16 * 4] = acc[j];
    __syncthreads();
    for (int at = threadIdx.x; at < 16 * OC / 2; at += kMx4SplitWaves * 64) {
        const int row = at / (OC / 2), c = at % (OC / 2) * 2;
        // (with SwiGLU the panel's first 16 columns are the gate's, their up columns the others)
        const int col = panel * OC + c;
        if (row >= rows || col >= p.N) continue;
        float v[2] = {0.f, 0.f}, g[2] = {0.f, 0.f};
#pragma unroll
        for (int w = 0; w < kMx4SplitWaves; ++w)
#pragma unroll
            for (int q = 0; q < 2; ++q) {
                v[q] += xch[(w * 16 + row) * PITCH + c + q];
                if (SWIGLU) g[q] += xch[(w * 16 + row) * PITCH + c + 16 + q];
            }
        int crow = list0 + row;
        float sc = 1.f;
        if (EPI == kEpiNone) {
            if (p.gates) sc = p.gates[crow];
            if (p.rm.c_rows) crow = p.rm.c_rows[crow];
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

// The streaming kernels go along K in steps of four k-tiles, which share their scales: 4 KiB of codes and 256 bytes of scales of a
// panel are five loads.  What lies past the end of a panel or of a row is asked for out of the buffer's range, which keeps the number of
// loads fixed (the waits count them), costs no memory access and gives zeros.
struct Mx4Step {
    u32x4 codes[4];
    u32x2 scales;
};
constexpr int kStepK = 4 * kMx4K, kStepBytes = 4 * kMx4Block + kMx4Scales;
constexpr unsigned kRowRange = 0xffffff80u, kRowPast = 0xfffffff0u;  // of the rows: fewer than 2^31 - 63 elements

__device__ __forceinline__ auto rows_rsrc(const Mx4Product& p) {
    return __builtin_amdgcn_make_buffer_rsrc((void*)p.A, 0, (int)kRowRange, 0x00027000);
}
// row of the product's operand at a list position
__device__ __forceinline__ int row_at(const Mx4Product& p, int pos) { return p.rm.a_rows ? p.rm.a_rows[pos] : pos; }
template <int AUX, class R>
__device__ __forceinline__ void load_step(Mx4Step& t, R rsrc, int step, bool in, int lane) {
    const unsigned at = in ? (unsigned)step * kStepBytes : 0xf0000000u;
    const unsigned codes = at + kMx4Scales + lane * 16, scales = at + (lane >> 5) * 128 + (lane & 15) * 8;
#pragma unroll
    for (int i = 0; i < 4; ++i)
        t.codes[i] = __builtin_bit_cast(u32x4, __builtin_amdgcn_raw_buffer_load_b128(rsrc, codes + i * kMx4Block, 0, AUX));
    t.scales = __builtin_bit_cast(u32x2, __builtin_amdgcn_raw_buffer_load_b64(rsrc, scales, 0, AUX));
}
// operand s (0, 1) of column half j of the step's k-tile i
template <int I, int S, int J>
__device__ __forceinline__ bf16x8 step_values(const Mx4Step& t) {
    const unsigned scales = t.scales[I >> 1];
    // bytes 2 (i & 1) + j of the word, brought to the exponent's place
    constexpr int byte = 2 * (I & 1) + J;
    const unsigned shifted = byte < 3 ? scales << (byte < 3 ? 23 - 8 * byte : 0) : scales >> 1;
    return mx4_values(t.codes[I][2 * S + J], __builtin_bit_cast(float, shifted));
}

// For few units: each wavefront takes every eighth of the steps' range by itself, its rows in LDS of its own (loads that write LDS directly)
// and from there in registers before the loads of the step after next may overwrite them.  8 KiB of LDS per wavefront: two steps of 8 rows
// or one of 16; M-tiles of more rows are done 16 at a time.  One token on 8 experts of 4096 x 1536 (27 MB a matrix): one matrix 8 to 10 us, the
// first product of an FFN 14 to 17; second products of 16 tokens on 8 of 4096 x 14336, five to eight of them with rows (K = 14336), 35 to 45.
constexpr int kMx4SplitLds = 8192;
template <int EPI>
__global__ __launch_bounds__(kMx4SplitWaves * 64, 4) void mx4_split_kernel(Mx4Product p) {
    __shared__ __align__(1024) unsigned char smem[kMx4SplitWaves * kMx4SplitLds];
    static_assert(sizeof(smem) >= kMx4SplitWaves * 16 * (kMx4N + 4) * sizeof(float), "the parts are added up in the same place");
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g16 = lane >> 4;
    const int steps = ceil_div(p.B.kt, 4);
    const int total = p.counts[kCntEntries] * p.B.panels;
    const int st0 = steps * wave / kMx4SplitWaves, n = steps * (wave + 1) / kMx4SplitWaves - st0;
    const size_t panel_bytes = mx4_panel_bytes(p.B.kt);
    unsigned char* const mine = smem + wave * kMx4SplitLds;
    const unsigned mine_at = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)mine;
    const auto a_rsrc = rows_rsrc(p);

    for (int u = blockIdx.x; u < total; u += gridDim.x) {
        const int entry = u / p.B.panels, panel = u - entry * p.B.panels;
        const MTile mt = p.mtiles[entry];
        const auto w_rsrc = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(p.B.at + (size_t)mt.expert * p.B.expert + (size_t)panel * panel_bytes), 0, (int)panel_bytes, 0x00027000);
        // rows [row0, row0 + 8 * EIGHTS) of the M-tile
        auto unit = [&](auto E_tag, int row0) {
            constexpr int EIGHTS = decltype(E_tag)::value;
            constexpr int D = EIGHTS == 1 ? 2 : 1;    // steps in LDS
            constexpr int NB = 5 + 4 * EIGHTS;        // loads of a step
            unsigned off[EIGHTS];                     // of this lane's piece of a row's k-tile 0
            int a_end[EIGHTS];                        // k-tiles in which it exists
#pragma unroll
            for (int i = 0; i < EIGHTS; ++i) {
                const int row = i * 8 + (lane >> 3), slot = (lane & 7) ^ swz(row);
                a_end[i] = ((p.K >> 3) - slot + 7) / 8;
                const int at = row0 + row < mt.rows ? row0 + row : mt.rows - 1;  // rows past the end repeat the last one
                off[i] = (unsigned)row_at(p, mt.list0 + at) * (unsigned)p.lda * 2u + slot * 16u;
            }
            unsigned a_lane[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) {
                const int row = EIGHTS == 1 ? l16 & 7 : l16;
                a_lane[s] = mine_at + row * 128 + (((g16 * 2 + s) ^ swz(row)) * 16);
            }
            f32x4 acc[2];
#pragma unroll
            for (int j = 0; j < 2; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
            Mx4Step t[2];
            auto load = [&](int i, auto B_tag) {  // step i of this wavefront's
                constexpr int b = decltype(B_tag)::value;
                const int kt = i < n ? (st0 + i) * 4 : 1 << 24;
#pragma unroll
                for (int q = 0; q < 4; ++q)
#pragma unroll
                    for (int e = 0; e < EIGHTS; ++e) {
                        const unsigned at = kt + q < a_end[e] ? off[e] + (unsigned)(kt + q) * 128u : kRowPast;
                        __builtin_amdgcn_raw_ptr_buffer_load_lds(
                            a_rsrc, (__attribute__((address_space(3))) void*)(mine + (((b % D) * 4 + q) * EIGHTS + e) * 1024), 16, at,
                            0, 0, 0);
                    }
                load_step<0>(t[b], w_rsrc, st0 + i, i < n, lane);
                __builtin_amdgcn_sched_barrier(0);
            };
            load(0, std::integral_constant<int, 0>{});
            if constexpr (D == 2) load(1, std::integral_constant<int, 1>{});
            auto body = [&](int i, auto U) {
                constexpr int b = decltype(U)::value;
                wait_vmcnt<NB*(D - 1)>();  // step i has landed
                bf16x8 af[8];
                static_for<8>([&](auto F) {
                    constexpr int f = decltype(F)::value;
                    lds_read_b128<((b % D) * 4 + f / 2) * EIGHTS * 1024>(af[f], a_lane[f & 1]);
                });
                lds_wait<0>();
#pragma unroll
                for (int f = 0; f < 8; ++f) lds_landed(af[f]);
                __builtin_amdgcn_sched_barrier(0);
                // (with one step in LDS the next one's codes go to the other buffer, with two the step after next's to this one's, below)
                if constexpr (D == 1) load(i + 1, std::integral_constant<int, (b + 1) % 2>{});
                static_for<8>([&](auto F) {
                    constexpr int f = decltype(F)::value, q = f / 2, s = f & 1;
                    acc[0] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(step_values<q, s, 0>(t[b]), af[f], acc[0], 0, 0, 0);
                    acc[1] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(step_values<q, s, 1>(t[b]), af[f], acc[1], 0, 0, 0);
                });
                __builtin_amdgcn_sched_barrier(0);
                if constexpr (D == 2) load(i + 2, std::integral_constant<int, b>{});
            };
            for (int i = 0; i < n; i += 2) {
                body(i, std::integral_constant<int, 0>{});
                if (i + 1 < n) body(i + 1, std::integral_constant<int, 1>{});
            }
            wait_vmcnt<0>();  // (nothing that still writes LDS is under way)
            const int left = mt.rows - row0;
            add_parts<EPI, false>(p, (float*)smem, wave, acc, mt.list0 + row0, left < 16 ? left : 16, panel);
            __syncthreads();  // (the next unit's rows go to the same place)
        };
        if (mt.rows <= 8) unit(std::integral_constant<int, 1>{}, 0);
        else
            for (int row0 = 0; row0 < mt.rows; row0 += 16) unit(std::integral_constant<int, 2>{}, row0);
    }
}

// For many units of few rows: eight panels side by side, one per wavefront, over all of K, and up to 32 rows, which the wavefronts share
// in LDS: three steps of them, one barrier a step.  128 tokens on 128 experts of 4096 x 1536 122 us (4.6 TB/s) and 69; nothing but the loads
// of the weights would take three quarters of that.  Units of 32 rows cost more than their bytes, those of 16 do not.  Two workgroups a CU leave 128
// registers: 21 to 40 values of a lane that hold for a unit are in scratch, stored at entry and reloaded ahead of the K loop and behind it, not in it.
constexpr int kMx4WideRows = 32, kMx4WideDepth = 3;
constexpr int kMx4WideStage = kMx4WideRows * kStepK * 2;
constexpr size_t kMx4WideLds = (size_t)kMx4WideDepth * kMx4WideStage;
template <int EPI>
__global__ __launch_bounds__(512, 4) void mx4_wide_kernel(Mx4Product p) {
    constexpr bool SWIGLU = EPI == kEpiSwiglu;
    constexpr int NW = 8, D = kMx4WideDepth;
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    const int l16 = lane & 15, g16 = lane >> 4;
    const int steps = ceil_div(p.B.kt, 4);
    const int n_units = ceil_div(p.B.panels, NW);
    const int total = p.counts[kCntEntries] * n_units;
    const size_t panel_bytes = mx4_panel_bytes(p.B.kt);
    const unsigned smem_at = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
    const auto a_rsrc = rows_rsrc(p);

    // Units are dealt in chunks of 16 to the 8 XCDs (workgroup b runs on XCD b % 8; the launch is a multiple of 128 workgroups), and an
    // expert's M-tiles follow each other under the same panels, which they then find in one L2.
    const int slot = blockIdx.x >> 3;
    for (int u = ((slot >> 4) * 8 + (blockIdx.x & 7)) * 16 + (slot & 15); u < total; u += gridDim.x) {
        int entry = u / n_units, nu = u - entry * n_units;
        MTile mt = p.mtiles[entry];
        if (mt.n_same > 1) {
            const int v = u - mt.first * n_units;
            nu = v / mt.n_same;
            mt = p.mtiles[mt.first + v % mt.n_same];
        }
        const int panel = nu * NW + wave;
        const bool live = panel < p.B.panels;
        const auto w_rsrc = __builtin_amdgcn_make_buffer_rsrc(
            (void*)(p.B.at + (size_t)mt.expert * p.B.expert + (size_t)(live ? panel : 0) * panel_bytes), 0, live ? (int)panel_bytes : 0,
            0x00027000);
        // TM: 16-row groups; ONCE: no other M-tile wants the weights, they are read past the caches
        auto unit = [&](auto TM_tag, auto once_tag) {
            constexpr int TM = decltype(TM_tag)::value;
            constexpr int AUX = decltype(once_tag)::value ? kNonTemporal : 0;
            constexpr int NB = 5 + TM;  // loads of a wavefront and step: TM kilobytes of rows (eight rows of a k-tile each)
            unsigned off[TM];
            int a_end[TM], a_kt[TM];
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                // piece `wave + 8 i` of the step: k-tile, eight rows of it
                const int piece = wave + i * NW, row = (piece % (2 * TM)) * 8 + (lane >> 3), at = (lane & 7) ^ swz(row);
                a_kt[i] = piece / (2 * TM);
                a_end[i] = ((p.K >> 3) - at + 7) / 8;
                off[i] = (unsigned)row_at(p, mt.list0 + (row < mt.rows ? row : mt.rows - 1)) * (unsigned)p.lda * 2u + at * 16u;
            }
            f32x4 acc[TM][2];
#pragma unroll
            for (int i = 0; i < TM; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            Mx4Step t[D];
            auto load = [&](int i, auto B_tag) {
                constexpr int b = decltype(B_tag)::value;
#pragma unroll
                for (int q = 0; q < TM; ++q) {
                    const int kt = i * 4 + a_kt[q];
                    const unsigned at = kt < a_end[q] ? off[q] + (unsigned)kt * 128u : kRowPast;  // (past the last step too)
                    __builtin_amdgcn_raw_ptr_buffer_load_lds(
                        a_rsrc, (__attribute__((address_space(3))) void*)(smem + b * kMx4WideStage + (wave + q * NW) * 1024), 16, at, 0, 0,
                        0);
                }
                load_step<AUX>(t[b], w_rsrc, i, i < steps, lane);
                __builtin_amdgcn_sched_barrier(0);
            };
            unsigned a_lane[2];
#pragma unroll
            for (int s = 0; s < 2; ++s) a_lane[s] = smem_at + l16 * 128 + (((g16 * 2 + s) ^ swz(l16)) * 16);
            static_for<D - 1>([&](auto B) { load(decltype(B)::value, B); });
            auto body = [&](int i, auto U) {
                constexpr int b = decltype(U)::value;
                wait_vmcnt<NB*(D - 2)>();  // this wavefront's share of step i has landed ...
                __builtin_amdgcn_s_barrier();  // ... and everybody's; and everybody is done with step i - 1
                load(i + D - 1, std::integral_constant<int, (b + D - 1) % D>{});
                constexpr int PER = 4 / TM;  // k-tiles at a time: eight fragments
                static_for<TM>([&](auto G) {
                    constexpr int q0 = decltype(G)::value * PER;
                    bf16x8 af[8];  // [k-tile][s][row group]
                    static_for<8>([&](auto F) {
                        constexpr int f = decltype(F)::value, q = q0 + f / (2 * TM), s = f / TM % 2, i16 = f % TM;
                        lds_read_b128<b * kMx4WideStage + (q * TM + i16) * 2048>(af[f], a_lane[s]);
                    });
                    bf16x8 w[2];
                    static_for<8>([&](auto F) {
                        constexpr int f = decltype(F)::value, q = q0 + f / (2 * TM), s = f / TM % 2, i16 = f % TM;
                        if constexpr (i16 == 0) {
                            w[0] = step_values<q, s, 0>(t[b]);
                            w[1] = step_values<q, s, 1>(t[b]);
                        }
                        lds_wait<7 - f>();
                        lds_landed(af[f]);
                        __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            acc[i16][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(w[j], af[f], acc[i16][j], 0, 0, 0);
                        __builtin_amdgcn_sched_barrier(0);
                    });
                });
            };
            for (int i = 0; i < steps; i += D)
                static_for<D>([&](auto U) {
                    if (decltype(U)::value == 0 || i + decltype(U)::value < steps) body(i + decltype(U)::value, U);
                });
            wait_vmcnt<0>();  // (nothing that still writes LDS is under way)
            __syncthreads();  // (nor does anybody still read it)
            const int col0 = SWIGLU ? panel * 16 + g16 * 4 : panel * kMx4N + g16 * 4;
#pragma unroll
            for (int i = 0; i < TM; ++i) {
                const int row = i * 16 + l16;
                if (row >= mt.rows || !live) continue;
                int crow = mt.list0 + row;
                float sc = 1.f;
                if (EPI == kEpiNone) {
                    if (p.gates) sc = p.gates[crow];
                    if (p.rm.c_rows) crow = p.rm.c_rows[crow];
                }
                bf16_t* out = (bf16_t*)p.C + (size_t)crow * p.ldc + col0;
#pragma unroll
                for (int j = 0; j < (SWIGLU ? 1 : 2); ++j) {
                    float v[4];
#pragma unroll
                    for (int q = 0; q < 4; ++q)
                        v[q] = SWIGLU ? silu_f(acc[i][0][q]) * acc[i][1][q]
                                      : EPI == kEpiRelu ? fmaxf(acc[i][j][q], 0.f) : acc[i][j][q] * sc;
                    if (col0 + j * 16 < p.N) *(uint2*)(out + j * 16) = make_uint2(pack_bf16x2(v[0], v[1]), pack_bf16x2(v[2], v[3]));
                }
            }
        };
        const bool once = mt.n_same <= 1;
        if (mt.rows <= 16 && once) unit(std::integral_constant<int, 1>{}, std::true_type{});
        else if (once) unit(std::integral_constant<int, 2>{}, std::true_type{});
        else unit(std::integral_constant<int, 2>{}, std::false_type{});
    }
}

// One form for every fp32 batch, right and far from a floor of three bf16 products: for each panel of 32 columns a workgroup loads its rows from
// global memory again and cuts them into parts again, some 200 vector instructions to 12 matrix instructions of 16 rows and a k-tile (counted in
// the source).  FFN of 8 experts of 1024 x 2048, 256 tokens 131 us (floor 16), 4096 tokens 1459 to 1513 (261; fp32 weights 1658); 64 of 2048 x
// 1408, 2048 tokens 2790 to 2804 (539); 16 tokens on 128 of 4096 x 1536 248 (79, 1.6 TB/s).
template <int EPI>
__global__ __launch_bounds__(kMx4SplitWaves * 64) void mx4_f32_kernel(Mx4Product p) {
    constexpr int NW = kMx4SplitWaves;
    __shared__ __align__(16) float xch[NW * 16 * (kMx4N + 4)];

    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g16 = lane >> 4;
    const int KT = p.B.kt;
    const int total = p.counts[kCntEntries] * p.B.panels;
    const int kt0 = (int)((long long)KT * wave / NW), kt1 = (int)((long long)KT * (wave + 1) / NW);
    const size_t panel_bytes = mx4_panel_bytes(KT);

    for (int u = blockIdx.x; u < total; u += gridDim.x) {
        const int entry = u / p.B.panels, panel = u - entry * p.B.panels;
        const MTile mt = p.mtiles[entry];
        const unsigned char* const weights = p.B.at + (size_t)mt.expert * p.B.expert + panel * panel_bytes;
        auto unit = [&](auto MT_tag) {
            constexpr int MT = decltype(MT_tag)::value;  // 16-row groups of the M-tile that hold rows, rounded up
            const char* arow[MT];
#pragma unroll
            for (int i = 0; i < MT; ++i) {
                int r = i * 16 + l16;
                r = row_at(p, mt.list0 + (r < mt.rows ? r : mt.rows - 1));
                arow[i] = (const char*)p.A + (size_t)r * p.lda * 4;
            }
            f32x4 acc[MT][2];
#pragma unroll
            for (int i = 0; i < MT; ++i)
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            struct Tile {
                uint4 codes;
                unsigned scales;
                f32x4 a[MT][2][2];
            };
            // 16 bytes of a row from element k on, zeros past its end (what lies there is not this row's)
            auto piece = [&](const char* row, int k) {
                const bool in = k < p.K;
                f32x4 v = *(const f32x4*)(row + (size_t)(in ? k : 0) * 4);
                if (!in) v = f32x4{0.f, 0.f, 0.f, 0.f};
                return v;
            };
            auto load = [&](int kt, Tile& t) {
                t.codes = *(const uint4*)(weights + mx4_codes_at(kt) + lane * 16);
                t.scales = *(const unsigned short*)(weights + mx4_scales_at(kt) + (g16 >> 1) * 128 + l16 * 8 + (kt & 3) * 2);
#pragma unroll
                for (int i = 0; i < MT; ++i)
#pragma unroll
                    for (int s = 0; s < 2; ++s) {
                        const int k = kt * kMx4K + g16 * 16 + s * 8;
                        t.a[i][s][0] = piece(arow[i], k);
                        t.a[i][s][1] = piece(arow[i], k + 4);
                    }
            };
            auto multiply = [&](const Tile& t) {
#pragma unroll
                for (int s = 0; s < 2; ++s) {
                    const bf16x8 b[2] = {mx4_values(s ? t.codes.z : t.codes.x, mx4_scale<0>(t.scales)),
                                         mx4_values(s ? t.codes.w : t.codes.y, mx4_scale<1>(t.scales))};
#pragma unroll
                    for (int i = 0; i < MT; ++i) {
                        bf16x8 a[3];
                        split_f32(t.a[i][s], a[2], a[1], a[0]);  // (smallest parts first)
#pragma unroll
                        for (int q = 0; q < 3; ++q)
#pragma unroll
                            for (int j = 0; j < 2; ++j)
                                acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(b[j], a[q], acc[i][j], 0, 0, 0);
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
#pragma unroll
            for (int i = 0; i < MT; ++i)
                if (i * 16 < mt.rows) add_parts<EPI, true>(p, xch, wave, acc[i], mt.list0 + i * 16, mt.rows - i * 16, panel);
        };
        if (mt.rows <= 16) unit(std::integral_constant<int, 1>{});
        else if (mt.rows <= 32) unit(std::integral_constant<int, 2>{});
        else unit(std::integral_constant<int, 4>{});
    }
}
