// Gradients of the expert weights: for every expert e, out_e[m, n] = sum over its rows r of P[r, m] Q[r, n], both operands
// row-major with the rows of an expert side by side in the row list.  Included by ffn_backward.hip inside namespace moegps.
//
// The sum runs over rows, so both operands lie the wrong way round for the matrix instruction, which wants eight
// consecutive terms of the sum in a lane.  They are staged in LDS as they lie in memory, 32 rows x 256 columns, and read with the
// transposing LDS read (ds_read_b64_tr_b16): four rows of 16 neighbouring columns to sixteen lanes, a column each.  Any
// order of the 32 rows will do as long as both operands have the same, so a lane takes rows 4 g .. 4 g + 3 and 16 + 4 g ..
// (g the quarter of the wavefront), and a half wavefront reads eight different rows at a time; piece (32 bytes) c of
// row r stands at c ^ (r & 7), which puts these on eight different groups of banks.
//
// A workgroup of eight wavefronts makes a tile of 256 x 256, 128 columns of Q by 64 of P each.  Four steps of 32 rows have room in
// LDS, three are under way; the rows of the listed operand are looked up four steps ahead of its loads.  A step is eight
// fragments of Q against four of P; the hand-over to the next step stands two fragments before the end, so that its first
// reads land under what is left to multiply.
//
// 8192 rows of 8 experts of 4096 x 14336: 2.98 ms, 0.97 PFLOP/s; 98304 of 64 of 2048 x 1408: 1.71 ms, 0.99.  A step takes 0.96 us, of
// which the transposing reads (96 KiB, at half the rate of 16-byte ones) need 0.6 and the matrix pipe 0.8 at the rate of a large
// product; a tile's stores, made by all workgroups at about the same time, come on top (0.4 ms of the 2.98).  Two
// workgroups on a CU with half as high tiles, and the next tile's first steps asked for ahead of the stores, were 3 % slower there
// and 12 to 17 % on the second shape, four wavefronts of 128 x 128 a third.
#pragma once

struct WeightGrad {
    const bf16_t *p, *q;
    const int32_t* rows;     // of the listed operand: row of every list position
    int ldp, ldq;            // row lengths, both multiples of 64
    bf16_t* out[2];          // [E][m_out][n_out]; packed pairs of columns: the first and the second matrix
    int M, N;                // columns of p and of q
    int m_out, n_out;
};

constexpr int kGradRows = 32, kGradTile = 256, kGradStages = 4;
constexpr int kGradPanel = kGradRows * kGradTile * 2;                     // bytes of one operand in a stage
constexpr int kGradNextAt = 2 * kGradStages * kGradPanel;                 // number of the next tile, behind the stages
constexpr int kGradOrderAt = kGradNextAt + 16;                            // the experts, most rows first
constexpr size_t grad_lds(int E) { return (size_t)kGradOrderAt + (size_t)E * sizeof(int32_t); }

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;

// Four rows of a column of a panel to every lane; see lds_read_b128 for when the result may be touched.
template <int OFF>
__device__ __forceinline__ void lds_read_tr(s16x4& dst, unsigned addr) {
    asm volatile("ds_read_b64_tr_b16 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(OFF) : "memory");
}

struct GradFrag {  // 16 columns x 32 rows
    s16x4 lo, hi;
};
__device__ __forceinline__ void landed(GradFrag& f) { asm volatile("" : "+v"(f.lo), "+v"(f.hi)); }
__device__ __forceinline__ bf16x8 whole(const GradFrag& f) {
    return __builtin_bit_cast(bf16x8, __builtin_shufflevector(f.lo, f.hi, 0, 1, 2, 3, 4, 5, 6, 7));
}

// A word of LDS, the same for the whole wavefront.  (As an ordinary read it would be taken to depend on every load into LDS under
// way, and with those wait for the stores of the tile before.)
__device__ __forceinline__ int lds_uniform(unsigned addr) {
    int v;
    asm volatile("ds_read_b32 %0, %1\n\ts_waitcnt lgkmcnt(0)" : "=v"(v) : "v"(addr) : "memory");
    return __builtin_amdgcn_readfirstlane(v);
}

// The experts in LDS, those with most rows first (equal ones by number): big tiles at the end of a launch would be waited for.
__device__ __forceinline__ void order_experts(int* order, int* count, const int32_t* bases, int E) {
    for (int e = threadIdx.x; e < E; e += blockDim.x) count[e] = bases[e + 1] - bases[e];
    __syncthreads();
    for (int e = threadIdx.x; e < E; e += blockDim.x) {
        const int mine = count[e];
        int at = 0;
        for (int o = 0; o < E; ++o) at += count[o] > mine || (count[o] == mine && o < e) ? 1 : 0;
        order[at] = e;
    }
    __syncthreads();
}

// Results of 16 * J columns of p from m0 on by two neighbouring groups of q's columns, from n0 (a multiple of 32) on.  A lane holds
// columns 4 g .. + 3 of a group of q (g the quarter of the wavefront) and column l16 of p's group j.  The two groups are
// regrouped (lane_swap_pairs): quarter g then has columns 8 g .. 8 g + 7 of the 32, 16 bytes of an output row.
template <bool PAIR, int J>
__device__ __forceinline__ void store_grads(const WeightGrad& w, int e, int m0, int n0, const f32x4 (&v0)[J], const f32x4 (&v1)[J],
                                            int lane) {
    const bool aligned = w.n_out % 8 == 0;
    const int c = (PAIR ? (n0 >> 6) * 32 : n0) + (lane >> 4) * 8;
    bf16_t* out = w.out[PAIR ? (n0 >> 5) & 1 : 0] + (size_t)e * w.m_out * w.n_out;
#pragma unroll
    for (int j = 0; j < J; ++j) {
        unsigned px = pack_bf16x2(v0[j][0], v0[j][1]), py = pack_bf16x2(v0[j][2], v0[j][3]);
        unsigned qx = pack_bf16x2(v1[j][0], v1[j][1]), qy = pack_bf16x2(v1[j][2], v1[j][3]);
        lane_swap_pairs(px, qx);
        lane_swap_pairs(py, qy);
        const int m = m0 + j * 16 + (lane & 15);
        if (m >= w.m_out) continue;
        bf16_t* to = out + (size_t)m * w.n_out + c;
        const u32x4 v = {px, py, qx, qy};
        if (aligned) {
            if (c < w.n_out) *(u32x4*)to = v;
        } else {
#pragma unroll
            for (int q = 0; q < 8; ++q)
                if (c + q < w.n_out) to[q] = (bf16_t)(v[q >> 1] >> (16 * (q & 1)));
        }
    }
}

// PAIR: columns of q are packed pairs in blocks of 32 (of one matrix, then of the other).  P_LISTED: the rows of p go through the
// list, those of q are in place; else the reverse.
template <bool PAIR, bool P_LISTED>
__device__ __forceinline__ void weight_grad(const WeightGrad& w, const int32_t* bases, int32_t* queues, int E,
                                            unsigned char* smem) {
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int wn = wave >> 2, wm = wave & 3;  // 128 columns of q by 64 of p each
    const int m_tiles = ceil_div(w.M, kGradTile), n_tiles = ceil_div(w.N, kGradTile);
    const int per_expert = m_tiles * n_tiles;
    const int64_t total = (int64_t)E * per_expert;
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;
    volatile __attribute__((address_space(3))) int& next_tile =
        *(volatile __attribute__((address_space(3))) int*)(__attribute__((address_space(3))) unsigned char*)(smem + kGradNextAt);

    // Tiles are claimed like those of ffn_tiles.h: runs of 32 consecutive ones go to the XCDs in turn, and the workgroups of an
    // XCD, which share its L2, take the tiles of its runs one by one from a counter; one whose XCD has run dry goes on with
    // the next XCD's.  The first claim of a workgroup is made in advance.
    constexpr int run = kGemmGrid / 8;
    int counter = blockIdx.x & 7, dry = 0;
    auto claimed = [&](int i) {  // tile of claim i of the counter, claiming on where it has run out; -1: no tile is left
        for (;;) {
            const int64_t t = ((int64_t)counter + 8 * (int64_t)(i / run)) * run + i % run;
            if (t < total) return t;
            if (++dry == 8) return (int64_t)-1;
            counter = (counter + 1) & 7;
            i = 0;
            if (lane == 0) i = atomicAdd(&queues[counter], 1);
            i = __builtin_amdgcn_readfirstlane(i);
        }
    };
    // (a tile number fits: the gradients of more than 2^31 tiles would be 2^48 bytes)
    if (wave == 0) next_tile = (int)claimed((int)(blockIdx.x >> 3));

    for (;;) {
        lds_wait<0>();
        __builtin_amdgcn_s_barrier();  // also: every wavefront has read the previous tile's stages
        const int tile = lds_uniform(lds_base + kGradNextAt);
        if (tile < 0) break;
        int ahead = 0;  // the claim for the tile after this one, looked at behind the sum
        if (wave == 0 && lane == 0 && dry < 8) ahead = atomicAdd(&queues[counter], 1);
        const int nth = tile / per_expert, in_e = tile - nth * per_expert;
        const int e = lds_uniform(lds_base + kGradOrderAt + (unsigned)nth * 4u);
        // along n first: what is written at a time is whole rows of the matrix (four tiles side by side, down all of m: 0 to 4 % slower)
        const int n0 = in_e % n_tiles * kGradTile, m0 = in_e / n_tiles * kGradTile;
        const int first = bases[e], last = bases[e + 1];
        const int KT = ceil_div(last - first, kGradRows);

        // Loads: instruction i of a wavefront brings rows 2 (wave + 8 i) and + 1 of the step, 512 bytes each.
        const int lane_p = opaque(lane);
        const int row0 = 2 * wave + (lane_p >> 5);
        const int piece = (lane_p & 31) ^ ((row0 & 7) << 1);  // (the same for both rows, 16 apart)
        constexpr unsigned kRange = 0xffffff80u, kPast = 0xfffffff0u;
        const unsigned colp = m0 + piece * 8 < w.M ? (unsigned)(m0 + piece * 8) * 2 : kPast;
        const unsigned colq = n0 + piece * 8 < w.N ? (unsigned)(n0 + piece * 8) * 2 : kPast;
        const bf16_t* listed = P_LISTED ? w.p : w.q;
        const bf16_t* placed = P_LISTED ? w.q : w.p;
        const int ld_l = P_LISTED ? w.ldp : w.ldq, ld_i = P_LISTED ? w.ldq : w.ldp;
        const unsigned col_l = P_LISTED ? colp : colq, col_i = P_LISTED ? colq : colp;
        const auto l_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)listed, 0, (int)kRange, 0x00027000);
        unsigned off_i[2];
#pragma unroll
        for (int i = 0; i < 2; ++i)
            off_i[i] = col_i == kPast ? kPast : (unsigned)(row0 + 16 * i) * (unsigned)ld_i * 2u + col_i;
        int ids[4][2], ids_next[4][2];  // rows of the listed operand that the loads of four steps want, and of the next four
        auto look_up = [&](int kt, int (&r)[2]) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int p = first + kt * kGradRows + row0 + 16 * i;
                r[i] = w.rows[p < last ? p : last - 1];
            }
        };
        auto load = [&](int kt, auto St, const int (&r)[2]) {
            constexpr int stage = decltype(St)::value;
            const int p0 = first + kt * kGradRows;
            const int left = last - p0;  // rows from here on; past them both operands are zeros
            // in place: a descriptor of the rows that are left (none: an empty one)
            const unsigned n = left <= 0 ? 0u : (unsigned)(left < kGradRows ? left : kGradRows) * (unsigned)ld_i * 2u;
            const auto i_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(placed + (size_t)p0 * ld_i), 0, (int)n, 0x00027000);
            unsigned char* to_l = smem + (P_LISTED ? stage : kGradStages + stage) * kGradPanel + wave * 1024;
            unsigned char* to_i = smem + (P_LISTED ? kGradStages + stage : stage) * kGradPanel + wave * 1024;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const unsigned off = row0 + 16 * i < left && col_l != kPast ? (unsigned)r[i] * (unsigned)ld_l * 2u + col_l : kPast;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(l_rsrc, (__attribute__((address_space(3))) void*)(to_l + 8192 * i), 16,
                                                         off, 0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(i_rsrc, (__attribute__((address_space(3))) void*)(to_i + 8192 * i), 16,
                                                         off_i[i], 0, 0, 0);
            }
        };

        f32x4 acc[8][4];
        if (KT > 0) {
            static_for<3>([&](auto U) { look_up(decltype(U)::value, ids_next[decltype(U)::value]); });
            static_for<4>([&](auto U) { look_up(3 + decltype(U)::value, ids[decltype(U)::value]); });
            static_for<3>([&](auto U) { load(decltype(U)::value, U, ids_next[decltype(U)::value]); });
        }
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        // where the lane reads 16-column group c (of the 8 that share a swizzle) of rows 4 g16 + (l16 >> 2)
        const int l16 = lane_p & 15, g16 = lane_p >> 4;
        const int rr = 4 * g16 + (l16 >> 2);
        const unsigned at = lds_base + (unsigned)(rr * 512 + (l16 & 3) * 8);
        unsigned q_at[8], p_at[4];
#pragma unroll
        for (int i = 0; i < 8; ++i) q_at[i] = at + kGradStages * kGradPanel + wn * 256 + ((i ^ (rr & 7)) * 32);
#pragma unroll
        for (int j = 0; j < 4; ++j) p_at[j] = at + (wm >> 1) * 256 + ((((wm & 1) * 4 + j) ^ (rr & 7)) * 32);

        if (KT > 0) {
            GradFrag pf[2][4], qf[4];  // of q: fragment f in qf[f % 4]
            auto read = [&](GradFrag& f, unsigned addr, auto St) {
                constexpr int off = decltype(St)::value * kGradPanel;
                lds_read_tr<off>(f.lo, addr);
                lds_read_tr<off + 16 * 512>(f.hi, addr);
            };
            constexpr int kLoads = 4, kRows = 8;  // of a wavefront: a step's share of both panels; rows looked up in four steps
            wait_vmcnt<2 * kLoads>();             // step 0 has landed
            __builtin_amdgcn_s_barrier();
            static_for<4>([&](auto J) { read(pf[0][decltype(J)::value], p_at[decltype(J)::value], std::integral_constant<int, 0>{}); });
            static_for<4>([&](auto I) { read(qf[decltype(I)::value], q_at[decltype(I)::value], std::integral_constant<int, 0>{}); });
            // step kt in stage U; 12 fragments of two reads each, in the order p0 .. p3, q0 .. q7.  MORE: one of four steps behind which
            // others come (behind the others nobody wants the rows that step 0 would look up)
            auto body = [&](int kt, auto U, auto more_tag) {
                constexpr bool MORE = decltype(more_tag)::value;
                constexpr int u = decltype(U)::value;
                constexpr std::integral_constant<int, (u + 1) % 4> next{};
                constexpr std::integral_constant<int, (u + 3) % 4> far{};
                static_for<8>([&](auto F) {
                    constexpr int f = decltype(F)::value;
                    if constexpr (f == 6) {
                        lds_wait<0>();                  // all reads of this step
                        // step kt + 1 has landed: newer are steps kt + 2 and kt + 3, and rows looked up in step 0 of these four
                        wait_vmcnt<2 * kLoads + (MORE && u < 3 ? kRows : 0)>();
                        __builtin_amdgcn_s_barrier();
                        static_for<4>([&](auto J) { read(pf[(u + 1) & 1][decltype(J)::value], p_at[decltype(J)::value], next); });
                        static_for<2>([&](auto I) { read(qf[decltype(I)::value], q_at[decltype(I)::value], next); });
                    } else if constexpr (f < 6) {
                        lds_wait<(f <= 4 ? 6 : 4)>();   // fragment f has landed; newer are three (at f = 5 two) of q
                    }
                    if constexpr (f == 0) static_for<4>([&](auto J) { landed(pf[u & 1][decltype(J)::value]); });
                    landed(qf[f % 4]);
                    __builtin_amdgcn_sched_barrier(0);
#pragma unroll
                    for (int j = 0; j < 4; ++j)
                        acc[f][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(whole(qf[f % 4]), whole(pf[u & 1][j]), acc[f][j], 0, 0, 0);
                    __builtin_amdgcn_sched_barrier(0);
                    if constexpr (f < 4) read(qf[f], q_at[f + 4], U);
                    else if constexpr (f >= 6) read(qf[f - 4], q_at[f - 4], next);
                    // stage far was read a step ago; the barrier at that step's end says so for every wavefront
                    if constexpr (f == 1) load(kt + 3, far, ids[u]);
                    if constexpr (MORE && f == 2 && u == 0) static_for<4>([&](auto V) { look_up(kt + 7 + decltype(V)::value, ids_next[decltype(V)::value]); });
                    __builtin_amdgcn_sched_barrier(0);
                });
            };
            int kt = 0;
            for (; kt + 4 < KT; kt += 4) {
                static_for<4>([&](auto U) { body(kt + decltype(U)::value, U, std::true_type{}); });
#pragma unroll
                for (int i = 0; i < 4; ++i)
#pragma unroll
                    for (int h = 0; h < 2; ++h) ids[i][h] = ids_next[i][h];
            }
            static_for<4>([&](auto U) {
                if (kt + decltype(U)::value < KT) body(kt + decltype(U)::value, U, std::false_type{});
            });
            // (the last hand-over read fragments that nobody multiplies)
            lds_wait<0>();
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                landed(pf[0][j]);
                landed(pf[1][j]);
                landed(qf[j]);
            }
        } else {
            __builtin_amdgcn_s_barrier();  // (every wavefront has read next_tile)
        }
        if (wave == 0) next_tile = dry < 8 ? (int)claimed(__builtin_amdgcn_readfirstlane(ahead)) : -1;
        const int lane_e = opaque(lane);
#pragma unroll
        for (int i = 0; i < 8; i += 2)
            store_grads<PAIR, 4>(w, e, m0 + wm * 64, n0 + wn * 128 + i * 16, acc[i], acc[i + 1], lane_e);
    }
}

// The gradients of the first product's matrices and of the second's in one launch: a workgroup that finds no tile of the first left
// goes on to the second.
template <bool PAIR>
__global__ __launch_bounds__(512, 2) void weight_grads_kernel(WeightGrad w13, WeightGrad w2, const int32_t* __restrict__ bases,
                                                              int32_t* __restrict__ queues, int E) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    order_experts((int*)(smem + kGradOrderAt), (int*)smem, bases, E);
    weight_grad<PAIR, true>(w13, bases, queues, E, smem);
    __builtin_amdgcn_s_barrier();  // (the number of the next tile is written again)
    weight_grad<false, false>(w2, bases, queues + 8, E, smem);
}

// ---------------------------------------------------------------------------
// few rows per expert
// ---------------------------------------------------------------------------
// What bounds the gradients then is writing them, and a tile is little more than its start, a step or two, and its stores.  So tiles
// are small, 64 of m by 256 of n, four workgroups share a CU, none waits for another, and tiles without rows are stores
// alone.  A wavefront has all of m by 64 of n.  Two steps of 32 rows have room in LDS.  128 tokens, top-8 of 128 experts of 4096 x
// 1536 (4.8 GB of gradients): 1403 us with the tiles above, 1240 with half as high ones and two workgroups on a CU.
constexpr int kFewM = 64, kFewN = 256, kFewStages = 2;
constexpr int kFewPanelM = kGradRows * kFewM * 2, kFewPanelN = kGradRows * kFewN * 2, kFewStage = kFewPanelM + kFewPanelN;

// bases null: there are no rows.
template <bool PAIR, bool P_LISTED>
__device__ __forceinline__ void few_rows_tile(const WeightGrad& w, const int32_t* bases, int64_t tile, unsigned char* smem) {
    const int lane = threadIdx.x & 63;
    const int wave = __builtin_amdgcn_readfirstlane((int)threadIdx.x >> 6);
    const int m_tiles = ceil_div(w.M, kFewM), n_tiles = ceil_div(w.N, kFewN);
    const int e = (int)(tile / ((int64_t)m_tiles * n_tiles));
    const int in_e = (int)(tile - (int64_t)e * ((int64_t)m_tiles * n_tiles));
    const int n0 = in_e % n_tiles * kFewN, m0 = in_e / n_tiles * kFewM;
    const int first = bases ? bases[e] : 0, rows = bases ? bases[e + 1] - first : 0;
    const int KT = ceil_div(rows, kGradRows);
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;

    f32x4 acc[4][4];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

    if (KT > 0) {
        // Loads: a wavefront brings 8 rows of p's panel (128 bytes each) with one instruction, and with four rows 2 (wave + 4 i) and + 1
        // of q's (512 bytes).  Pieces of 32 bytes stand at piece ^ ((row >> 1) & 3) and piece ^ (row & 7): see above.
        constexpr unsigned kRange = 0xffffff80u, kPast = 0xfffffff0u;
        const int row_p = 8 * wave + (lane >> 3), row_q = 2 * wave + (lane >> 5);
        const int at_p = m0 + ((lane & 7) ^ (((row_p >> 1) & 3) << 1)) * 8, at_q = n0 + ((lane & 31) ^ ((row_q & 7) << 1)) * 8;
        const auto p_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)w.p, 0, (int)kRange, 0x00027000);
        const auto q_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)w.q, 0, (int)kRange, 0x00027000);
        // Rows that go through the list are addressed from the start of their operand (the host checks that 32 bits reach); those in
        // place from the step's first, as all of a batch's rows may be this expert's: 32768 of 65792 values are 2^32 bytes.
        auto load = [&](int kt) {
            unsigned char* to = smem + (kt & 1) * kFewStage;
            const int left = rows - kt * kGradRows;  // rows from the step's first on
            const int p0 = first + kt * kGradRows;
            const int32_t* list = w.rows + p0;
            const auto here = __builtin_amdgcn_make_buffer_rsrc((void*)(P_LISTED ? w.q + (size_t)p0 * w.ldq : w.p + (size_t)p0 * w.ldp),
                                                                0, (int)kRange, 0x00027000);
            unsigned off = kPast;  // past the rows and the columns: zeros
            const int rp = opaque(row_p), rq0 = opaque(row_q);  // (offsets kept across the steps would not leave the registers)
            if (rp < left && at_p < w.M)
                off = ((unsigned)(P_LISTED ? list[(unsigned)rp] : rp) * (unsigned)w.ldp + (unsigned)at_p) * 2u;
            __builtin_amdgcn_raw_ptr_buffer_load_lds(P_LISTED ? p_rsrc : here,
                                                     (__attribute__((address_space(3))) void*)(to + wave * 1024), 16, off, 0, 0, 0);
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const int rq = rq0 + 8 * i;
                off = kPast;
                if (rq < left && at_q < w.N)
                    off = ((unsigned)(P_LISTED ? rq : list[(unsigned)rq]) * (unsigned)w.ldq + (unsigned)at_q) * 2u;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    P_LISTED ? here : q_rsrc,
                    (__attribute__((address_space(3))) void*)(to + kFewPanelM + (wave + 4 * i) * 1024), 16, off, 0, 0, 0);
            }
        };
        const int l16 = lane & 15, g16 = lane >> 4, rr = 4 * g16 + (l16 >> 2);
        const unsigned at = lds_base + (l16 & 3) * 8;
        load(0);
        for (int kt = 0; kt < KT; ++kt) {
            if (kt + 1 < KT) load(kt + 1);
            __builtin_amdgcn_sched_barrier(0);
            if (kt + 1 < KT) wait_vmcnt<5>();  // (the loads of the next step)
            else wait_vmcnt<0>();
            __builtin_amdgcn_s_barrier();
            const unsigned stage = at + (unsigned)((kt & 1) * kFewStage);
            GradFrag pf[4], qf[4];
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                const unsigned p = stage + (unsigned)(rr * (kFewM * 2) + (i ^ ((rr >> 1) & 3)) * 32);
                const unsigned q = stage + (unsigned)(kFewPanelM + rr * (kFewN * 2) + (wave >> 1) * 256 +
                                                      (((wave & 1) * 4 + i) ^ (rr & 7)) * 32);
                lds_read_tr<0>(pf[i].lo, p);
                lds_read_tr<16 * kFewM * 2>(pf[i].hi, p);
                lds_read_tr<0>(qf[i].lo, q);
                lds_read_tr<16 * kFewN * 2>(qf[i].hi, q);
            }
            lds_wait<0>();
#pragma unroll
            for (int i = 0; i < 4; ++i) {
                landed(pf[i]);
                landed(qf[i]);
            }
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int i = 0; i < 4; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(whole(qf[i]), whole(pf[j]), acc[i][j], 0, 0, 0);
            __builtin_amdgcn_s_barrier();  // everybody has read the stage
        }
    }
#pragma unroll
    for (int i = 0; i < 4; i += 2) store_grads<PAIR, 4>(w, e, m0, n0 + wave * 64 + i * 16, acc[i], acc[i + 1], lane);
}

template <bool PAIR>
__global__ __launch_bounds__(256, 4) void few_rows_grads_kernel(WeightGrad w13, WeightGrad w2, const int32_t* __restrict__ bases,
                                                                int64_t tiles13, int64_t tiles) {
    __shared__ __attribute__((aligned(1024))) unsigned char smem[kFewStages * kFewStage];
    for (int64_t t = blockIdx.x; t < tiles; t += gridDim.x) {
        if (t < tiles13) few_rows_tile<PAIR, true>(w13, bases, t, smem);
        else few_rows_tile<false, false>(w2, bases, t - tiles13, smem);
    }
}
inline int64_t few_rows_tiles(const WeightGrad& w, int E) {
    return (int64_t)E * ceil_div(w.M, kFewM) * ceil_div(w.N, kFewN);
}
