// Gradients of the expert weights: for every expert e, out_e[m, n] = sum over its rows r of P[r, m] Q[r, n], both operands
// row-major with the rows of an expert side by side in the row list.  Included by ffn_backward.hip inside namespace moegps.
//
// The sum runs over rows, so both operands lie the wrong way round for the matrix instruction, which wants eight
// consecutive terms of the sum in a lane.  They are staged in LDS as they lie in memory, 32 rows x 256 columns, and read with the
// transposing LDS read (ds_read_b64_tr_b16): four rows of 16 neighbouring columns to sixteen lanes, a column each.  Any
// order of the 32 rows will do as long as both operands have the same, so a lane takes rows 4 g .. 4 g + 3 and 16 + 4 g ..
// (g the quarter of the wavefront), and a half wavefront reads eight different rows at a time; piece (32 bytes) c of
// row r stands at c ^ (r & 7), which puts these on eight different groups of banks.
#pragma once

struct WeightGrad {
    const bf16_t *p, *q;
    const int32_t* rows;     // of the listed operand: row of every list position
    int ldp, ldq;            // row lengths, both multiples of 64
    const int32_t* bases;    // [E + 1] first list position of an expert; null: there are no rows
    bf16_t* out[2];          // [E][m_out][n_out]; packed pairs of columns: the first and the second matrix
    int M, N;                // columns of p and of q
    int m_out, n_out;
    int E;
};

constexpr int kGradRows = 32, kGradTile = 256, kGradStages = 4;
constexpr int kGradPanel = kGradRows * kGradTile * 2;                     // bytes of one operand in a stage
constexpr size_t kGradLds = (size_t)2 * kGradStages * kGradPanel;

typedef __attribute__((__vector_size__(4 * sizeof(short)))) short s16x4;

// PAIR: columns of q are packed pairs in blocks of 32 (of one matrix, then of the other).  P_LISTED: the rows of p go through the
// list, those of q are in place; else the reverse.
template <bool PAIR, bool P_LISTED>
__global__ __launch_bounds__(512, 2) void weight_grad_kernel(WeightGrad w) {
    extern __shared__ __attribute__((aligned(1024))) unsigned char smem[];
    const int tid = threadIdx.x;
    const int lane = tid & 63;
    const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
    const int l16 = lane & 15, g16 = lane >> 4;
    const int wn = wave >> 2, wm = wave & 3;  // 128 columns of q by 64 of p each
    const int m_tiles = ceil_div(w.M, kGradTile), n_tiles = ceil_div(w.N, kGradTile);
    const int64_t total = (int64_t)w.E * m_tiles * n_tiles;
    const unsigned lds_base = (unsigned)(size_t)(__attribute__((address_space(3))) unsigned char*)smem;

    for (int64_t tile = blockIdx.x; tile < total; tile += gridDim.x) {
        const int e = (int)(tile / (m_tiles * n_tiles));
        const int in_e = (int)(tile - (int64_t)e * (m_tiles * n_tiles));
        const int n0 = (in_e % n_tiles) * kGradTile, m0 = (in_e / n_tiles) * kGradTile;
        const int first = w.bases ? w.bases[e] : 0, last = w.bases ? w.bases[e + 1] : 0;
        const int KT = ceil_div(last - first, kGradRows);

        // Loads: instruction i of a wavefront brings rows 2 (wave + 8 i) and + 1 of the step, 512 bytes each
        const int row_of[2] = {2 * wave + (lane >> 5), 2 * (wave + 8) + (lane >> 5)};
        const int piece = (lane & 31) ^ ((row_of[0] & 7) << 1);  // (the same for both rows, 16 apart)
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
        for (int i = 0; i < 2; ++i) off_i[i] = col_i == kPast ? kPast : (unsigned)row_of[i] * (unsigned)ld_i * 2u + col_i;
        auto fetch_rows = [&](int kt, int (&r)[2]) {
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int p = first + kt * kGradRows + row_of[i];
                r[i] = w.rows[p < last ? p : last - 1];
            }
        };
        auto load = [&](int kt, int stage, const int (&r)[2]) {
            unsigned char* to_p = smem + stage * kGradPanel;
            unsigned char* to_q = smem + (kGradStages + stage) * kGradPanel;
            const int p0 = first + kt * kGradRows;
            const int left = last - p0;  // rows from here on; past them both operands are zeros
            // in place: a descriptor of the rows that are left (none: an empty one)
            const unsigned n = left <= 0 ? 0u : (unsigned)(left < kGradRows ? left : kGradRows) * (unsigned)ld_i * 2u;
            const auto i_rsrc = __builtin_amdgcn_make_buffer_rsrc((void*)(placed + (size_t)p0 * ld_i), 0, (int)n, 0x00027000);
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const unsigned off = row_of[i] < left && col_l != kPast ? (unsigned)r[i] * (unsigned)ld_l * 2u + col_l : kPast;
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    l_rsrc, (__attribute__((address_space(3))) void*)((P_LISTED ? to_p : to_q) + (wave + 8 * i) * 1024), 16, off,
                    0, 0, 0);
                __builtin_amdgcn_raw_ptr_buffer_load_lds(
                    i_rsrc, (__attribute__((address_space(3))) void*)((P_LISTED ? to_q : to_p) + (wave + 8 * i) * 1024), 16,
                    off_i[i], 0, 0, 0);
            }
        };

        f32x4 acc[8][4];
#pragma unroll
        for (int i = 0; i < 8; ++i)
#pragma unroll
            for (int j = 0; j < 4; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        // where the lane reads 16-column group c (of the 8 that share a swizzle) of rows 4 g16 + (l16 >> 2)
        const int rr = 4 * g16 + (l16 >> 2);
        const unsigned at = lds_base + (unsigned)(rr * 512 + (l16 & 3) * 8);
        unsigned q_at[8], p_at[4];
#pragma unroll
        for (int i = 0; i < 8; ++i)
            q_at[i] = at + kGradStages * kGradPanel + wn * 256 + ((i ^ (rr & 7)) * 32);
#pragma unroll
        for (int j = 0; j < 4; ++j)
            p_at[j] = at + (wm >> 1) * 256 + ((((wm & 1) * 4 + j) ^ (rr & 7)) * 32);

        for (int kt = 0; kt < KT; ++kt) {
            int r[2];
            fetch_rows(kt, r);
            load(kt, 0, r);
            __syncthreads();
            auto frag = [&](unsigned a) {
                const s16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(size_t)a);
                const s16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((__attribute__((address_space(3))) s16x4*)(size_t)(a + 16 * 512));
                return __builtin_bit_cast(bf16x8, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
            };
            bf16x8 qf[8], pf[4];
#pragma unroll
            for (int j = 0; j < 4; ++j) pf[j] = frag(p_at[j]);
#pragma unroll
            for (int i = 0; i < 8; ++i) qf[i] = frag(q_at[i]);
#pragma unroll
            for (int i = 0; i < 8; ++i)
#pragma unroll
                for (int j = 0; j < 4; ++j)
                    acc[i][j] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(qf[i], pf[j], acc[i][j], 0, 0, 0);
            __syncthreads();
        }
        // A lane holds columns 4 g16 .. + 3 of q's group i and column l16 of p's group j.  Two neighbouring groups are
        // regrouped (lane_swap_pairs): quarter g then has columns 8 g .. 8 g + 7 of the 32, 16 bytes of an output row.
        const bool aligned = w.n_out % 8 == 0;
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            const int col = n0 + wn * 128 + i * 16;  // of q, a multiple of 32
            const int sel = PAIR ? (col >> 5) & 1 : 0;
            const int c = (PAIR ? (col >> 6) * 32 : col) + g16 * 8;
            bf16_t* out = w.out[sel] + (size_t)e * w.m_out * w.n_out;
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                unsigned px = pack_bf16x2(acc[i][j][0], acc[i][j][1]), py = pack_bf16x2(acc[i][j][2], acc[i][j][3]);
                unsigned qx = pack_bf16x2(acc[i + 1][j][0], acc[i + 1][j][1]);
                unsigned qy = pack_bf16x2(acc[i + 1][j][2], acc[i + 1][j][3]);
                lane_swap_pairs(px, qx);
                lane_swap_pairs(py, qy);
                const int m = m0 + wm * 64 + j * 16 + l16;
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
    }
}
