// Grouped products and the experts' FFN with weights in 4 bits (include/moegps_mx4.h; layout: mx4.h).
//
// Rows are tiled by expert, as in grouped_ffn.hip: the rows of all segments of an expert are listed one after the other by the table
// builder (ffn_tables.h) and cut into M-tiles together.  Bound by the weights' bytes up to some 50 rows per expert, then by the matrix
// pipe; fp32 rows by neither (mx4_f32_kernel).  Both products and tables, us, bf16 weights -> 4 bits on the same batches: top-8 of 128
// experts of 4096 x 1536, 1 token 59 -> 33, 128 391 -> 162, 1000 599 -> 372; top-2 of 8 of 4096 x 14336, 16 tokens 335 -> 118, 128
// 471 -> 192, 1000 745 -> 606, 4096 2283 -> 2073 (1.39 PFLOP/s).
//
// With bf16 rows the hidden activation is rounded to bf16 between the products, as it is with bf16 weights: the second product takes bf16
// operands, and a hidden row is half as long.  It doubles the error's square: results are 2.3 to 2.4e-3 from 64 bits in norm, where rounding
// them alone makes 1.6 to 1.7e-3.  Kept in two bf16 parts it would double the second product's matrix instructions and the hidden rows.
#include "mx4.h"

namespace moegps {

#include "ffn_tiles.h"
#include "mx4_stream.h"

// The weights' way into the tiles of ffn_tiles.h: a wavefront's 32 columns are a panel, a k-tile is 16 bytes and two scales per lane.
struct Mx4Weights {
    static constexpr bool kFour = true;
    static __device__ __forceinline__ size_t panel_bytes(int kt) { return mx4_panel_bytes(kt); }
    static __device__ __forceinline__ unsigned lane_scales(int lane) { return (lane >> 5) * 128 + (lane & 15) * 8; }
    static __device__ __forceinline__ unsigned codes_at(int i) { return mx4_codes_at(i); }
    static __device__ __forceinline__ unsigned scales_at(int i) { return mx4_scales_at(i) + (i & 3) * 2; }
    static __device__ __forceinline__ bf16x8 values(unsigned codes, unsigned scales, int j) {
        return mx4_values(codes, j ? mx4_scale<1>(scales) : mx4_scale<0>(scales));
    }
};

template <int EPI>
__global__ __launch_bounds__(512, 2) void mx4_tile_kernel(Mx4Product p, int32_t* __restrict__ queues, int n_packed, bool past_caches) {
    tile_product<EPI, kAlone, Mx4Weights>((const bf16_t*)p.A, p.lda, (const bf16_t*)p.B.at, p.B.expert, (bf16_t*)p.C, p.ldc, p.mtiles,
                                          p.counts, queues, n_packed, p.B.kt * kMx4K, kTileGroup, past_caches, p.rm, nullptr,
                                          RowCopy{}, nullptr);
}

struct Mx4Ws {
    int32_t* rowlist;
    int32_t* tokens;  // of the rows at the list's positions, and their gate weights
    float* gates;
    MTile* tiles[2];
    int32_t* counts;  // kCntStride ints per table
    int32_t* queues;  // per-XCD claim counters of both products
    void* h;          // hidden activations in row-list order (FFN)
    int capacity;
};

// hidden: width of a hidden row, 0: none
static size_t mx4_ws_layout(int64_t A, int hidden, int nseg, int dtype, char* base, Mx4Ws* ws) {
    size_t off = 0;
    auto take = [&](size_t bytes) {
        void* p = base ? (void*)(base + off) : nullptr;
        off += align_up(bytes, 256);
        return p;
    };
    const int64_t A1 = A > 0 ? A : 1;
    Mx4Ws w;
    w.capacity = (int)(ceil_div64(A1, kMinBM) + nseg);
    w.rowlist = (int32_t*)take((size_t)A1 * sizeof(int32_t));
    w.tokens = (int32_t*)take((size_t)A1 * sizeof(int32_t));
    w.gates = (float*)take((size_t)A1 * sizeof(float));
    for (int i = 0; i < 2; ++i) w.tiles[i] = (MTile*)take((size_t)w.capacity * sizeof(MTile));
    w.counts = (int32_t*)take(256);
    w.queues = w.counts ? w.counts + 2 * kCntStride : nullptr;
    w.h = hidden ? take((size_t)A1 * hidden * dtype_size(dtype)) : nullptr;
    if (ws) *ws = w;
    return off;
}

// How a product is done: K split between wavefronts, eight panels side by side, fp32 (mx4_stream.h), tiles of up to 256 rows (ffn_tiles.h).
enum Mx4Form { kSplit, kWide, kF32, kTiles };
constexpr int kFormRows[] = {kMx4SplitRows, kMx4WideRows, kMx4F32Rows, 0};  // of an M-tile; 0: the table builder chooses

// The form goes by the whole batch (A rows, E experts), not by the launched slot range, so that a row gets the same bits from a launch
// over some slots as from one over all.  Both products, us, split / wide / tiles:
//   split where eight panels side by side are fewer units than CUs, up to 8 rows per expert: 1 token, top-8 of 128 experts of 4096 x 1536
//     35 / 38 / 51, top-2 of 8 of 4096 x 14336 51 / 79 / 107, 4 tokens 99 / 115 / 162, 16 tokens (the second product alone) 126 / 140 / 181;
//   wide up to 24 rows per expert: 128 tokens, top-8 of 128 312 / 204 / 223, 64, top-2 of 8 232 / 179 / 216, 200, top-6 of 64 of 2048 x 1408
//     147 / 79 / 88, but 512, top-8 of 128 - / 332 / 320, 777, top-6 of 64 - / 162 / 139; up to 128 where tiles would not
//     go once round the chip: 400, top-4 of 16 of 4096 x 688, first product alone 46 / 30 / 40.
// The rule sees the mean, not how the rows lie: where a few experts have nearly all of them it may choose the slower form.  rule / tiles, top-8 of
// 128 experts of 4096 x 1536: 384 tokens on 95 of them (up to 257 rows) 283 / 280, on 32 (up to 346) 198 / 163, on 16 172 / 144; 128 tokens on
// 32 (up to 117) 116 / 125, on 14 84 / 81; top-2 of 8 of 4096 x 14336, 96 tokens (96 rows on one) 124 / 144.
// Hidden rows of 2^31 values and more are left to the tiles, which address them from the tile's first row; the others have 32-bit
// offsets into all of them.  values: of the product's rows.
static Mx4Form form_of(int opt, int dtype, int64_t A, int E, const Mx4Matrix& m, int64_t values) {
    if (dtype == MOE_DTYPE_F32) return kF32;
    if (values > (1ll << 31) - 64) return kTiles;
    if (opt >= 0) return opt == 0 ? kTiles : opt == 1 ? kSplit : kWide;
    const int64_t experts = A < E ? A : E, across = ceil_div(m.panels, 8);
    if (A <= (int64_t)8 * E && experts * across < kGemmGrid) return kSplit;
    if (A <= (int64_t)24 * E) return kWide;
    return A <= (int64_t)128 * E && (ceil_div64(A, 128) + E) * across < kGemmGrid ? kWide : kTiles;
}

template <int EPI>
static int launch_mx4(const Mx4Product& p, Mx4Form form, int E, int32_t* queues, hipStream_t st) {
    auto go = [&](auto kern, int grid, size_t lds, auto... more) {
        hipLaunchKernelGGL(kern, dim3(grid), dim3(512), lds, st, p, more...);
        return check_launch();
    };
    const int n_packed = EPI == kEpiSwiglu ? 2 * p.N : p.N;
    const bool past = past_caches(E, p.B.expert / sizeof(bf16_t));
    static std::atomic<unsigned long long> raised{0}, raised_wide{0};
    switch (form) {
        case kSplit: return go(mx4_split_kernel<EPI>, 4 * kGemmGrid, 0);
        case kF32: return go(mx4_f32_kernel<EPI>, 4 * kGemmGrid, 0);
        case kWide: {
            const auto kern = mx4_wide_kernel<EPI>;
            if (const int rc = raise_lds((const void*)kern, kMx4WideLds, raised_wide); rc != MOE_OK) return rc;
            return go(kern, 2 * kGemmGrid, kMx4WideLds);
        }
        default: {
            const auto kern = mx4_tile_kernel<EPI>;
            if (const int rc = raise_lds((const void*)kern, kStageLds + 16, raised); rc != MOE_OK) return rc;
            return go(kern, kGemmGrid, kStageLds + 16, queues, n_packed, past);
        }
    }
}

// What both calls check.
struct Mx4Rows {
    int dtype, E, nseg, seg_begin, seg_end, k;
    int64_t A, rows_x;
    const void* x;
    const int32_t *assign_of_row, *seg_offsets, *slot_expert;
    const float* topk_w;
    const void *packed, *y, *workspace;
};
static int check_rows(const Mx4Rows& r, int K, int N, int ffn) {
    if (r.dtype != MOE_DTYPE_F32 && r.dtype != MOE_DTYPE_BF16) return MOE_ERR_INVALID_ARG;
    if (r.A < 0 || K < 1 || N < 1 || ffn < 1 || r.E < 1 || r.nseg < 1) return MOE_ERR_INVALID_ARG;
    if (r.seg_begin < 0 || r.seg_end > r.nseg || r.seg_begin > r.seg_end) return MOE_ERR_INVALID_ARG;
    if (r.assign_of_row && (r.k < 1 || r.rows_x < 0)) return MOE_ERR_INVALID_ARG;
    if (r.topk_w && !r.assign_of_row) return MOE_ERR_INVALID_ARG;
    if (r.nseg > MOE_MAX_SEGMENTS || r.E > MOE_MAX_EXPERTS || r.A >= (1ll << 31)) return MOE_ERR_UNSUPPORTED;
    if (K > kMaxWidth || N > kMaxWidth || ffn > kMaxWidth) return MOE_ERR_UNSUPPORTED;
    if ((size_t)K * dtype_size(r.dtype) % 16 != 0 || (size_t)N * dtype_size(r.dtype) % 16 != 0) return MOE_ERR_UNSUPPORTED;
    const int64_t rows = r.assign_of_row ? r.rows_x : r.A;
    if (rows >= (1ll << 31) || rows * K > (1ll << 31) - 64) return MOE_ERR_UNSUPPORTED;  // 32-bit offsets
    if (!r.seg_offsets || !r.slot_expert || !r.packed || !r.workspace) return MOE_ERR_INVALID_ARG;
    if (r.A > 0 && (!r.x || !r.y)) return MOE_ERR_INVALID_ARG;
    return MOE_OK;
}

// The lists that the table builder makes: with rows that are gathered their tokens (looked up once, not twice for every tile), and their gate weights.
static RowLists row_lists(const Mx4Rows& r, const Mx4Ws& ws) {
    return RowLists{ws.rowlist, r.assign_of_row ? ws.tokens : nullptr, r.assign_of_row, r.k, r.topk_w ? ws.gates : nullptr, r.topk_w};
}

int mx4_ffn_call(const moe_ffn_mx4_args& a, hipStream_t st, const FfnOptions& opt, FfnStage stage, TableJob* job_out) {
    if (a.reserved != 0) return MOE_ERR_INVALID_ARG;
    const Mx4Rows rows{a.dtype, a.E, a.nseg, a.seg_begin, a.seg_end, a.k, a.A, a.rows_x, a.x, a.assign_of_row,
                       a.seg_offsets, a.slot_expert, a.topk_w, a.packed, a.y, a.workspace};
    if (const int rc = check_rows(rows, a.d, a.d, a.ffn); rc != MOE_OK) return rc;
    const int hidden = mx4_hidden(a.ffn);
    Mx4Ws ws;
    if (a.workspace_bytes < mx4_ws_layout(a.A, hidden, a.nseg, a.dtype, (char*)a.workspace, &ws)) return MOE_ERR_WORKSPACE_TOO_SMALL;
    if (a.A == 0 || a.seg_begin == a.seg_end) {
        if (job_out) *job_out = TableJob{};
        return MOE_OK;
    }
    const Mx4Matrix m1 = mx4_first(a.packed, a.d, a.ffn, a.relu), m2 = mx4_second(a.packed, a.E, a.d, a.ffn, a.relu);
    const Mx4Form form1 = form_of(opt.stream, a.dtype, a.A, a.E, m1, 0), form2 = form_of(opt.stream, a.dtype, a.A, a.E, m2, a.A * hidden);
    // Products with M-tiles of the same given height share a table; where the builder chooses the height, by the tiles that a product
    // has, each has its own.
    const bool own2 = kFormRows[form1] != kFormRows[form2] || form2 == kTiles;
    const TableSpec t1{ws.tiles[0], ws.counts, nullptr, kFormRows[form1], ws.capacity, m1.kt, 0, ceil_div(m1.panels, 8), 0, 0};
    const TableSpec t2{own2 ? ws.tiles[1] : nullptr, ws.counts + kCntStride, nullptr, kFormRows[form2], ws.capacity, m2.kt, 0,
                       ceil_div(m2.panels, 8), 0, 0};
    const int second = own2 ? 1 : 0;
    const TableJob job{a.E, a.seg_begin, a.seg_end, t1, t2, row_lists(rows, ws), ws.queues, 16, nullptr, nullptr};
    if (stage == kFfnJobOnly) {
        *job_out = job;
        return MOE_OK;
    }
    if (stage == kFfnAll)
        if (const int rc = launch_tables(a.A, a.seg_offsets, a.slot_expert, job, st); rc != MOE_OK) return rc;
    const RowMap rm1{a.assign_of_row ? ws.tokens : ws.rowlist, nullptr, 1, nullptr, nullptr, nullptr};
    const RowMap rm2{nullptr, nullptr, 1, ws.rowlist, a.topk_w ? a.assign_of_row : nullptr, a.topk_w};
    const Mx4Product p1{a.x, a.d, a.d, m1, ws.h, hidden, hidden, ws.tiles[0], ws.counts, rm1, nullptr};
    const Mx4Product p2{ws.h, hidden, hidden, m2, a.y, a.d, a.d, ws.tiles[second], ws.counts + second * kCntStride, rm2,
                        a.topk_w ? ws.gates : nullptr};
    const int rc = a.relu ? launch_mx4<kEpiRelu>(p1, form1, a.E, ws.queues, st) : launch_mx4<kEpiSwiglu>(p1, form1, a.E, ws.queues, st);
    return rc != MOE_OK ? rc : launch_mx4<kEpiNone>(p2, form2, a.E, ws.queues + 8, st);
}

}  // namespace moegps

extern "C" size_t moe_grouped_product_mx4_workspace_bytes(int64_t A, int K, int N, int nseg, int dtype) {
    using namespace moegps;
    if (!ffn_shape_in_range(A, K, N, nseg, dtype)) return 0;
    return mx4_ws_layout(A, 0, nseg, dtype, nullptr, nullptr);
}

extern "C" int moe_grouped_product_mx4(const moe_product_mx4_args* a, void* stream) {
    using namespace moegps;
    if (!a) return MOE_ERR_INVALID_ARG;
    const Mx4Rows rows{a->dtype, a->E, a->nseg, a->seg_begin, a->seg_end, a->k, a->A, a->rows_x, a->x, a->assign_of_row,
                       a->seg_offsets, a->slot_expert, a->topk_w, a->packed, a->y, a->workspace};
    if (const int rc = check_rows(rows, a->K, a->N, 1); rc != MOE_OK) return rc;
    Mx4Ws ws;
    if (a->workspace_bytes < mx4_ws_layout(a->A, 0, a->nseg, a->dtype, (char*)a->workspace, &ws)) return MOE_ERR_WORKSPACE_TOO_SMALL;
    if (a->A == 0 || a->seg_begin == a->seg_end) return MOE_OK;
    hipStream_t st = (hipStream_t)stream;
    const Mx4Matrix m = mx4_matrix(a->packed, a->K, ceil_div(a->N, kMx4N));
    const Mx4Form form = form_of(ffn_options().stream, a->dtype, a->A, a->E, m, 0);
    const TableSpec t1{ws.tiles[0], ws.counts, nullptr, kFormRows[form], ws.capacity, m.kt, 0, ceil_div(m.panels, 8), 0, 0}, none{};
    const TableJob job{a->E, a->seg_begin, a->seg_end, t1, none, row_lists(rows, ws), ws.queues, 16, nullptr, nullptr};
    if (const int rc = launch_tables(a->A, a->seg_offsets, a->slot_expert, job, st); rc != MOE_OK) return rc;
    const RowMap rm{a->assign_of_row ? ws.tokens : ws.rowlist, nullptr, 1, ws.rowlist, a->topk_w ? a->assign_of_row : nullptr, a->topk_w};
    const Mx4Product p{a->x, a->K, a->K, m, a->y, a->N, a->N, ws.tiles[0], ws.counts, rm,
                       a->topk_w ? ws.gates : nullptr};
    return launch_mx4<kEpiNone>(p, form, a->E, ws.queues, st);
}

extern "C" size_t moe_grouped_ffn_mx4_workspace_bytes(int64_t A, int d, int ffn, int nseg, int dtype) {
    using namespace moegps;
    if (!ffn_shape_in_range(A, d, ffn, nseg, dtype)) return 0;
    return mx4_ws_layout(A, mx4_hidden(ffn), nseg, dtype, nullptr, nullptr);
}

extern "C" int moe_grouped_ffn_mx4(const moe_ffn_mx4_args* a, void* stream) {
    using namespace moegps;
    if (!a) return MOE_ERR_INVALID_ARG;
    return mx4_ffn_call(*a, (hipStream_t)stream, ffn_options(), kFfnAll, nullptr);
}
