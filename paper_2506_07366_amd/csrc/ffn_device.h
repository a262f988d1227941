// What the kernels of the grouped FFN share (grouped_ffn.hip, ffn_backward.hip): the packed form of the weights,
// waits and register-to-register helpers, where the rows of a product live, the pieces of the row copy.
#pragma once
#include "ffn_tables.h"
#include <atomic>
#include <type_traits>
#include <utility>

namespace moegps {

typedef __attribute__((__vector_size__(8 * sizeof(__bf16)))) __bf16 bf16x8;
typedef __attribute__((__vector_size__(4 * sizeof(float)))) float f32x4;
typedef f32x4 __attribute__((aligned(4))) f32x4_any;  // four floats at any float's address, still one access
typedef unsigned short bf16_t;  // storage

// The packed form of a weight matrix is what the GEMM's loads want to find: the transposed
// matrix W^T [N_out][K_out] cut into tiles of kPackN rows by kPackK columns, tiles of one
// row block side by side along K, every tile 32 KiB in one piece.  Inside a tile the matrix is
// stored by MFMA fragment: the 16 rows x 32 columns one v_mfma_f32_16x16x32_bf16 takes are
// 1 KiB in one piece, in lane order (lane 16*q + r holds row r, columns 8q .. 8q+7), the two
// fragments of a 16-row group along K side by side.  So
//   - a k-tile of a weight panel is one contiguous read instead of 256 pieces of 128 bytes a row
//     apart, which the memory system serves a quarter slower at some row lengths (8 KiB among
//     them);
//   - a fragment is loaded into registers as one contiguous kilobyte, without a detour through LDS.
constexpr int kPackN = 256, kPackK = 64;
constexpr int kFragElems = 16 * 32;  // one MFMA operand fragment
__host__ __device__ inline size_t packed_index(int n, int k, int K_out) {
    const int row = n % kPackN, kk = k % kPackK;
    const size_t tile = (size_t)(n / kPackN) * (K_out / kPackK) + k / kPackK;
    const int frag = (row >> 4) * (kPackK / 32) + (kk >> 5);
    return tile * (kPackN * kPackK) + frag * kFragElems + (((kk >> 3) & 3) * 16 + (row & 15)) * 8 + (kk & 7);
}
// Activation tiles keep rows of 128 bytes in LDS: 16-byte piece `slot` of LDS row `row` holds
// piece slot ^ swz(row) of the row.  The LDS
// has 64 four-byte banks and serves a ds_read_b128 sixteen lanes at a time, so the
// 16 consecutive rows one such group touches must land on 16 distinct 16-byte bank
// groups of a 256-byte span: with 128-byte rows that is (row&1, slot) -> xor with
// (row>>1)&7.
__host__ __device__ inline int swz(int row) { return (row >> 1) & 7; }

// s_waitcnt with only vmcnt set (gfx9 encoding: vmcnt[3:0] | expcnt[6:4] | lgkmcnt[11:8] | vmcnt[15:14])
template <int N>
__device__ __forceinline__ void wait_vmcnt() {
    static_assert(N >= 0 && N < 64, "vmcnt range");
    __builtin_amdgcn_s_waitcnt((N & 0xf) | (0x7 << 4) | (0xf << 8) | ((N >> 4) << 14));
}

// compile-time loop: f(integral_constant<int, 0>) ... f(integral_constant<int, N-1>)
template <int... I, class F>
__device__ __forceinline__ void static_for_impl(std::integer_sequence<int, I...>, F&& f) {
    (f(std::integral_constant<int, I>{}), ...);
}
template <int N, class F>
__device__ __forceinline__ void static_for(F&& f) {
    static_for_impl(std::make_integer_sequence<int, N>{}, f);
}

// LDS fragment read issued as an instruction of its own: the compiler does not track
// when the data lands, the kernel waits with lds_wait<N>() ("at most N LDS reads of
// this wavefront still in flight"; LDS reads complete in issue order) and then ties
// the destination registers with lds_landed() before they are used.
template <int OFF>
__device__ __forceinline__ void lds_read_b128(bf16x8& dst, unsigned addr) {
    asm volatile("ds_read_b128 %0, %1 offset:%2" : "=v"(dst) : "v"(addr), "n"(OFF) : "memory");
}
template <int N>
__device__ __forceinline__ void lds_wait() {
    static_assert(N >= 0 && N < 16, "lgkmcnt range");
    __builtin_amdgcn_s_waitcnt(0xc07f | (N << 8));  // vmcnt and expcnt untouched
}
__device__ __forceinline__ void lds_landed(bf16x8& v) { asm volatile("" : "+v"(v)); }

// A copy of a lane-dependent value that the compiler cannot trace back: what is computed
// from it is computed where it is used (per tile) instead of once per kernel and then kept
// in a register, or in scratch memory, across the K loop.
__device__ __forceinline__ int opaque(int v) {
    asm volatile("" : "+v"(v));
    return v;
}
// the same for a value that is uniform over the wavefront (scalar register)
__device__ __forceinline__ int opaque_uniform(int v) {
    asm volatile("" : "+s"(v));
    return v;
}

// With the wavefront seen as four quarters of 16 lanes, p = [p0 p1 p2 p3] and q = [q0 q1 q2 q3]
// become p = [p0 p2 q0 q2] and q = [p1 p3 q1 q3] (two register-to-register swap instructions).
__device__ __forceinline__ void lane_swap_pairs(unsigned& p, unsigned& q) {
    auto r = __builtin_amdgcn_permlane32_swap(p, q, false, false);  // p: [p0 p1 q0 q1], q: [p2 p3 q2 q3]
    auto t = __builtin_amdgcn_permlane16_swap(r[0], r[1], false, false);
    p = t[0];
    q = t[1];
}

// two floats rounded to bf16 (nearest even) and packed, low half first: one conversion instruction
__device__ __forceinline__ unsigned pack_bf16x2(float lo, float hi) {
    typedef __attribute__((__vector_size__(2 * sizeof(float)))) float f32x2;
    typedef __attribute__((__vector_size__(2 * sizeof(__bf16)))) __bf16 bf16x2;
    const f32x2 v = {lo, hi};
    return __builtin_bit_cast(unsigned, __builtin_convertvector(v, bf16x2));
}

// silu(g) = g / (1 + exp(-g)) with the hardware reciprocal (1 ulp) and the hardware
// exponential in place of an IEEE division and expf; the result is rounded to bf16 right after.
__device__ __forceinline__ float silu_f(float g) { return g * __builtin_amdgcn_rcpf(1.0f + __expf(-g)); }

// EPI selects what happens to the accumulators before they are stored: kEpiNone (plain
// product, optionally scaled per row), kEpiSwiglu (silu(gate) * up on interleaved column
// pairs, half as many output columns), kEpiRelu (max(., 0)); in the backward pass (ffn_backward.hip)
// kEpiFloat (plain product in place, not rounded) and kEpiSwigluGrad and kEpiReluGrad (the hidden activation and the
// gradients of what it is made of, from the gradient of the hidden activation).
constexpr int kEpiNone = 0, kEpiSwiglu = 1, kEpiRelu = 2, kEpiSwigluGrad = 3, kEpiReluGrad = 4, kEpiFloat = 5;
// the first products of the forward pass take a share of the row copy along
constexpr bool epi_copies(int epi) { return epi == kEpiSwiglu || epi == kEpiRelu; }

// Where the rows of a product live.  List position p of an M-tile is
//   operand row  a_rows ? a_rows[p] : p, and then, with a_rows2, a_rows2[that] / a_div
//                (the first product reads x_perm through the row list, or rows of x through the list
//                of their tokens, or through the row list and assign_of_row);
//   output row   c_rows ? c_rows[p] : p  (the second product writes y_perm through the row list);
//   output scale scale ? scale[scale_idx[output row]] : 1  (gate weight of the row's assignment).
struct RowMap {
    const int32_t* a_rows;
    const int32_t* a_rows2;
    int a_div;
    const int32_t* c_rows;
    const int32_t* scale_idx;
    const float* scale;
};

// A wavefront's share of the row copy that goes with the first product.
__device__ __forceinline__ void copy_part(const RowCopy& copy, int wv) {
    if (copy.chunks >= 4 * kWave) copy_rows<4>(copy, wv);
    else copy_rows<1>(copy, wv);
}

// n pieces of the row copy (row_copy.h) from number `first` on, and the rows they go to, asked for by a wavefront into
// its LDS at `lds`, kCopyPieceLds bytes each (a piece's bytes past the end of its row and destinations past the k-th come as
// zeros, out of the buffers' ranges) ...
constexpr int kCopyPieceLds = kCopyPieceBytes + kWave * 4;
__device__ __forceinline__ void request_pieces(const RowCopy& c, int first, int n, unsigned char* lds) {
    const unsigned lane = threadIdx.x & (kWave - 1);
    const int per_row = ceil_div(c.chunks, kWave);
    int t = first / per_row, q = first - t * per_row;
    for (int i = 0; i < n; ++i) {
        const auto row = __builtin_amdgcn_make_buffer_rsrc((void*)(c.x + (size_t)t * c.chunks + q * kWave), 0,
                                                           (c.chunks - q * kWave) * 16, 0x00027000);
        const auto ids = __builtin_amdgcn_make_buffer_rsrc((void*)(c.row_of_assign + (size_t)t * c.k), 0, c.k * 4, 0x00027000);
        unsigned char* at = lds + i * kCopyPieceLds;
        __builtin_amdgcn_raw_ptr_buffer_load_lds(row, (__attribute__((address_space(3))) void*)at, 16, lane * 16, 0, 0, 0);
        __builtin_amdgcn_raw_ptr_buffer_load_lds(ids, (__attribute__((address_space(3))) void*)(at + kCopyPieceBytes), 4,
                                                 lane * 4, 0, 0, 0);
        if (++q == per_row) {
            q = 0;
            ++t;
        }
    }
}

// ... and, once they have landed (LDS address `at`), stored to these rows, which nothing in the call reads: past the caches.
__device__ __forceinline__ void store_pieces(const RowCopy& c, int first, int n, unsigned at) {
    typedef __attribute__((__vector_size__(4 * sizeof(unsigned)))) unsigned u32x4;
    const int lane = opaque((int)threadIdx.x) & (kWave - 1);
    const int per_row = ceil_div(c.chunks, kWave);
    int q = first % per_row;
    for (int i = 0; i < n; ++i, at += kCopyPieceLds) {
        bf16x8 v;
        int row;
        lds_read_b128<0>(v, at + lane * 16);
        asm volatile("ds_read_b32 %0, %1 offset:%2" : "=v"(row) : "v"(at + lane * 4), "n"(kCopyPieceBytes) : "memory");
        lds_wait<0>();
        lds_landed(v);
        asm volatile("" : "+v"(row));
        u32x4* dst = (u32x4*)c.x_perm + q * kWave + lane;
        if (q * kWave + lane < c.chunks)
            for (int j = 0; j < c.k; ++j)
                __builtin_nontemporal_store(__builtin_bit_cast(u32x4, v),
                                            dst + (size_t)__builtin_amdgcn_readlane(row, j) * c.chunks);
        if (++q == per_row) q = 0;
    }
}

// ---------------------------------------------------------------------------
// host side: what the forward and the backward pass share
// ---------------------------------------------------------------------------
// The bf16 kernels work on a hidden width padded to a multiple of 64: the packed weights
// carry zero columns (W1, W3) and zero rows (W2) for the padding, so the padded hidden
// activations are exact zeros and add nothing to the second product.
// Widths above this are refused: it keeps every size computed on the host inside 64 bits and
// every tile offset computed on the device inside 32.
constexpr int kMaxWidth = 1 << 22;
inline bool ffn_shape_in_range(int64_t A, int d, int ffn, int nseg, int dtype) {
    return (dtype == MOE_DTYPE_F32 || dtype == MOE_DTYPE_BF16) && A >= 0 && A < (1ll << 31) && d >= 1 &&
           d <= kMaxWidth && ffn >= 1 && ffn <= kMaxWidth && nseg >= 1 && nseg <= MOE_MAX_SEGMENTS;
}

inline int padded_ffn(int ffn, int dtype) {
    return dtype == MOE_DTYPE_BF16 ? (int)align_up((size_t)ffn, 64) : ffn;
}
// rows of a packed bf16 weight matrix: whole tiles
inline size_t packed_rows(size_t n) { return align_up(n, (size_t)kPackN); }
// elements of one expert's packed matrices: the first product's n1 matrices, the second product's
inline size_t packed_elems1(int n1, int d, int fp) { return packed_rows((size_t)n1 * fp) * d; }
inline size_t packed_elems2(int d, int fp) { return packed_rows((size_t)d) * fp; }

constexpr int kMinBM = 32;  // the lowest tile shape

// A kernel that uses more LDS than the default limit: raised once per kernel (`raised`: bit per device).
int raise_lds(const void* kern, size_t bytes, std::atomic<unsigned long long>& raised);
// Weights of a product that tiles read past the caches where they share them with no other tile.
bool past_caches(int E, size_t b_stride);
// The table builder as a launch of its own, for A rows.
int launch_tables(int64_t A, const int32_t* seg_offsets, const int32_t* slot_expert, const TableJob& job, hipStream_t st);
// A plain product by tiles: C[c_rows[p], 0 .. N) = A[a_rows[p], 0 .. K) x packed weights, for the rows of a table.
int launch_product(const bf16_t* A, int lda, const bf16_t* Bp, size_t b_stride, int E, bf16_t* C, int ldc,
                   const MTile* tiles, const int32_t* counts, int32_t* queues, int N, int K, const RowMap& rm,
                   hipStream_t st);

}  // namespace moegps
