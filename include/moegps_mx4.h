/*
 * moegps_mx4.h -- experts whose weights are kept in 4 bits: the layer's products with the weights of moegps.h brought to
 * 4.25 bits each, for serving.  Conventions, notation, return codes and data types are those of moegps.h.
 *
 * A decode batch takes as long as the weights of the experts that it touches take to arrive; in 4 bits they are 3.8 times fewer
 * bytes, and so is what a replica of an expert costs.
 */
#ifndef MOEGPS_MX4_H
#define MOEGPS_MX4_H

#include "moegps.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Weights in 4 bits.  MOE_MX4_GROUP neighbours of a column along the dimension that a product sums over (d for W1 and W3, ffn for W2; the
 * last group may be shorter) share a scale 2^(b - 127), b one byte:
 *     b      the smallest with max|w| <= 6 * 2^(b - 127), between 2 and 253; 127 for a group of zeros
 *     codes  e2m1: a sign and one of 0, 0.5, 1, 1.5, 2, 3, 4, 6; w / 2^(b - 127) to the nearest, ties to the one whose last bit is 0.
 *            What would be rounded to 2^128 is held as 3 * 2^126: finite weights stay finite
 * A weight below 3.5 * 2^126 is off by a fifth of itself at most (2.5 held as 2) while it is 2^(b - 127) or more, and by 2^(b - 129) below;
 * one from there up, being held as 3 * 2^126, by a quarter.  What is held, code * 2^(b - 127), is exact in bf16 and in fp32, so packing what
 * moe_unpack_weights_mx4 gives back holds the same values.  Weights that come in such a format from elsewhere are packed from their values
 * without loss where their scales' bytes are 2 to 253 and none is above 3 * 2^126 (bytes of 0 and 1 have values that are no multiples of
 * 2^-126, which are rounded).  A group that holds an infinity or a NaN is all NaN.
 *
 * moe_pack_weights_mx4 brings the weights of an FFN to 4 bits and lays them out for moe_grouped_ffn_mx4:
 *   W1, W3 [E, d, ffn], W2 [E, ffn, d]  dtype in (row-major); W3 NULL: the ReLU form, without a gate matrix
 *   packed  out, moe_packed_weights_mx4_bytes(E, d, ffn, relu) bytes, the same for both data types
 * moe_unpack_weights_mx4 gives the values back, in dtype: the gradient through experts that stay as they are is
 * moe_grouped_ffn_backward with these values packed for it.  An output may be NULL, not wanted (W3 is with relu).
 * moe_pack_matrix_mx4 and moe_unpack_matrix_mx4 do the same with one matrix per expert, W [E, K, N], for moe_grouped_product_mx4.
 * The layout is opaque and the same whatever is packed into it: it does not say which widths or which form it was packed for, and is read
 * with those that it was packed with (other widths may have as many bytes).
 * Limits: 1 <= E <= MOE_MAX_EXPERTS, widths up to 2^22, any of them.  Size queries return 0 outside.
 */
#define MOE_MX4_GROUP 32
size_t moe_packed_weights_mx4_bytes(int E, int d, int ffn, int relu);
int moe_pack_weights_mx4(const void* W1, const void* W3, const void* W2, int dtype, int E, int d, int ffn, void* packed,
                         void* stream);
int moe_unpack_weights_mx4(const void* packed, int E, int d, int ffn, int relu, void* W1, void* W3, void* W2, int dtype,
                           void* stream);
size_t moe_packed_matrix_mx4_bytes(int E, int K, int N);
int moe_pack_matrix_mx4(const void* W, int dtype, int E, int K, int N, void* packed, void* stream);
int moe_unpack_matrix_mx4(const void* packed, int E, int K, int N, void* W, int dtype, void* stream);

/*
 * One matrix per expert, ragged numbers of rows: for every row r of a segment in [seg_begin, seg_end), e = slot_expert of it,
 *     y[r] = g_r * (x_r W_e)
 *   x_r  row r of x [A, K], or with assign_of_row (from moe_permute; NULL: none) row assign_of_row[r] / k of x [rows_x, K]
 *   g_r  topk_w[assign_of_row[r]], in fp32 before the row is rounded; 1 with topk_w NULL.  topk_w goes with assign_of_row
 *   y [A, N] dtype out; rows of other segments and of segments whose slot holds no expert are not written
 *   packed  in, from moe_pack_matrix_mx4 (E experts, K, N)
 *   seg_offsets [nseg + 1], slot_expert [nseg], assign_of_row [A] int32, topk_w [A] float in
 * bf16: exact products, summed in fp32, rounded once.  fp32: the rows are taken as three bf16 parts that add up to them, whose products
 * are summed in fp32.  Sums do not depend on the order of the launch.  Infinities and NaN stay in the rows, and with weights that are NaN
 * the columns, that have them.
 * K and N times the size of dtype must be multiples of 16; A < 2^31; rows of x (A, or rows_x) times K up to 2^31 - 64.
 * Outputs and workspace overlap nothing.  A = 0 is a no-op.
 */
typedef struct moe_product_mx4_args {
    int32_t dtype, K, N, E, nseg, seg_begin, seg_end, k;
    int64_t A, rows_x;   /* rows_x: read with assign_of_row only */
    const void* x;
    const int32_t *assign_of_row, *seg_offsets, *slot_expert;
    const float* topk_w;
    const void* packed;
    void* y;
    void* workspace;
    size_t workspace_bytes;
} moe_product_mx4_args;
size_t moe_grouped_product_mx4_workspace_bytes(int64_t A, int K, int N, int nseg, int dtype);
int moe_grouped_product_mx4(const moe_product_mx4_args* args, void* stream);

/*
 * The experts' FFN of moegps.h with weights in 4 bits: y[r] = g_r * ((silu(x_r W1_e) * (x_r W3_e)) W2_e), or with relu
 * g_r * (max(x_r W1_e, 0) W2_e); max(NaN, 0) is 0.  Rows, gate weights and limits as above with K = N = d, any ffn.
 * bf16: the hidden activation is rounded to bf16 between the products, results once.
 *
 * moe_layer_step_mx4 is moe_layer_step with such weights: `packed` from moe_pack_weights_mx4, workspace_ffn of
 * moe_grouped_ffn_mx4_workspace_bytes(T*k, ...), x_perm NULL (the rows are always gathered, with relu too).
 */
typedef struct moe_ffn_mx4_args {
    int32_t dtype, d, ffn, E, nseg, seg_begin, seg_end, k, relu, reserved; /* reserved: 0 */
    int64_t A, rows_x;
    const void* x;
    const int32_t *assign_of_row, *seg_offsets, *slot_expert;
    const float* topk_w;
    const void* packed;
    void* y;
    void* workspace;
    size_t workspace_bytes;
} moe_ffn_mx4_args;
size_t moe_grouped_ffn_mx4_workspace_bytes(int64_t A, int d, int ffn, int nseg, int dtype);
int moe_grouped_ffn_mx4(const moe_ffn_mx4_args* args, void* stream);
int moe_layer_step_mx4(const moe_layer_step_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOEGPS_MX4_H */
