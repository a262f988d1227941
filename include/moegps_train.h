/*
 * moegps_train.h -- training calls of libmoegps: the gradients of the layer that moegps.h runs forward, and
 * activations kept in 8 bits between the two passes.
 *
 * A training step is moe_layer_step (or the six calls) forward, checkpoints of what the backward pass reads (x, and the
 * rows y_perm that moe_combine adds up), and then, from the gradient dout of the layer's output,
 *     moe_combine_backward      dy_perm, and the gradients of the gate weights and of the router logits
 *     moe_grouped_ffn_backward  dx_perm, and the gradients of the expert weights
 *     moe_combine               dx from dx_perm, without weights
 * The plan, a choice of where rows are computed, has no gradient.  Conventions, notation, return codes and data types are
 * those of moegps.h.
 */
#ifndef MOEGPS_TRAIN_H
#define MOEGPS_TRAIN_H

#include "moegps.h"

#ifdef __cplusplus
extern "C" {
#endif

/*
 * Activation checkpoints: rows kept in 8 bits between the forward and the backward pass.  Every MOE_CHECKPOINT_GROUP
 * values of a row (the last group may be shorter) share a scale 2^(b - 127), b one byte:
 *     b      the smallest with max|x| <= 448 * 2^(b - 127), 1 at least; 127 for a group of zeros
 *     codes  e4m3 (4 exponent bits, bias 7, 3 mantissa bits, largest 448, no infinity), x / 2^(b - 127)
 *            to nearest even: within 2^-4 of a value, or 2^-10 of the scale for values below 2^-6 of it.
 *            What would be rounded to 2^128 is held as 240 * 2^120: finite values come back finite
 * moe_checkpoint_load gives code * 2^(b - 127), exact also in bf16 (but for results below its normal range).  Infinite
 * values and NaN come back as NaN and do not touch the scale.
 *   x [rows, d] dtype;  codes [rows, d], scales [rows, ceil(d / MOE_CHECKPOINT_GROUP)] bytes
 * moe_combine_backward and moe_grouped_ffn_backward read checkpoints as they are.  What that costs gradients, of their norm, for
 * normal inputs (a kept value is off by 2.5 %, rms): dtopk_w 2.5 %; from x, with SwiGLU dx 3 %, dW1 4 to 5 %, dW3 and dW2 4 %, with ReLU
 * dx and dW1 13 % (sums that the error moves through 0), dW2 2.7 %.
 * d * sizeof(dtype) must be a multiple of 16, d <= 2^22, rows < 2^31.  rows = 0 is a no-op.
 */
#define MOE_CHECKPOINT_GROUP 32
int moe_checkpoint_store(const void* x, int dtype, int64_t rows, int d, uint8_t* codes, uint8_t* scales, void* stream);
int moe_checkpoint_load(const uint8_t* codes, const uint8_t* scales, int64_t rows, int d, void* x, int dtype,
                        void* stream);

/*
 * Gradient of the way back from the experts and of the gate: with
 *     out[t, :] = sum_{j<k} topk_w[t, j] * y_perm[row_of_assign[t*k + j], :]   (moe_combine)
 * and the gradient dout of out,
 *     dy_perm[row_of_assign[t*k + j], :] = topk_w[t, j] * dout[t, :]
 *     dtopk_w[t, j]                      = sum_i dout[t, i] * y_perm[row_of_assign[t*k + j], i]
 *     dlogits[t, e] = topk_w[t, j] * (dtopk_w[t, j] - sum_i topk_w[t, i] * dtopk_w[t, i])   for e = topk_idx[t, j],
 *                     0 for the experts that were not selected (moe_route_topk: softmax over the k selected logits)
 * The gradient of the way there, of moe_permute's row copy, is moe_combine of dx_perm with topk_w = NULL:
 * dx[t, :] = sum_j dx_perm[row_of_assign[t*k + j], :].
 *   dout [T, d], dy_perm [A, d] dtype, in and out;  row_of_assign [A] int32, topk_w [T, k] float in
 *   y_perm    [A, d] in: dtype, or with y_scales the codes of a checkpoint of it (moe_checkpoint_store).  NULL: only
 *             dy_perm is wanted (dtopk_w and dlogits NULL too)
 *   dtopk_w   [T, k] float out
 *   dlogits   [T, E] float out, written whole; may be NULL (topk_idx is then not read).  topk_idx [T, k] int32 in, distinct ids
 * dy_perm may be y_perm (in dtype): a value is read before its place is written.  Otherwise outputs overlap nothing.
 * The products are taken and summed in fp32; dy_perm is rounded once.  Sums do not depend on the order of the launch.
 * d * sizeof(dtype) must be a multiple of 16.  T = 0 is a no-op.
 */
int moe_combine_backward(const void* dout, int dtype, int T, int d, int k, int E, const int32_t* row_of_assign,
                         const float* topk_w, const int32_t* topk_idx, const void* y_perm, const uint8_t* y_scales,
                         void* dy_perm, float* dtopk_w, float* dlogits, void* stream);

/*
 * Gradient of the grouped expert FFN (moe_grouped_ffn and its forms; relu: moe_grouped_ffn_relu).  For every row r of a
 * segment, with e = slot_expert of it, x_r = x[assign_of_row[r] / k] and dy_r = dy_perm[r]:
 *     a = x_r W1_e, b = x_r W3_e, s = 1 / (1 + exp(-a)), h = a s b       relu: h = max(a, 0)
 *     dh = dy_r W2_e^T,  da = dh b s (1 + a (1 - s)),  db = dh a s       relu: da = dh where a > 0, else 0
 *     dx_perm[r] = da W1_e^T + db W3_e^T                                 relu: da W1_e^T
 *     dW1_e = sum_r x_r^T da,  dW3_e = sum_r x_r^T db,  dW2_e = sum_r h^T dy_r
 * over all rows of the expert, its replicas' among them.  The hidden activations are worked out again from x, so the forward
 * pass keeps nothing but x.
 *   x          [T, d] dtype in, or with x_scales the codes of a checkpoint of it (moe_checkpoint_store)
 *   assign_of_row [T*k], seg_offsets [nseg + 1], slot_expert [nseg] int32 in, as in the forward pass
 *   packed     in, from moe_pack_weights (relu: moe_pack_weights_relu)
 *   packed_backward  in, from moe_pack_weights_backward; not read with MOE_DTYPE_F32
 *   dy_perm    [T*k, d] dtype in
 *   dx_perm    [T*k, d] dtype out, rows of segments whose slot holds no expert are not written; NULL: not wanted
 *   dW1, dW3 [E, d, ffn], dW2 [E, ffn, d] dtype out, written whole (zeros for experts without rows); NULL, all of them: not
 *              wanted.  dW3 is NULL with relu
 * Infinities and NaN reach dx_perm of the rows that have them and the weight gradients of these rows' experts, nothing else;
 * with relu a sum a that is NaN counts as 0 (h = da = 0), as in the forward pass.
 * bf16: sums in fp32; h, da and db are rounded to bf16 as operands of the next products, results once.  The result does
 * not depend on the order in which parts of the launch run.  Outputs and workspace overlap nothing.
 * bf16 needs d % 64 == 0 and T*k*d < 2^31, and for dx_perm ffn <= 2^21 (relu: below 2^22), f32 d % 4 == 0 and ffn % 4 == 0;
 * limits otherwise as in the forward pass.
 * T = 0 writes zeros to the weight gradients.  Arguments are checked before the first launch.
 *
 * moe_pack_weights_backward lays the weights out for the products with transposed weights, like moe_pack_weights whenever they have
 * changed (W3 NULL: the ReLU form): 1.27 ms for 8 experts of 4096 x 14336, beside 1.19 for the forward pass's layout.  Nothing to do
 * for MOE_DTYPE_F32, whose size is 0.
 */
typedef struct moe_ffn_backward_args {
    int32_t dtype, T, k, d, ffn, E, nseg, relu;
    const void* x;
    const uint8_t* x_scales;
    const int32_t *assign_of_row, *seg_offsets, *slot_expert;
    const void *packed, *packed_backward;
    const void* dy_perm;
    void *dx_perm, *dW1, *dW3, *dW2;
    void* workspace;
    size_t workspace_bytes;
} moe_ffn_backward_args;
size_t moe_packed_weights_backward_bytes(int E, int d, int ffn, int dtype, int relu);
int moe_pack_weights_backward(const void* W1, const void* W3, const void* W2, int dtype, int E, int d, int ffn,
                              void* packed, void* stream);
size_t moe_grouped_ffn_backward_workspace_bytes(int T, int k, int d, int ffn, int E, int nseg, int dtype, int relu);
int moe_grouped_ffn_backward(const moe_ffn_backward_args* args, void* stream);

#ifdef __cplusplus
}
#endif
#endif /* MOEGPS_TRAIN_H */
