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
 * moe_combine_backward and moe_grouped_ffn_backward read checkpoints as they are.
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

#ifdef __cplusplus
}
#endif
#endif /* MOEGPS_TRAIN_H */
