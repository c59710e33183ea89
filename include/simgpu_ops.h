/*
 * simgpu operators -- what an expert-parallel step computes beside the
 * traffic that simgpu.h simulates: 4-bit microscaled tensors and their
 * product, the router with the experts' token lists, and the experts' layer
 * for few tokens, all experts on one GPU.
 *
 * C ABI of libsimgpu.so, in the manner of simgpu.h: every call returns a
 * sim_status, no C++ exception crosses the boundary, all array arguments are
 * caller-owned device memory that must stay valid until the stream reaches
 * the work, nothing is allocated and nothing is kept between calls.  Work is
 * enqueued on hip_stream (a hipStream_t; NULL = the null stream) of the
 * current device and the call returns.  Argument errors return synchronously
 * and enqueue nothing; sim_ops_last_error has their text.  Sizes of zero are
 * allowed unless a call says otherwise (nothing is enqueued where nothing is
 * to be written).  Strides count elements.  What a call writes must not overlap
 * what it reads, unless it says otherwise.  The results of a call depend on its
 * arguments only: no atomic whose order changes a result is used.
 */
#ifndef SIMGPU_OPS_H
#define SIMGPU_OPS_H

#include <stddef.h>
#include <stdint.h>

#include "simgpu.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Element types. */
typedef enum { SIM_TYPE_F32 = 0, SIM_TYPE_F16 = 1, SIM_TYPE_BF16 = 2, SIM_TYPE_MX4 = 3 } sim_type;

/*
 * A 4-bit microscaled matrix of R rows and K columns.  Each block of 32
 * columns of a row shares one 8-bit scale; element i stands for q_i 2^s with
 *   s   = max(floor(log2 max|x|) - 2, -127) of the block (-127 if all zero),
 *         stored as the byte s + 127;
 *   q_i = x_i 2^-s rounded to the nearest of 0, .5, 1, 1.5, 2, 3, 4, 6 with
 *         its sign, halfway cases to the even code, at most 6 in magnitude,
 *         stored as sign << 3 | code.
 * A block that holds a NaN or an infinity gets the scale byte 255 and codes
 * 0; all its elements stand for NaN.
 *   codes  [R, sim_mx4_code_pitch(K)]  = ceil(K / 256) * 128 bytes a row, the
 *          even element in the low four bits;
 *   scales [R, sim_mx4_scale_pitch(K)] = ceil(K / 256) * 8 bytes a row.
 * Codes and scales past column K are 0.  Codes are 16-byte, scales 8-byte
 * aligned, as any run of whole rows is.
 */
int64_t sim_mx4_code_pitch(int64_t K);
int64_t sim_mx4_scale_pitch(int64_t K);

/*
 * Put x into 4 bits.  x: rows x cols of type (not SIM_TYPE_MX4), row_stride
 * >= cols elements from one row to the next.  transpose = 0: the result has
 * rows rows, blocks along the columns; 1: it is the transpose of x (cols
 * rows, blocks along the rows of x).  Codes and scales are written whole,
 * padding included.
 */
sim_status sim_mx4_quantize(void *hip_stream, const void *x, int32_t type, int64_t rows, int64_t cols,
                            int64_t row_stride, int32_t transpose, uint8_t *codes, uint8_t *scales);

/* out[r, c] = the value that element (r, c) stands for, rounded to type. */
sim_status sim_mx4_dequantize(void *hip_stream, const uint8_t *codes, const uint8_t *scales, int64_t rows,
                              int64_t cols, void *out, int32_t type, int64_t row_stride);

/*
 * out[m, n] = sum over k of A[m, k] B[n, k], A: M x K, B: N x K, both in 4
 * bits; summed in 32 bits and rounded once to type.  K = 0 gives zeros.
 */
sim_status sim_mx4_matmul(void *hip_stream, const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes,
                          const uint8_t *b_scales, int64_t M, int64_t N, int64_t K, void *out, int32_t type,
                          int64_t row_stride);

/*
 * The same product of x (M x K of x_type, put into 4 bits on the way exactly
 * as sim_mx4_quantize does) with a 4-bit W (N x K): a linear layer.
 * workspace: sim_mx4_linear_workspace bytes, 16-byte aligned (NULL if 0).
 */
size_t sim_mx4_linear_workspace(int64_t M, int64_t N, int64_t K);
sim_status sim_mx4_linear(void *hip_stream, const void *x, int32_t x_type, int64_t x_stride, const uint8_t *w_codes,
                          const uint8_t *w_scales, int64_t M, int64_t N, int64_t K, void *out, int32_t type,
                          int64_t row_stride, void *workspace, size_t workspace_bytes);

/*
 * Gradients of that layer, Y = X W^T, where rounding to 4 bits passes
 * gradients through: dX = dY W and dW = dY^T X, each of the four operands put
 * into 4 bits along the axis that is summed over.  dY [M, N], X [M, K], W
 * [N, K], dX and dW of one type, with row strides; dX or dW may be NULL (not
 * wanted).  workspace: sim_mx4_linear_grad_workspace bytes, 16-byte aligned.
 */
size_t sim_mx4_linear_grad_workspace(int64_t M, int64_t N, int64_t K);
sim_status sim_mx4_linear_grad(void *hip_stream, int32_t type, const void *dy, int64_t dy_stride, const void *x,
                               int64_t x_stride, const void *w, int64_t w_stride, int64_t M, int64_t N, int64_t K, void *dx,
                               int64_t dx_stride, void *dw, int64_t dw_stride, void *workspace, size_t workspace_bytes);

#define SIM_MOE_MAX_EXPERTS 1024
#define SIM_MOE_MAX_TOPK 32
#define SIM_MOE_LAYER_MAX_TOKENS 1024

/*
 * Router: for each of T tokens the k experts with the highest logits.
 *   logits [T, E] of type (F32, F16, BF16), row stride logit_stride;
 *   mask   NULL, or bytes [E] with mask_stride 0 (one for all tokens), or
 *          [T, E] with row stride mask_stride: an expert is allowed where
 *          the byte is not 0.  What logits hold elsewhere has no effect;
 *   1 <= k <= min(E, SIM_MOE_MAX_TOPK), E <= SIM_MOE_MAX_EXPERTS,
 *   T k < 2^31.
 * Choices are in falling order of the logits, ties to the lowest expert, a
 * NaN above every number; -infinity is never chosen.  The weights are the
 * softmax over the token's allowed experts, in 32 bits, with renormalize
 * divided by their sum over the chosen ones.  A NaN or +infinity among the
 * allowed logits makes the token's weights what the formula gives (NaN).
 * Where fewer than k can be chosen, the rest are expert -1 with weight 0.
 *   experts [T, k] i32, weights [T, k] f32;
 *   offsets [E + 1] i32: slots (token k + choice) of the experts before e;
 *   order   [T, k] i32: the slots sorted by expert, then by slot; -1 past
 *           offsets[E].
 * offsets and order may both be NULL.  workspace: sim_moe_route_workspace
 * bytes, 16-byte aligned (NULL if 0).
 */
size_t sim_moe_route_workspace(int64_t T, int32_t E, int32_t k);
sim_status sim_moe_route(void *hip_stream, const void *logits, int32_t type, int64_t T, int32_t E,
                         int64_t logit_stride, const uint8_t *mask, int64_t mask_stride, int32_t k,
                         int32_t renormalize, int32_t *experts, float *weights, int32_t *offsets, int32_t *order,
                         void *workspace, size_t workspace_bytes);

/*
 * Gradient of the weights with respect to the logits: d_logits [T, E] of
 * type, contiguous, from d_weights [T, k] f32 and the experts that
 * sim_moe_route chose for the same logits, mask, k and renormalize.
 *   renormalize: w_e (g_e - sum g w) at the chosen experts, 0 elsewhere;
 *   else:        p_e ([e chosen] g_e - sum g p) at every allowed expert.
 * Masked experts and choices of -1 get and give no gradient.
 */
sim_status sim_moe_route_grad(void *hip_stream, const void *logits, int32_t type, int64_t T, int32_t E,
                              int64_t logit_stride, const uint8_t *mask, int64_t mask_stride, int32_t k,
                              int32_t renormalize, const int32_t *experts, const float *d_weights, void *d_logits);

/*
 * The experts' layer for few tokens, from the router's logits:
 *   y_t = sum over the chosen experts e of  w_te W2_e (silu(G_e x_t) * (U_e x_t))
 * with experts chosen as by sim_moe_route, and its weights to within a few
 * units in the last place (for few tokens a kernel of its own computes them,
 * in another order).  The sum runs over all E experts that are routed to, so
 * the call needs the weights of all of them.
 *   x [T, D], y [T, D] of type (F16 or BF16), row strides x_stride, y_stride;
 *   w13 [E, 2 F, D]: the F rows of G_e, then the F rows of U_e; w2 [E, D, F];
 *   weight_type: type (both contiguous, s13 = s2 = NULL), or SIM_TYPE_MX4
 *   (codes in w13, w2 and scales in s13, s2, of E 2 F x D and E D x F);
 *   T <= SIM_MOE_LAYER_MAX_TOKENS.
 * Sums, softmax, silu and the weights are in 32 bits; what passes between
 * the two products is kept to 16 significant bits, in two parts; y is rounded
 * once.  An infinity among a token's x or its experts' weights makes the
 * results that it enters infinite or NaN, and no others.  A token without
 * experts gets zeros.  y may be x: it is written once x has been read.
 * workspace: sim_moe_layer_workspace bytes, 16-byte aligned.
 */
size_t sim_moe_layer_workspace(int64_t T, int64_t D, int32_t E, int32_t k, int64_t F);
sim_status sim_moe_layer(void *hip_stream, const void *x, int32_t type, int64_t T, int64_t D, int64_t x_stride,
                         const void *logits, int32_t logit_type, int32_t E, int64_t logit_stride,
                         const uint8_t *mask, int64_t mask_stride, int32_t k, int32_t renormalize, const void *w13,
                         const uint8_t *s13, const void *w2, const uint8_t *s2, int32_t weight_type, int64_t F,
                         void *y, int64_t y_stride, void *workspace, size_t workspace_bytes);

/* Text of this thread's last refused or failed operator call ("" if none). */
const char *sim_ops_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SIMGPU_OPS_H */
