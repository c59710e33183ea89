/*
 * simgpu operators -- what an expert-parallel step computes beside the
 * traffic that simgpu.h simulates: attention over a paged key-value cache,
 * 4-bit microscaled tensors and their product, the router with the experts'
 * token lists, the experts' layer for few tokens, all experts or a share of
 * them on one GPU, and the choice of the next token.
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
 * The router with scores, a bias for the choice and groups.  As sim_moe_route,
 * but
 *   score: an expert's score s_e, the softmax over the token's allowed experts
 *     or the sigmoid of its logit (0 where that is -infinity, which is never
 *     chosen), in 32 bits, rounded from 64;
 *   bias: NULL, or [E] f32: experts are chosen by s_e + bias_e, added in 32
 *     bits (by their logits without one, which have the scores' order), ties to
 *     the lowest expert; one whose sum is -infinity is never chosen;
 *   groups: E / groups consecutive experts each (a whole number); of these the
 *     top_groups highest take part (1 <= top_groups <= groups <= 64).  A group
 *     is as high as the highest of its experts (group_best 1), or as the sum in
 *     32 bits of s_e + bias_e of its two highest (2; of one where it has no
 *     second that can be chosen); ties to the lowest group;
 *   weights: the chosen scores, without bias, in 64 bits; with renormalize
 *     divided by their sum; times scale (finite); rounded to 32 bits.
 */
enum { SIM_SCORE_SOFTMAX = 0, SIM_SCORE_SIGMOID = 1 };
#define SIM_MOE_MAX_GROUPS 64
sim_status sim_moe_route_scored(void *hip_stream, const void *logits, int32_t type, int64_t T, int32_t E,
                                int64_t logit_stride, const uint8_t *mask, int64_t mask_stride, int32_t score,
                                const float *bias, int32_t groups, int32_t top_groups, int32_t group_best, int32_t k,
                                int32_t renormalize, float scale, int32_t *experts, float *weights, int32_t *offsets,
                                int32_t *order, void *workspace, size_t workspace_bytes);

/*
 * Gradient of its weights with respect to the logits (the choice has none, nor
 * has the bias), as sim_moe_route_grad; for sigmoid scores at the chosen e
 *   renormalize: w_e (1 - s_e) (g_e - sum g w / scale);  else: w_e (1 - s_e) g_e.
 */
sim_status sim_moe_route_scored_grad(void *hip_stream, const void *logits, int32_t type, int64_t T, int32_t E,
                                     int64_t logit_stride, const uint8_t *mask, int64_t mask_stride, int32_t score,
                                     int32_t k, int32_t renormalize, float scale, const int32_t *experts,
                                     const float *d_weights, void *d_logits);

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

/*
 * The same layer on choices that are given, for a share of the experts: those
 * first .. first + n - 1, whose weights w13 [n, 2 F, D] and w2 [n, D, F] hold:
 *   y_t = sum over the choices j with first <= e = experts[t, j] < first + n of
 *         weights[t, j] W2_e (silu(G_e x_t) * (U_e x_t)).
 *   experts [T, k] i32, any values (an expert twice counts twice); weights
 *   [T, k] f32; 1 <= k <= SIM_MOE_MAX_TOPK, 1 <= n <= SIM_MOE_MAX_EXPERTS.
 * The sum of y over the shares is the layer's result.
 * workspace: sim_moe_experts_workspace bytes, 16-byte aligned.
 */
size_t sim_moe_experts_workspace(int64_t T, int64_t D, int32_t n, int32_t k, int64_t F);
sim_status sim_moe_experts(void *hip_stream, const void *x, int32_t type, int64_t T, int64_t D, int64_t x_stride,
                           const int32_t *experts, const float *weights, int32_t k, int32_t first, int32_t n,
                           const void *w13, const uint8_t *s13, const void *w2, const uint8_t *s2, int32_t weight_type,
                           int64_t F, void *y, int64_t y_stride, void *workspace, size_t workspace_bytes);

/*
 * A paged key-value cache: keys and values are arrays of pages, page p of
 * [kv_heads, page_size, D] elements, contiguous, at p * page_stride elements
 * (the two may be parts of one buffer).  type is F16 or BF16; D a multiple of
 * 8 up to SIM_CACHE_MAX_D; arrays 16-byte aligned, page strides multiples of 8.
 *
 * Write the rows k and v [T, kv_heads, D] of T tokens into it: token t goes to
 * place slots[t] % page_size of page slots[t] / page_size.  A slot outside the
 * cache is skipped, and so is its token.  Tokens must differ in their slots:
 * where two have the same, each 16 bytes that it holds after the call are of
 * one of them.  Strides between tokens and heads count elements; a row of D is
 * contiguous and may lie anywhere its type may, in the cache too where no slot
 * is written, but not where one is.  The pages of keys and those of values must
 * not share memory: arrays that reach into each other have one page stride.
 */
#define SIM_CACHE_MAX_D 256
sim_status sim_cache_append(void *hip_stream, int32_t type, const void *k, int64_t k_stride, int64_t k_head_stride,
                            const void *v, int64_t v_stride, int64_t v_head_stride, int64_t T, int32_t kv_heads, int32_t D,
                            const int64_t *slots, void *k_cache, int64_t k_page_stride, void *v_cache,
                            int64_t v_page_stride, int64_t pages, int32_t page_size);

/*
 * Attention of one new token of each of B sequences over the cache:
 *   out[b, h] = sum over j of p_j V_j,  p = softmax over j of (scale q[b, h] . K_j),
 * K_j and V_j the rows of kv head h / (q_heads / kv_heads) of token j of the
 * sequence: place j % page_size of page table[b, j / page_size], for
 *   max(0, n - window) <= j < n = lengths[b]  (window 0: from 0 on).
 * lengths count the new token where its row is in the cache; below 0 they
 * count as 0, above table_pages * page_size (at most 2^30) as that.  Tokens on
 * a page that is not one of the cache's (-1 say) are left out.  A score of
 * -infinity has no weight; where nothing has any, out is 0.  What other places
 * of the cache hold has no effect.  Scores, weights and sums are in 32 bits (the
 * products' operands: q, K and V as they are, the weights in two parts of type);
 * V are summed before the division, so V whose sum passes 3.4e38 give infinities.
 * An infinity among the V of tokens that are not left out makes the results that
 * it enters infinite or NaN, with a weight of 0 too, and no others.
 *   q, out [B, q_heads, D] of type, out's heads contiguous; kv_heads divides
 *   q_heads; scale up to 2e38; table [B, table_pages] i32; lengths [B] i32;
 *   lse NULL or [B, q_heads] f32: log of the sum over j of e^(scale q . K_j),
 *   -infinity where nothing is left; by it, parts of a sequence that different
 *   calls attend to can be joined.
 * workspace: sim_cache_attention_workspace bytes, 16-byte aligned (NULL if 0).
 */
size_t sim_cache_attention_workspace(int64_t B, int32_t q_heads, int32_t kv_heads, int32_t D, int32_t table_pages,
                                     int32_t page_size, int32_t window);
sim_status sim_cache_attention(void *hip_stream, int32_t type, const void *q, int64_t q_stride, int64_t q_head_stride,
                               int64_t B, int32_t q_heads, int32_t kv_heads, int32_t D, const void *k_cache,
                               int64_t k_page_stride, const void *v_cache, int64_t v_page_stride, int64_t pages,
                               int32_t page_size, const int32_t *table, int64_t table_stride, int32_t table_pages,
                               const int32_t *lengths, float scale, int32_t window, void *out, int64_t out_stride,
                               float *lse, void *workspace, size_t workspace_bytes);

/*
 * The next token of each of B rows of logits [B, V] (F32, F16 or BF16, V <=
 * SIM_SAMPLE_MAX_V), from uniform random numbers u [B] that are given:
 *   w_i = e^((z_i - max z) / temperature); logits in falling order, ties to the
 *     lowest index, i's place in it being its rank;
 *   kept are those with rank < top_k, of these the ones before which the
 *     order's weights sum up to less than top_p times the first top_k's sum,
 *     and of these the ones with w_i >= min_p; the highest always is;
 *   the token is the first kept i, in the order of the indices, up to and with
 *     which the kept weights' sum is above u times the sum of all of them.
 * Weights and sums are in 64 bits, a weight good to 2^-42 of itself, so that only
 * values that close to a border depend on how it is computed; but top_p's sums over more logits than a
 * top_k of 2048 count each weight to the nearest 2^-43 (the highest is 1).  A
 * weight below 2^-1022 is 0, and so is that of a logit more than 3.4e38 below
 * the highest.  A temperature that is not above 0 means
 * the highest logit's first index; top_k below 1 or above V, a top_p of 1 or
 * more or NaN, and a min_p that is not above 0 keep all; a top_p of 0 or less
 * and a min_p above 1 keep the highest.  u below 0 or NaN counts as 0, above 1
 * - 2^-24 as that.  -infinity is never chosen; a row whose highest logit is
 * -infinity, +infinity or NaN gets -1.
 *   temperature, top_k, top_p, min_p: [B] (f32; top_k i32), or NULL for the
 *   same value in all rows, which is given beside it (temperature >= 0, finite;
 *   0 <= top_p <= 1; 0 <= min_p <= 1; not read where there is an array).
 * workspace: sim_sample_workspace bytes, 16-byte aligned (NULL if 0).
 */
#define SIM_SAMPLE_MAX_V (1 << 20)
size_t sim_sample_workspace(int64_t B, int32_t V);
sim_status sim_sample(void *hip_stream, const void *logits, int32_t type, int64_t B, int32_t V, int64_t logit_stride,
                      const float *u, const float *temperature, float all_temperature, const int32_t *top_k, int32_t all_k,
                      const float *top_p, float all_p, const float *min_p, float all_min, int32_t *tokens, void *workspace,
                      size_t workspace_bytes);

/* Text of this thread's last refused or failed operator call ("" if none). */
const char *sim_ops_last_error(void);

#ifdef __cplusplus
}
#endif
#endif /* SIMGPU_OPS_H */
