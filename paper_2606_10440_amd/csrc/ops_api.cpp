// C entry points of the operators: every argument is checked here, before
// anything is enqueued; the launchers rely on what passed.
#include <algorithm>
#include <cmath>
#include <string>

#include "ops_common.h"

using namespace simops;

namespace {

thread_local char g_error[160] = "";

sim_status refuse(sim_status s, const char *call, const char *why) {
    snprintf(g_error, sizeof g_error, "%s: %s", call, why);
    return s;
}
sim_status done(sim_status s, const char *call) {
    if (s == SIM_OK) {
        g_error[0] = 0;
        return s;
    }
    return refuse(s, call, "the launch failed");
}

// Sizes up to which every index the kernels form, and every grid, fits.
constexpr int64_t kMaxDim = (int64_t)1 << 31;
constexpr int64_t kMaxElems = (int64_t)1 << 35;
constexpr int64_t kMaxTokens = (int64_t)1 << 27;
constexpr int64_t kMaxLayerTiles = (int64_t)1 << 23;

bool is_float(int t) { return t == SIM_TYPE_F32 || t == SIM_TYPE_F16 || t == SIM_TYPE_BF16; }
size_t size_of(int t) { return t == SIM_TYPE_F32 ? 4 : 2; }
bool aligned_to(const void *p, size_t n) { return (uintptr_t)p % n == 0; }
bool dims_ok(int64_t rows, int64_t cols) {
    return rows >= 0 && cols >= 0 && rows < kMaxDim && cols < kMaxDim && (cols == 0 || rows <= kMaxElems / (groups_of(cols) * kGroup));
}

// What the calls take and their workspace queries, which give 0 for what is refused.
bool linear_fits(int64_t M, int64_t N, int64_t K) { return dims_ok(M, N) && dims_ok(N, M) && dims_ok(M, K) && dims_ok(N, K); }
bool linear_grad_fits(int64_t M, int64_t N, int64_t K) { return linear_fits(M, N, K) && dims_ok(K, M) && dims_ok(K, N); }
bool layer_dims_fit(int64_t D, int64_t F) { return D < ((int64_t)1 << 20) && F < ((int64_t)1 << 20); }
bool layer_tiles_fit(int64_t T, int64_t D, int32_t E, int32_t k, int64_t F) {
    return std::min<int64_t>(E, T * k) * (std::max(D, F) / 16 + 1) <= kMaxLayerTiles;
}

#define NEED(cond, why) \
    do { \
        if (!(cond)) return refuse(SIM_ERR_INVALID_ARG, __func__, why); \
    } while (0)
#define FITS(cond, why) \
    do { \
        if (!(cond)) return refuse(SIM_ERR_SIZE, __func__, why); \
    } while (0)

// what the route's three users check alike
const char *route_bad(const void *logits, int32_t type, int64_t T, int32_t E, int64_t stride, const uint8_t *mask,
                      int64_t mask_stride, int32_t k) {
    if (!is_float(type)) return "logits must be f32, f16 or bf16";
    if (T < 0) return "negative token count";
    if (E < 1 || E > SIM_MOE_MAX_EXPERTS) return "expert count out of range";
    if (k < 1 || k > E || k > SIM_MOE_MAX_TOPK) return "k out of range";
    if (T > 0 && !logits) return "null logits";
    if (!aligned_to(logits, size_of(type))) return "logits not aligned to their type";
    if (T > 1 && stride < E) return "logit stride below the expert count";
    if (mask && mask_stride != 0 && T > 1 && mask_stride < E) return "mask stride below the expert count";
    return nullptr;
}

}  // namespace

extern "C" {

const char *sim_ops_last_error(void) { return g_error; }

int64_t sim_mx4_code_pitch(int64_t K) { return K > 0 ? groups_of(K) * kGroupCodes : 0; }
int64_t sim_mx4_scale_pitch(int64_t K) { return K > 0 ? groups_of(K) * kGroupScales : 0; }

sim_status sim_mx4_quantize(void *stream, const void *x, int32_t type, int64_t rows, int64_t cols, int64_t row_stride,
                            int32_t transpose, uint8_t *codes, uint8_t *scales) {
    NEED(is_float(type), "x must be f32, f16 or bf16");
    NEED(rows >= 0 && cols >= 0, "negative size");
    FITS(dims_ok(rows, cols) && dims_ok(cols, rows), "matrix too large");
    NEED(transpose == 0 || transpose == 1, "transpose must be 0 or 1");
    if (rows == 0 || cols == 0) return done(SIM_OK, __func__);
    NEED(x && codes && scales, "null array");
    NEED(rows == 1 || row_stride >= cols, "row stride below the row length");
    NEED(aligned_to(x, size_of(type)), "x not aligned to its type");
    NEED(aligned_to(codes, 16) && aligned_to(scales, 8), "codes must be 16-byte, scales 8-byte aligned");
    return done(launch_quantize((hipStream_t)stream, x, type, rows, cols, row_stride, transpose, codes, scales), __func__);
}

sim_status sim_mx4_dequantize(void *stream, const uint8_t *codes, const uint8_t *scales, int64_t rows, int64_t cols,
                              void *out, int32_t type, int64_t row_stride) {
    NEED(is_float(type), "out must be f32, f16 or bf16");
    NEED(rows >= 0 && cols >= 0, "negative size");
    FITS(dims_ok(rows, cols), "matrix too large");
    if (rows == 0 || cols == 0) return done(SIM_OK, __func__);
    NEED(codes && scales && out, "null array");
    NEED(rows == 1 || row_stride >= cols, "row stride below the row length");
    NEED(aligned_to(out, size_of(type)), "out not aligned to its type");
    NEED(aligned_to(codes, 16) && aligned_to(scales, 8), "codes must be 16-byte, scales 8-byte aligned");
    return done(launch_dequantize((hipStream_t)stream, codes, scales, rows, cols, out, type, row_stride), __func__);
}

sim_status sim_mx4_matmul(void *stream, const uint8_t *a_codes, const uint8_t *a_scales, const uint8_t *b_codes,
                          const uint8_t *b_scales, int64_t M, int64_t N, int64_t K, void *out, int32_t type,
                          int64_t row_stride) {
    NEED(is_float(type), "out must be f32, f16 or bf16");
    NEED(M >= 0 && N >= 0 && K >= 0, "negative size");
    FITS(linear_fits(M, N, K), "matrix too large");
    if (M == 0 || N == 0) return done(SIM_OK, __func__);
    NEED(out && (K == 0 || (a_codes && a_scales && b_codes && b_scales)), "null array");
    NEED(M == 1 || row_stride >= N, "row stride below the row length");
    NEED(aligned_to(out, size_of(type)), "out not aligned to its type");
    NEED(aligned_to(a_codes, 16) && aligned_to(a_scales, 8) && aligned_to(b_codes, 16) && aligned_to(b_scales, 8),
         "codes must be 16-byte, scales 8-byte aligned");
    return done(launch_matmul((hipStream_t)stream, a_codes, a_scales, b_codes, b_scales, M, N, K, out, type, row_stride),
                __func__);
}

size_t sim_mx4_linear_workspace(int64_t M, int64_t N, int64_t K) {
    if (!linear_fits(M, N, K) || M == 0 || N == 0 || K == 0 || linear_in_one(M, K)) return 0;
    return (size_t)((M * (sim_mx4_code_pitch(K) + sim_mx4_scale_pitch(K)) + 15) / 16 * 16);
}

sim_status sim_mx4_linear(void *stream, const void *x, int32_t x_type, int64_t x_stride, const uint8_t *w_codes,
                          const uint8_t *w_scales, int64_t M, int64_t N, int64_t K, void *out, int32_t type,
                          int64_t row_stride, void *workspace, size_t workspace_bytes) {
    NEED(is_float(x_type) && is_float(type), "x and out must be f32, f16 or bf16");
    NEED(M >= 0 && N >= 0 && K >= 0, "negative size");
    FITS(linear_fits(M, N, K), "matrix too large");
    if (M == 0 || N == 0) return done(SIM_OK, __func__);
    NEED(out && (K == 0 || (x && w_codes && w_scales)), "null array");
    NEED(M == 1 || (x_stride >= K && row_stride >= N), "row stride below the row length");
    NEED(aligned_to(x, size_of(x_type)) && aligned_to(out, size_of(type)), "x or out not aligned to its type");
    NEED(aligned_to(w_codes, 16) && aligned_to(w_scales, 8), "codes must be 16-byte, scales 8-byte aligned");
    const size_t need = sim_mx4_linear_workspace(M, N, K);
    NEED(need == 0 || (workspace && workspace_bytes >= need && aligned_to(workspace, 16)), "workspace too small or not aligned");
    if (linear_in_one(M, K))
        return done(launch_linear((hipStream_t)stream, x, x_type, x_stride, w_codes, w_scales, M, N, K, out, type, row_stride),
                    __func__);
    uint8_t *codes = (uint8_t *)workspace, *scales = codes + M * sim_mx4_code_pitch(K);
    if (K > 0) {
        const sim_status s = launch_quantize((hipStream_t)stream, x, x_type, M, K, x_stride, false, codes, scales);
        if (s != SIM_OK) return done(s, __func__);
    }
    return done(launch_matmul((hipStream_t)stream, codes, scales, w_codes, w_scales, M, N, K, out, type, row_stride), __func__);
}

// Codes and scales of an R x C operand, one after the other.
static size_t operand_bytes(int64_t R, int64_t C) {
    return (size_t)(R * sim_mx4_code_pitch(C) + (R * sim_mx4_scale_pitch(C) + 15) / 16 * 16);
}

size_t sim_mx4_linear_grad_workspace(int64_t M, int64_t N, int64_t K) {
    if (!linear_grad_fits(M, N, K) || M == 0 || N == 0 || K == 0) return 0;
    return operand_bytes(M, N) + operand_bytes(K, N) + operand_bytes(N, M) + operand_bytes(K, M);
}

sim_status sim_mx4_linear_grad(void *stream, int32_t type, const void *dy, int64_t dy_stride, const void *x, int64_t x_stride,
                               const void *w, int64_t w_stride, int64_t M, int64_t N, int64_t K, void *dx, int64_t dx_stride,
                               void *dw, int64_t dw_stride, void *workspace, size_t workspace_bytes) {
    NEED(is_float(type), "dy, x and w must be f32, f16 or bf16");
    NEED(M >= 0 && N >= 0 && K >= 0, "negative size");
    FITS(linear_grad_fits(M, N, K), "matrix too large");
    const bool want_x = dx && M > 0 && K > 0, want_w = dw && N > 0 && K > 0;
    if (!want_x && !want_w) return done(SIM_OK, __func__);
    const size_t s = size_of(type);
    const bool sum_n = N > 0, sum_m = M > 0;  // an empty sum gives zeros
    NEED((!sum_n || !sum_m || dy) && (!(want_x && sum_n) || w) && (!(want_w && sum_m) || x), "null array");
    NEED((M <= 1 || dy_stride >= N) && (M <= 1 || x_stride >= K) && (N <= 1 || w_stride >= K), "row stride below the row length");
    NEED((!want_x || M == 1 || dx_stride >= K) && (!want_w || N == 1 || dw_stride >= K), "row stride below the row length");
    NEED(aligned_to(dy, s) && aligned_to(x, s) && aligned_to(w, s) && aligned_to(dx, s) && aligned_to(dw, s),
         "array not aligned to its type");
    const size_t need = sim_mx4_linear_grad_workspace(M, N, K);
    NEED(need == 0 || (workspace && workspace_bytes >= need && aligned_to(workspace, 16)), "workspace too small or not aligned");
    uint8_t *at = (uint8_t *)workspace;
    QuantizeJob job[kMaxJobs];
    int n = 0;
    // the operand of R rows whose blocks lie along C; x is C x R where it is transposed
    const auto operand = [&](const void *from, int64_t R, int64_t C, int64_t stride, bool transpose) {
        QuantizeJob &j = job[n++];
        j = QuantizeJob{from, transpose ? C : R, transpose ? R : C, stride, transpose, at, at + R * sim_mx4_code_pitch(C)};
        at += operand_bytes(R, C);
        return &j;
    };
    const QuantizeJob *dy_n = nullptr, *w_n = nullptr, *dy_m = nullptr, *x_m = nullptr;
    if (want_x && sum_n) dy_n = operand(dy, M, N, dy_stride, false), w_n = operand(w, K, N, w_stride, true);
    if (want_w && sum_m) dy_m = operand(dy, N, M, dy_stride, true), x_m = operand(x, K, M, x_stride, true);
    sim_status st = n ? launch_quantize_jobs((hipStream_t)stream, type, job, n) : SIM_OK;
    if (st == SIM_OK && want_x)
        st = dy_n ? launch_matmul((hipStream_t)stream, dy_n->codes, dy_n->scales, w_n->codes, w_n->scales, M, K, N, dx, type, dx_stride)
                  : launch_matmul((hipStream_t)stream, nullptr, nullptr, nullptr, nullptr, M, K, 0, dx, type, dx_stride);
    if (st == SIM_OK && want_w)
        st = dy_m ? launch_matmul((hipStream_t)stream, dy_m->codes, dy_m->scales, x_m->codes, x_m->scales, N, K, M, dw, type, dw_stride)
                  : launch_matmul((hipStream_t)stream, nullptr, nullptr, nullptr, nullptr, N, K, 0, dw, type, dw_stride);
    return done(st, __func__);
}

size_t sim_moe_route_workspace(int64_t T, int32_t E, int32_t k) { return T > 0 && E > 0 ? route_workspace(T, E, k) : 0; }

sim_status sim_moe_route(void *stream, const void *logits, int32_t type, int64_t T, int32_t E, int64_t logit_stride,
                         const uint8_t *mask, int64_t mask_stride, int32_t k, int32_t renormalize, int32_t *experts,
                         float *weights, int32_t *offsets, int32_t *order, void *workspace, size_t workspace_bytes) {
    if (const char *why = route_bad(logits, type, T, E, logit_stride, mask, mask_stride, k))
        return refuse(SIM_ERR_INVALID_ARG, __func__, why);
    FITS(T <= kMaxTokens && T < kMaxDim / k, "too many tokens");
    NEED((offsets != nullptr) == (order != nullptr) || (T == 0 && offsets), "offsets and order go together");
    NEED(T == 0 || (experts && weights), "null array");
    NEED(aligned_to(experts, 4) && aligned_to(weights, 4) && aligned_to(offsets, 4) && aligned_to(order, 4), "output not aligned");
    const size_t need = order ? sim_moe_route_workspace(T, E, k) : 0;
    NEED(need == 0 || (workspace && workspace_bytes >= need && aligned_to(workspace, 16)), "workspace too small or not aligned");
    const RouteArgs a = {logits, type, T, E, logit_stride, mask, mask_stride, k, renormalize != 0};
    return done(launch_route((hipStream_t)stream, a, experts, weights, offsets, order, workspace), __func__);
}

sim_status sim_moe_route_grad(void *stream, const void *logits, int32_t type, int64_t T, int32_t E, int64_t logit_stride,
                              const uint8_t *mask, int64_t mask_stride, int32_t k, int32_t renormalize,
                              const int32_t *experts, const float *d_weights, void *d_logits) {
    if (const char *why = route_bad(logits, type, T, E, logit_stride, mask, mask_stride, k))
        return refuse(SIM_ERR_INVALID_ARG, __func__, why);
    FITS(T <= kMaxTokens && T < kMaxDim / k, "too many tokens");
    if (T == 0) return done(SIM_OK, __func__);
    NEED(experts && d_weights && d_logits, "null array");
    NEED(aligned_to(experts, 4) && aligned_to(d_weights, 4) && aligned_to(d_logits, size_of(type)), "array not aligned");
    const RouteArgs a = {logits, type, T, E, logit_stride, mask, mask_stride, k, renormalize != 0};
    return done(launch_route_grad((hipStream_t)stream, a, experts, d_weights, d_logits), __func__);
}

static const char *scored_bad(int32_t score, float scale) {
    if (score != SIM_SCORE_SOFTMAX && score != SIM_SCORE_SIGMOID) return "unknown score";
    if (!std::isfinite(scale)) return "scale must be finite";
    return nullptr;
}

sim_status sim_moe_route_scored(void *stream, const void *logits, int32_t type, int64_t T, int32_t E, int64_t logit_stride,
                                const uint8_t *mask, int64_t mask_stride, int32_t score, const float *bias, int32_t groups,
                                int32_t top_groups, int32_t group_best, int32_t k, int32_t renormalize, float scale,
                                int32_t *experts, float *weights, int32_t *offsets, int32_t *order, void *workspace,
                                size_t workspace_bytes) {
    if (const char *why = route_bad(logits, type, T, E, logit_stride, mask, mask_stride, k))
        return refuse(SIM_ERR_INVALID_ARG, __func__, why);
    if (const char *why = scored_bad(score, scale)) return refuse(SIM_ERR_INVALID_ARG, __func__, why);
    NEED(groups >= 1 && groups <= SIM_MOE_MAX_GROUPS && E % groups == 0, "groups must divide the experts, 64 at most");
    NEED(top_groups >= 1 && top_groups <= groups, "top_groups out of range");
    NEED(group_best == 1 || group_best == 2, "group_best must be 1 or 2");
    NEED(aligned_to(bias, 4), "bias not aligned to its type");
    FITS(T <= kMaxTokens && T < kMaxDim / k, "too many tokens");
    NEED((offsets != nullptr) == (order != nullptr) || (T == 0 && offsets), "offsets and order go together");
    NEED(T == 0 || (experts && weights), "null array");
    NEED(aligned_to(experts, 4) && aligned_to(weights, 4) && aligned_to(offsets, 4) && aligned_to(order, 4), "output not aligned");
    const size_t need = order ? sim_moe_route_workspace(T, E, k) : 0;
    NEED(need == 0 || (workspace && workspace_bytes >= need && aligned_to(workspace, 16)), "workspace too small or not aligned");
    RouteArgs a = {logits, type, T, E, logit_stride, mask, mask_stride, k, renormalize != 0};
    a.scored = true, a.score = score, a.bias = bias;
    a.groups = groups, a.top_groups = top_groups, a.group_best = group_best, a.scale = scale;
    return done(launch_route((hipStream_t)stream, a, experts, weights, offsets, order, workspace), __func__);
}

sim_status sim_moe_route_scored_grad(void *stream, const void *logits, int32_t type, int64_t T, int32_t E, int64_t logit_stride,
                                     const uint8_t *mask, int64_t mask_stride, int32_t score, int32_t k, int32_t renormalize,
                                     float scale, const int32_t *experts, const float *d_weights, void *d_logits) {
    if (const char *why = route_bad(logits, type, T, E, logit_stride, mask, mask_stride, k))
        return refuse(SIM_ERR_INVALID_ARG, __func__, why);
    if (const char *why = scored_bad(score, scale)) return refuse(SIM_ERR_INVALID_ARG, __func__, why);
    FITS(T <= kMaxTokens && T < kMaxDim / k, "too many tokens");
    if (T == 0) return done(SIM_OK, __func__);
    NEED(experts && d_weights && d_logits, "null array");
    NEED(aligned_to(experts, 4) && aligned_to(d_weights, 4) && aligned_to(d_logits, size_of(type)), "array not aligned");
    RouteArgs a = {logits, type, T, E, logit_stride, mask, mask_stride, k, renormalize != 0};
    a.score = score, a.scale = scale;
    return done(launch_route_grad((hipStream_t)stream, a, experts, d_weights, d_logits), __func__);
}

size_t sim_moe_layer_workspace(int64_t T, int64_t D, int32_t E, int32_t k, int64_t F) {
    if (T <= 0 || T > SIM_MOE_LAYER_MAX_TOKENS || D <= 0 || F < 0 || E < 1 || E > SIM_MOE_MAX_EXPERTS || k < 1 || k > E ||
        k > SIM_MOE_MAX_TOPK || !layer_dims_fit(D, F) || !layer_tiles_fit(T, D, E, k, F))
        return 0;
    return layer_workspace(T, D, E, k, F);
}

sim_status sim_moe_layer(void *stream, const void *x, int32_t type, int64_t T, int64_t D, int64_t x_stride,
                         const void *logits, int32_t logit_type, int32_t E, int64_t logit_stride, const uint8_t *mask,
                         int64_t mask_stride, int32_t k, int32_t renormalize, const void *w13, const uint8_t *s13,
                         const void *w2, const uint8_t *s2, int32_t weight_type, int64_t F, void *y, int64_t y_stride,
                         void *workspace, size_t workspace_bytes) {
    if (const char *why = route_bad(logits, logit_type, T, E, logit_stride, mask, mask_stride, k))
        return refuse(SIM_ERR_INVALID_ARG, __func__, why);
    NEED(type == SIM_TYPE_F16 || type == SIM_TYPE_BF16, "x must be f16 or bf16");
    NEED(weight_type == type || weight_type == SIM_TYPE_MX4, "weights must have the type of x or be in 4 bits");
    NEED(D >= 0 && F >= 0, "negative size");
    FITS(T <= SIM_MOE_LAYER_MAX_TOKENS, "too many tokens for one call");
    FITS(layer_dims_fit(D, F), "matrix too large");
    FITS(layer_tiles_fit(T, D, E, k, F), "too many experts of that size");
    if (T == 0 || D == 0) return done(SIM_OK, __func__);
    const bool mx4 = weight_type == SIM_TYPE_MX4;
    NEED(x && y && (F == 0 || (w13 && w2)), "null array");
    NEED(F == 0 || (mx4 ? s13 && s2 : !s13 && !s2), "scales go with 4-bit weights");
    NEED(T == 1 || (x_stride >= D && y_stride >= D), "row stride below the row length");
    NEED(aligned_to(x, 2) && aligned_to(y, 2) && aligned_to(w13, mx4 ? 16 : 2) && aligned_to(w2, mx4 ? 16 : 2) &&
             aligned_to(s13, 8) && aligned_to(s2, 8),
         "array not aligned");
    const size_t need = sim_moe_layer_workspace(T, D, E, k, F);
    NEED(workspace && workspace_bytes >= need && aligned_to(workspace, 16), "workspace too small or not aligned");
    LayerArgs a;
    a.route = RouteArgs{logits, logit_type, T, E, logit_stride, mask, mask_stride, k, renormalize != 0};
    a.x = x, a.type = type, a.D = D, a.x_stride = x_stride;
    a.w13 = w13, a.w2 = w2, a.s13 = s13, a.s2 = s2, a.mx4 = mx4, a.F = F;
    a.y = y, a.y_stride = y_stride;
    return done(launch_layer((hipStream_t)stream, a, workspace), __func__);
}

static bool experts_fit(int64_t T, int64_t D, int32_t n, int32_t k, int64_t F) {
    return layer_dims_fit(D, F) && layer_tiles_fit(T, D, n, k, F);
}

size_t sim_moe_experts_workspace(int64_t T, int64_t D, int32_t n, int32_t k, int64_t F) {
    if (T <= 0 || T > SIM_MOE_LAYER_MAX_TOKENS || D <= 0 || F < 0 || n < 1 || n > SIM_MOE_MAX_EXPERTS || k < 1 ||
        k > SIM_MOE_MAX_TOPK || !experts_fit(T, D, n, k, F))
        return 0;
    return layer_workspace(T, D, n, k, F);
}

sim_status sim_moe_experts(void *stream, const void *x, int32_t type, int64_t T, int64_t D, int64_t x_stride,
                           const int32_t *experts, const float *weights, int32_t k, int32_t first, int32_t n, const void *w13,
                           const uint8_t *s13, const void *w2, const uint8_t *s2, int32_t weight_type, int64_t F, void *y,
                           int64_t y_stride, void *workspace, size_t workspace_bytes) {
    NEED(type == SIM_TYPE_F16 || type == SIM_TYPE_BF16, "x must be f16 or bf16");
    NEED(weight_type == type || weight_type == SIM_TYPE_MX4, "weights must have the type of x or be in 4 bits");
    NEED(T >= 0 && D >= 0 && F >= 0, "negative size");
    NEED(k >= 1 && k <= SIM_MOE_MAX_TOPK, "k out of range");
    NEED(first >= 0 && n >= 1 && n <= SIM_MOE_MAX_EXPERTS && first <= INT32_MAX - n, "share of the experts out of range");
    FITS(T <= SIM_MOE_LAYER_MAX_TOKENS, "too many tokens for one call");
    FITS(layer_dims_fit(D, F), "matrix too large");
    FITS(layer_tiles_fit(T, D, n, k, F), "too many experts of that size");
    if (T == 0 || D == 0) return done(SIM_OK, __func__);
    const bool mx4 = weight_type == SIM_TYPE_MX4;
    NEED(x && y && experts && weights && (F == 0 || (w13 && w2)), "null array");
    NEED(F == 0 || (mx4 ? s13 && s2 : !s13 && !s2), "scales go with 4-bit weights");
    NEED(T == 1 || (x_stride >= D && y_stride >= D), "row stride below the row length");
    NEED(aligned_to(x, 2) && aligned_to(y, 2) && aligned_to(w13, mx4 ? 16 : 2) && aligned_to(w2, mx4 ? 16 : 2) &&
             aligned_to(s13, 8) && aligned_to(s2, 8) && aligned_to(experts, 4) && aligned_to(weights, 4),
         "array not aligned");
    const size_t need = sim_moe_experts_workspace(T, D, n, k, F);
    NEED(workspace && workspace_bytes >= need && aligned_to(workspace, 16), "workspace too small or not aligned");
    LayerArgs a;
    a.route = RouteArgs{nullptr, SIM_TYPE_F32, T, n, 0, nullptr, 0, k, false};
    a.route.given = experts, a.route.given_weights = weights, a.route.first = first;
    a.x = x, a.type = type, a.D = D, a.x_stride = x_stride;
    a.w13 = w13, a.w2 = w2, a.s13 = s13, a.s2 = s2, a.mx4 = mx4, a.F = F;
    a.y = y, a.y_stride = y_stride;
    return done(launch_layer((hipStream_t)stream, a, workspace), __func__);
}

namespace {
constexpr int64_t kMaxKeys = (int64_t)1 << 30;  // of one sequence
constexpr int64_t kMaxGroups = (int64_t)1 << 31;  // workgroups of one launch

// what the cache's users check alike
const char *cache_bad(int32_t type, int32_t kv_heads, int32_t D, const void *k, int64_t k_page_stride, const void *v,
                      int64_t v_page_stride, int64_t pages, int32_t page_size) {
    if (type != SIM_TYPE_F16 && type != SIM_TYPE_BF16) return "the cache must be f16 or bf16";
    if (kv_heads < 1) return "kv_heads must be positive";
    if (D < 8 || D > SIM_CACHE_MAX_D || D % 8) return "D must be a multiple of 8 up to 256";
    if (pages < 0 || page_size < 1) return "bad page count or size";
    if (pages > 0 && (!k || !v)) return "null cache";
    if (!aligned_to(k, 16) || !aligned_to(v, 16) || k_page_stride % 8 || v_page_stride % 8)
        return "the cache must be 16-byte aligned, its page strides multiples of 8";
    if (pages > 1 && (k_page_stride / D / kv_heads < page_size || v_page_stride / D / kv_heads < page_size))
        return "page stride below the page";
    return nullptr;
}
bool cache_fits(int32_t kv_heads, int64_t pages, int32_t page_size) {
    return kv_heads <= 65536 && pages < kMaxDim && (int64_t)page_size * kv_heads < kMaxDim;
}
bool attention_fits(int64_t B, int32_t q_heads, int32_t kv_heads, int32_t D, int32_t table_pages, int32_t page_size, int32_t window) {
    if (B < 1 || B >= kMaxDim || q_heads < 1 || kv_heads < 1 || q_heads % kv_heads || q_heads > 65536 || D < 8 ||
        D > SIM_CACHE_MAX_D || D % 8 || table_pages < 0 || page_size < 1 || window < 0 ||
        (int64_t)table_pages * page_size > kMaxKeys)
        return false;
    const int64_t tiles = attend_tiles(q_heads / kv_heads, D), units = attend_units(kv_heads * tiles, attend_resident(D, attend_heads(q_heads / kv_heads, D)));
    return (attend_max_units(B, units, (int64_t)table_pages * page_size, window) * kv_heads + 8) * tiles < kMaxGroups / 256 &&
           B * q_heads < kMaxGroups / 256;  // (a launch has 2^32 threads at most)
}
}  // namespace

sim_status sim_cache_append(void *stream, int32_t type, const void *k, int64_t k_stride, int64_t k_head_stride, const void *v,
                            int64_t v_stride, int64_t v_head_stride, int64_t T, int32_t kv_heads, int32_t D,
                            const int64_t *slots, void *k_cache, int64_t k_page_stride, void *v_cache, int64_t v_page_stride,
                            int64_t pages, int32_t page_size) {
    if (const char *why = cache_bad(type, kv_heads, D, k_cache, k_page_stride, v_cache, v_page_stride, pages, page_size))
        return refuse(SIM_ERR_INVALID_ARG, __func__, why);
    NEED(T >= 0, "negative token count");
    FITS(cache_fits(kv_heads, pages, page_size) && T < kMaxDim, "too large");
    NEED(k_stride >= 0 && k_head_stride >= 0 && v_stride >= 0 && v_head_stride >= 0, "negative stride");
    if (T == 0 || pages == 0) return done(SIM_OK, __func__);
    NEED(k && v && slots, "null array");
    NEED(aligned_to(k, 2) && aligned_to(v, 2) && aligned_to(slots, 8), "array not aligned to its type");
    NEED(!pages_meet((uintptr_t)k_cache, (uint64_t)k_page_stride * 2, (uintptr_t)v_cache, (uint64_t)v_page_stride * 2, (uint64_t)pages,
                     (uint64_t)kv_heads * page_size * D * 2),
         "keys and values must be written to places of their own");
    const AppendArgs a = {k, v, k_stride, k_head_stride, v_stride, v_head_stride, T, kv_heads, D, slots, k_cache, v_cache,
                          k_page_stride, v_page_stride, pages, page_size};
    return done(launch_append((hipStream_t)stream, a), __func__);
}

size_t sim_cache_attention_workspace(int64_t B, int32_t q_heads, int32_t kv_heads, int32_t D, int32_t table_pages,
                                     int32_t page_size, int32_t window) {
    if (!attention_fits(B, q_heads, kv_heads, D, table_pages, page_size, window)) return 0;
    const int64_t capacity = (int64_t)table_pages * page_size;
    if (!attend_splits(capacity, window)) return 0;
    const int group = q_heads / kv_heads;
    const int64_t units = attend_units((int64_t)kv_heads * attend_tiles(group, D), attend_resident(D, attend_heads(group, D)));
    return (size_t)((attend_max_units(B, units, capacity, window) * q_heads * (D + 2) * 4 + 15) / 16 * 16);
}

sim_status sim_cache_attention(void *stream, int32_t type, const void *q, int64_t q_stride, int64_t q_head_stride, int64_t B,
                               int32_t q_heads, int32_t kv_heads, int32_t D, const void *k_cache, int64_t k_page_stride,
                               const void *v_cache, int64_t v_page_stride, int64_t pages, int32_t page_size,
                               const int32_t *table, int64_t table_stride, int32_t table_pages, const int32_t *lengths,
                               float scale, int32_t window, void *out, int64_t out_stride, float *lse, void *workspace,
                               size_t workspace_bytes) {
    if (const char *why = cache_bad(type, kv_heads, D, k_cache, k_page_stride, v_cache, v_page_stride, pages, page_size))
        return refuse(SIM_ERR_INVALID_ARG, __func__, why);
    NEED(B >= 0 && table_pages >= 0 && window >= 0, "negative size");
    NEED(q_heads >= 1 && q_heads % kv_heads == 0, "kv_heads must divide q_heads");
    const float scale_log2 = (float)(scale * 1.4426950408889634);
    NEED(std::isfinite(scale_log2), "scale must be finite, 2e38 at most");
    NEED(q_stride >= 0 && q_head_stride >= 0 && table_stride >= 0, "negative stride");
    FITS((int64_t)table_pages * page_size <= kMaxKeys, "a row of the table has room for more than 2^30 tokens");
    if (B == 0) return done(SIM_OK, __func__);
    FITS(cache_fits(kv_heads, pages, page_size) && attention_fits(B, q_heads, kv_heads, D, table_pages, page_size, window), "too large");
    NEED(q && out && lengths && (table_pages == 0 || table), "null array");
    NEED(B == 1 || out_stride >= (int64_t)q_heads * D, "out's stride below its row");
    NEED(aligned_to(q, 2) && aligned_to(out, 2) && aligned_to(table, 4) && aligned_to(lengths, 4) && aligned_to(lse, 4),
         "array not aligned to its type");
    const size_t need = sim_cache_attention_workspace(B, q_heads, kv_heads, D, table_pages, page_size, window);
    NEED(need == 0 || (workspace && workspace_bytes >= need && aligned_to(workspace, 16)), "workspace too small or not aligned");
    AttendArgs a;
    a.q = q, a.q_stride = q_stride, a.q_head_stride = q_head_stride, a.B = B;
    a.type = type, a.q_heads = q_heads, a.kv_heads = kv_heads, a.D = D;
    a.k_cache = k_cache, a.v_cache = v_cache, a.k_page_stride = k_page_stride, a.v_page_stride = v_page_stride;
    a.pages = pages, a.page_size = page_size;
    a.table = table, a.table_stride = table_stride, a.capacity = (int64_t)table_pages * page_size, a.lengths = lengths;
    a.scale_log2 = scale_log2, a.window = window;
    a.out = out, a.out_stride = out_stride, a.lse = lse, a.part = (float *)workspace;
    a.tiles = attend_tiles(q_heads / kv_heads, D), a.units = attend_units((int64_t)kv_heads * a.tiles, attend_resident(D, attend_heads(q_heads / kv_heads, D)));
    a.max_units = attend_max_units(B, a.units, a.capacity, window);
    a.splits = attend_splits(a.capacity, window);
    a.q_aligned = aligned_to(q, 16) && (B == 1 || q_stride % 8 == 0) && (q_heads == 1 || q_head_stride % 8 == 0);
    a.out_aligned = aligned_to(out, 16) && (B == 1 || out_stride % 8 == 0);
    return done(launch_attention((hipStream_t)stream, a), __func__);
}

static bool sample_fits(int64_t B, int32_t V) { return B >= 0 && B < kMaxDim / 1024 && V <= SIM_SAMPLE_MAX_V; }

size_t sim_sample_workspace(int64_t B, int32_t V) { return B > 0 && V > 0 && sample_fits(B, V) ? sample_workspace(B, V) : 0; }

sim_status sim_sample(void *stream, const void *logits, int32_t type, int64_t B, int32_t V, int64_t logit_stride, const float *u,
                      const float *temperature, float all_temperature, const int32_t *top_k, int32_t all_k, const float *top_p,
                      float all_p, const float *min_p, float all_min, int32_t *tokens, void *workspace, size_t workspace_bytes) {
    NEED(is_float(type), "logits must be f32, f16 or bf16");
    NEED(B >= 0 && V >= 1, "there must be a logit to choose");
    FITS(sample_fits(B, V), "too many logits");
    NEED(temperature || (all_temperature >= 0 && std::isfinite(all_temperature)), "temperature must be finite and not negative");
    NEED(top_p || (all_p >= 0 && all_p <= 1), "top_p must be from 0 to 1");
    NEED(min_p || (all_min >= 0 && all_min <= 1), "min_p must be from 0 to 1");
    NEED(top_k || all_k >= 0, "top_k must not be negative");
    if (B == 0) return done(SIM_OK, __func__);
    NEED(logits && u && tokens, "null array");
    NEED(B == 1 || logit_stride >= V, "logit stride below the row length");
    NEED(aligned_to(logits, size_of(type)) && aligned_to(u, 4) && aligned_to(temperature, 4) && aligned_to(top_k, 4) &&
             aligned_to(top_p, 4) && aligned_to(min_p, 4) && aligned_to(tokens, 4),
         "array not aligned to its type");
    const size_t need = sim_sample_workspace(B, V);
    NEED(need == 0 || (workspace && workspace_bytes >= need && aligned_to(workspace, 16)), "workspace too small or not aligned");
    const SampleArgs a = {logits, type, B, logit_stride, V, u, temperature, top_p, min_p, top_k, all_temperature, all_p, all_min, all_k, tokens};
    return done(launch_sample((hipStream_t)stream, a, workspace), __func__);
}

}  // extern "C"
