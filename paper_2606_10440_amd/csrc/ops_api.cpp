// C entry points of the operators: every argument is checked here, before
// anything is enqueued; the launchers rely on what passed.
#include <algorithm>
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

}  // extern "C"
