// cf_head_api.hip -- the C ABI of the operators for heads over features:
// argument validation on the host (no HIP call before every check has
// passed), then their launchers.
#include "cf_check.h"
#include "cf_head.h"

namespace {

using namespace cf;

cf_status check_any_act(const char *what, cf_act act) {
    return (int)act == CF_ACT_SILU ? CF_OK : check_act(what, act);
}

// N images of P pixels as rows
cf_status check_images(const char *what, int64_t N, int64_t P, int C, int G) {
    if (N < 0 || P < 0 || (double)N * (double)P > 4.0e12)
        return api_fail(CF_ERR_INVALID, "%s: N=%lld and P=%lld must not be negative, nor the tensor too large", what,
                        (long long)N, (long long)P);
    CF_TRY(check_rows(what, N * P, C, "C"));
    if (G <= 0 || C % G)
        return api_fail(CF_ERR_INVALID, "%s: groups=%d must be positive and divide C=%d", what, G, C);
    return CF_OK;
}

cf_status no_images(const char *what, int64_t N, int64_t P, int C, int G) {
    return api_fail(CF_ERR_UNSUPPORTED, "%s: no kernel for N=%lld P=%lld C=%d groups=%d (a group of up to %d channels)",
                    what, (long long)N, (long long)P, C, G, CF_GROUP_MAX);
}
// row strides: an image's pixels beside each other are told apart in 32 bits
cf_status check_near(const char *what, int64_t rows, int64_t ld) {
    if (rows > 1 && ld >= (int64_t)1 << 22)
        return api_fail(CF_ERR_UNSUPPORTED, "%s: row strides must be below 2^22, got %lld", what, (long long)ld);
    return CF_OK;
}
bool images_fit(int64_t N, int64_t P, int C, int G) { return C / G <= CF_GROUP_MAX && group_norm_fits(N, P, C, G); }

// whether the matrix products could read these rows in place, were their length
// a multiple of 8
bool readable(const void *p, int64_t ld) { return products_read(p, ld, 8); }

cf_status too_large(const char *what) {
    return api_fail(CF_ERR_UNSUPPORTED, "%s: no kernel for sizes this large", what);
}

}  // namespace

extern "C" {

size_t cf_group_norm_workspace_bytes(int64_t N, int64_t P, int C, int G) {
    return N <= 0 || P <= 0 || C <= 0 || G <= 0 || C % G || !images_fit(N, P, C, G)
               ? 0
               : group_norm_workspace_bytes(N, P, C, G);
}

cf_status cf_group_norm_forward(const void *x, void *y, const float *weight, const float *bias, float *stats, void *ws,
                                size_t ws_bytes, int64_t N, int64_t P, int C, int G, int64_t ldx, int64_t ldy,
                                float eps, cf_dtype dt, cf_act act, void *stream) {
    const char *const what = "cf_group_norm_forward";
    CF_TRY(check_images(what, N, P, C, G));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_any_act(what, act));
    const int64_t rows = N * P;
    CF_TRY(check_ld(what, "ldx", ldx, 0, rows));
    CF_TRY(check_ld(what, "ldy", ldy, C, rows));
    if (!(eps >= 0.0f) || eps > 1.0e30f)
        return api_fail(CF_ERR_INVALID, "%s: eps must be a finite number that is not negative", what);
    if (rows == 0)
        return api_done(hipSuccess, what);
    if (!x || !y)
        return api_fail(CF_ERR_INVALID, "%s: x and y must be non-NULL", what);
    const Span t[] = {{"x", x, rows, C, ldx, 2},
                      dense("weight", weight, 1, C, 4),
                      dense("bias", bias, 1, C, 4),
                      {"y", y, rows, C, ldy, 2},
                      dense("stats", stats, N, 2 * (int64_t)G, 4)};
    CF_TRY(check_aligned(what, t, 5));
    if (!aligned(stats, 8))
        return api_fail(CF_ERR_INVALID, "%s: stats must be 8-byte aligned", what);
    for (int i = 3; i < 5; i++)
        CF_TRY(check_out(what, t[i], t, i, i == 3 ? t[0].name : ""));
    if (!images_fit(N, P, C, G))
        return no_images(what, N, P, C, G);
    CF_TRY(check_near(what, rows, ldx));
    CF_TRY(check_near(what, rows, ldy));
    CF_TRY(check_ws(what, ws, ws_bytes, cf_group_norm_workspace_bytes(N, P, C, G), t, 5));
    const GroupNorm a = {x, ldx, weight, bias, N, P, C, G, (int)act};
    return api_done(launch_group_norm(a, y, ldy, stats, eps, dt == CF_BF16, ws, (hipStream_t)stream), what);
}

size_t cf_group_norm_backward_workspace_bytes(int64_t N, int64_t P, int C, int G) {
    return N <= 0 || P <= 0 || C <= 0 || G <= 0 || C % G || !images_fit(N, P, C, G)
               ? 0
               : group_norm_backward_workspace_bytes(N, P, C, G);
}

cf_status cf_group_norm_backward(const void *dy, const void *x, const float *stats, const float *weight,
                                 const float *bias, void *dx, float *dweight, float *dbias, void *ws, size_t ws_bytes,
                                 int64_t N, int64_t P, int C, int G, int64_t lddy, int64_t ldx, int64_t lddx,
                                 cf_dtype dt, cf_act act, void *stream) {
    const char *const what = "cf_group_norm_backward";
    CF_TRY(check_images(what, N, P, C, G));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_any_act(what, act));
    const int64_t rows = N * P;
    CF_TRY(check_ld(what, "lddy", lddy, 0, rows));
    CF_TRY(check_ld(what, "ldx", ldx, 0, rows));
    CF_TRY(check_ld(what, "lddx", lddx, C, rows));
    if (!dweight != !dbias)
        return api_fail(CF_ERR_INVALID, "%s: dweight and dbias go together", what);
    if (rows > 0 && (!dy || !x || !stats || !dx))
        return api_fail(CF_ERR_INVALID, "%s: dy, x, stats and dx must be non-NULL", what);
    const Span t[] = {{"dy", dy, rows, C, lddy, 2},
                      {"x", x, rows, C, ldx, 2},
                      dense("stats", stats, N, 2 * (int64_t)G, 4),
                      dense("weight", weight, 1, C, 4),
                      dense("bias", bias, 1, C, 4),
                      {"dx", dx, rows, C, lddx, 2},
                      dense("dweight", dweight, 1, C, 4),
                      dense("dbias", dbias, 1, C, 4)};
    CF_TRY(check_aligned(what, t, 8));
    if (!aligned(stats, 8))
        return api_fail(CF_ERR_INVALID, "%s: stats must be 8-byte aligned", what);
    for (int i = 5; i < 8; i++)
        CF_TRY(check_out(what, t[i], t, i, i == 5 ? t[0].name : ""));
    if (rows > 0 && !images_fit(N, P, C, G))
        return no_images(what, N, P, C, G);
    CF_TRY(check_near(what, rows, lddy));
    CF_TRY(check_near(what, rows, ldx));
    CF_TRY(check_near(what, rows, lddx));
    if (rows == 0 && !dweight)
        return api_done(hipSuccess, what);
    CF_TRY(check_ws(what, ws, ws_bytes, cf_group_norm_backward_workspace_bytes(N, P, C, G), t, 8));
    const GroupNorm a = {x, ldx, weight, bias, N, P, C, G, (int)act};
    return api_done(launch_group_norm_backward(a, dy, lddy, stats, dx, lddx, dweight, dbias, dt == CF_BF16, ws,
                                               (hipStream_t)stream),
                    what);
}

size_t cf_gated_ffn_workspace_bytes(int64_t rows, int C, int H, int aligned) {
    return rows <= 0 || C <= 0 || H <= 0 || !gated_fits(rows, C, H) ? 0
                                                                     : gated_workspace_bytes(rows, C, H, aligned != 0);
}

cf_status cf_gated_ffn_forward(const void *x, const void *w_gate, const void *w_up, const void *w_down, void *y,
                               float *saved, void *ws, size_t ws_bytes, int64_t rows, int C, int H, int64_t ldx,
                               int64_t ld_gate, int64_t ld_up, int64_t ld_down, int64_t ldy, cf_dtype dt, cf_act act,
                               void *stream) {
    const char *const what = "cf_gated_ffn_forward";
    CF_TRY(check_rows(what, rows, C, "C"));
    CF_TRY(check_rows(what, rows, H, "H"));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_any_act(what, act));
    CF_TRY(check_ld(what, "ldx", ldx, 0, rows));
    CF_TRY(check_ld(what, "ld_gate", ld_gate, 0, H));
    CF_TRY(check_ld(what, "ld_up", ld_up, 0, H));
    CF_TRY(check_ld(what, "ld_down", ld_down, 0, C));
    CF_TRY(check_ld(what, "ldy", ldy, C, rows));
    if (rows == 0)
        return api_done(hipSuccess, what);
    if (!x || !w_gate || !w_up || !w_down || !y)
        return api_fail(CF_ERR_INVALID, "%s: x, the weights and y must be non-NULL", what);
    const Span t[] = {{"x", x, rows, C, ldx, 2},
                      {"w_gate", w_gate, H, C, ld_gate, 2},
                      {"w_up", w_up, H, C, ld_up, 2},
                      {"w_down", w_down, C, H, ld_down, 2},
                      {"y", y, rows, C, ldy, 2},
                      dense("saved", saved, rows, 2 * (int64_t)H, 4)};
    CF_TRY(check_aligned(what, t, 6));
    for (int i = 4; i < 6; i++)
        CF_TRY(check_out(what, t[i], t, i));
    if (!gated_fits(rows, C, H))
        return too_large(what);
    const bool plain = readable(x, ldx) && readable(w_gate, ld_gate) && readable(w_up, ld_up) &&
                       readable(w_down, ld_down) && ld_gate == ld_up;
    CF_TRY(check_ws(what, ws, ws_bytes, cf_gated_ffn_workspace_bytes(rows, C, H, plain), t, 6));
    const GatedFfn a = {{x, ldx}, {w_gate, ld_gate}, {w_up, ld_up}, {w_down, ld_down}, (int)rows, C, H, (int)act};
    return api_done(launch_gated(a, y, ldy, saved, dt == CF_BF16, ws, (hipStream_t)stream), what);
}

size_t cf_gated_ffn_backward_workspace_bytes(int64_t rows, int C, int H, int aligned) {
    return rows <= 0 || C <= 0 || H <= 0 || !gated_fits(rows, C, H)
               ? 0
               : gated_backward_workspace_bytes(rows, C, H, aligned != 0);
}

cf_status cf_gated_ffn_backward(const void *dy, const void *x, const float *saved, const void *w_gate, const void *w_up,
                                const void *w_down, void *dx, void *dw_gate, void *dw_up, void *dw_down, void *ws,
                                size_t ws_bytes, int64_t rows, int C, int H, int64_t lddy, int64_t ldx, int64_t ld_gate,
                                int64_t ld_up, int64_t ld_down, int64_t lddx, cf_dtype dt, cf_act act, void *stream) {
    const char *const what = "cf_gated_ffn_backward";
    CF_TRY(check_rows(what, rows, C, "C"));
    CF_TRY(check_rows(what, rows, H, "H"));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_any_act(what, act));
    CF_TRY(check_ld(what, "lddy", lddy, 0, rows));
    CF_TRY(check_ld(what, "ldx", ldx, 0, rows));
    CF_TRY(check_ld(what, "ld_gate", ld_gate, 0, H));
    CF_TRY(check_ld(what, "ld_up", ld_up, 0, H));
    CF_TRY(check_ld(what, "ld_down", ld_down, 0, C));
    CF_TRY(check_ld(what, "lddx", lddx, C, rows));
    if (!dw_gate || !dw_up || !dw_down)
        return api_fail(CF_ERR_INVALID, "%s: the weights' gradients must be non-NULL", what);
    if (rows > 0 && (!dy || !x || !saved || !w_gate || !w_up || !w_down || !dx))
        return api_fail(CF_ERR_INVALID, "%s: dy, x, saved, the weights and dx must be non-NULL", what);
    const Span t[] = {{"dy", dy, rows, C, lddy, 2},
                      {"x", x, rows, C, ldx, 2},
                      dense("saved", saved, rows, 2 * (int64_t)H, 4),
                      {"w_gate", w_gate, H, C, ld_gate, 2},
                      {"w_up", w_up, H, C, ld_up, 2},
                      {"w_down", w_down, C, H, ld_down, 2},
                      {"dx", dx, rows, C, lddx, 2},
                      dense("dw_gate", dw_gate, H, C, 2),
                      dense("dw_up", dw_up, H, C, 2),
                      dense("dw_down", dw_down, C, H, 2)};
    CF_TRY(check_aligned(what, t, 10));
    for (int i = 6; i < 10; i++)
        CF_TRY(check_out(what, t[i], t, i));
    if (!gated_fits(rows, C, H))
        return too_large(what);
    const bool plain = readable(dy, lddy) && readable(x, ldx) && readable(w_gate, ld_gate) && readable(w_up, ld_up) &&
                       readable(w_down, ld_down) && ld_gate == ld_up;
    CF_TRY(check_ws(what, ws, ws_bytes, cf_gated_ffn_backward_workspace_bytes(rows, C, H, plain), t, 10));
    const GatedFfn a = {{x, ldx}, {w_gate, ld_gate}, {w_up, ld_up}, {w_down, ld_down}, (int)rows, C, H, (int)act};
    const GatedGrads g = {dx, lddx, dw_gate, dw_up, dw_down};
    return api_done(launch_gated_backward(a, RowsIn{dy, lddy}, saved, g, dt == CF_BF16, ws, (hipStream_t)stream), what);
}

size_t cf_linear_log_probs_workspace_bytes(int64_t rows, int C, int V, int aligned) {
    return rows <= 0 || C <= 0 || V <= 0 || !linear_fits(rows, C, V) ? 0
                                                                      : linear_workspace_bytes(rows, C, V, aligned != 0);
}

cf_status cf_linear_log_probs_forward(const void *x, const void *weight, const int64_t *tokens, float *logp, float *lse,
                                      void *ws, size_t ws_bytes, int64_t rows, int C, int V, int64_t ldx, int64_t ldw,
                                      cf_dtype dt, void *stream) {
    const char *const what = "cf_linear_log_probs_forward";
    CF_TRY(check_rows(what, rows, C, "C"));
    CF_TRY(check_rows(what, rows, V, "V"));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_ld(what, "ldx", ldx, 0, rows));
    CF_TRY(check_ld(what, "ldw", ldw, 0, V));
    if (rows == 0)
        return api_done(hipSuccess, what);
    if (!x || !weight || !lse)
        return api_fail(CF_ERR_INVALID, "%s: x, weight and lse must be non-NULL", what);
    if (!tokens != !logp)
        return api_fail(CF_ERR_INVALID, "%s: tokens and logp go together", what);
    const Span t[] = {{"x", x, rows, C, ldx, 2},
                      {"weight", weight, V, C, ldw, 2},
                      dense("tokens", tokens, rows, 1, 8),
                      dense("logp", logp, rows, 1, 4),
                      dense("lse", lse, rows, 1, 4)};
    CF_TRY(check_aligned(what, t, 5));
    for (int i = 3; i < 5; i++)
        CF_TRY(check_out(what, t[i], t, i));
    if (!linear_fits(rows, C, V))
        return too_large(what);
    const bool plain = readable(x, ldx) && readable(weight, ldw);
    CF_TRY(check_ws(what, ws, ws_bytes, cf_linear_log_probs_workspace_bytes(rows, C, V, plain), t, 5));
    const LinearLogProbs a = {{x, ldx}, {weight, ldw}, tokens, (int)rows, C, V};
    return api_done(launch_linear_log_probs(a, logp, lse, dt == CF_BF16, ws, (hipStream_t)stream), what);
}

size_t cf_linear_log_probs_backward_workspace_bytes(int64_t rows, int C, int V, int aligned) {
    return rows <= 0 || C <= 0 || V <= 0 || !linear_fits(rows, C, V)
               ? 0
               : linear_backward_workspace_bytes(rows, C, V, aligned != 0);
}

cf_status cf_linear_log_probs_backward(const void *x, const void *weight, const int64_t *tokens, const float *logp,
                                       const float *lse, const float *d_logp, const float *d_lse, void *dx, void *dweight, void *ws,
                                       size_t ws_bytes, int64_t rows, int C, int V, int64_t ldx, int64_t ldw,
                                       int64_t lddx, cf_dtype dt, void *stream) {
    const char *const what = "cf_linear_log_probs_backward";
    CF_TRY(check_rows(what, rows, C, "C"));
    CF_TRY(check_rows(what, rows, V, "V"));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_ld(what, "ldx", ldx, 0, rows));
    CF_TRY(check_ld(what, "ldw", ldw, 0, V));
    CF_TRY(check_ld(what, "lddx", lddx, C, rows));
    if (!dweight)
        return api_fail(CF_ERR_INVALID, "%s: dweight must be non-NULL", what);
    if (rows > 0 && (!x || !weight || !lse || !dx))
        return api_fail(CF_ERR_INVALID, "%s: x, weight, lse and dx must be non-NULL", what);
    if (rows > 0 && !d_logp && !d_lse)
        return api_fail(CF_ERR_INVALID, "%s: d_logp or d_lse must be non-NULL", what);
    if (rows > 0 && d_logp && (!tokens || !logp))
        return api_fail(CF_ERR_INVALID, "%s: d_logp needs tokens and their logp", what);
    const Span t[] = {{"x", x, rows, C, ldx, 2},
                      {"weight", weight, V, C, ldw, 2},
                      dense("tokens", tokens, rows, 1, 8),
                      dense("logp", logp, rows, 1, 4),
                      dense("lse", lse, rows, 1, 4),
                      dense("d_logp", d_logp, rows, 1, 4),
                      dense("d_lse", d_lse, rows, 1, 4),
                      {"dx", dx, rows, C, lddx, 2},
                      dense("dweight", dweight, V, C, 2)};
    CF_TRY(check_aligned(what, t, 9));
    for (int i = 7; i < 9; i++)
        CF_TRY(check_out(what, t[i], t, i));
    if (!linear_fits(rows, C, V))
        return too_large(what);
    const bool plain = readable(x, ldx) && readable(weight, ldw);
    CF_TRY(check_ws(what, ws, ws_bytes, cf_linear_log_probs_backward_workspace_bytes(rows, C, V, plain), t, 9));
    const LinearLogProbs a = {{x, ldx}, {weight, ldw}, tokens, (int)rows, C, V};
    const LinearGrads g = {logp, lse, d_logp, d_lse, dx, lddx, dweight};
    return api_done(launch_linear_log_probs_backward(a, g, dt == CF_BF16, ws, (hipStream_t)stream), what);
}

}  // extern "C"
