// cf_train_api.hip -- the C ABI of the training and scoring operators:
// argument validation on the host (no HIP call before every check has
// passed), then their launchers.
#include "cf_check.h"
#include "cf_train.h"

namespace {

using namespace cf;

int64_t scales_of(int C) { return (C + CF_CKPT_BLOCK - 1) / CF_CKPT_BLOCK; }

// h = act(u) and the checkpoints of both
cf_status act_forward(const char *what, const void *u, void *h, int8_t *qu, float *scale_u, int8_t *qh,
                      float *scale_h, int64_t rows, int C, int64_t ldu, int64_t ldh, cf_dtype dt, cf_act act,
                      void *stream) {
    CF_TRY(check_rows(what, rows, C, "C"));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_act(what, act));
    CF_TRY(check_ld(what, "row stride", ldu, 0, rows));
    if (h)
        CF_TRY(check_ld(what, "ldh", ldh, C, rows));
    if (rows == 0)
        return api_done(hipSuccess, what);
    if (!u || (!h && !qu && !qh))
        return api_fail(CF_ERR_INVALID, "%s: the input and an output must be non-NULL", what);
    if (!qu != !scale_u || !qh != !scale_h)
        return api_fail(CF_ERR_INVALID, "%s: a checkpoint needs both q and scale", what);
    const Span in = {"u", u, rows, C, ldu, 2};
    const Span t[] = {in,
                      {"h", h, rows, C, ldh, 2},
                      dense("qu", qu, rows, C, 1),
                      dense("scale_u", scale_u, rows, scales_of(C), 4),
                      dense("qh", qh, rows, C, 1),
                      dense("scale_h", scale_h, rows, scales_of(C), 4)};
    CF_TRY(check_aligned(what, t, 6));
    for (int i = 1; i < 6; i++)
        CF_TRY(check_out(what, t[i], t, i, i == 1 ? in.name : ""));
    if (!cf::act_fits(rows, C))
        return api_fail(CF_ERR_UNSUPPORTED, "%s: rows * ceil(C/64) * 8 must stay below 2^31", what);
    return api_done(cf::launch_act_forward(u, ldu, h, ldh, cf::Ckpt{qu, scale_u}, cf::Ckpt{qh, scale_h}, rows, C,
                                           (int)act, dt == CF_BF16, (hipStream_t)stream),
                    what);
}

// du = dh act'(u), or (no dh) the values of u
cf_status act_backward(const char *what, const void *dh, const int8_t *qu, const float *scale_u, void *du,
                       int64_t rows, int C, int64_t lddh, int64_t lddu, cf_dtype dt, cf_act act, bool needs_dh,
                       void *stream) {
    CF_TRY(check_rows(what, rows, C, "C"));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_act(what, act));
    if (needs_dh)
        CF_TRY(check_ld(what, "lddh", lddh, 0, rows));
    CF_TRY(check_ld(what, "row stride", lddu, C, rows));
    if (rows == 0)
        return api_done(hipSuccess, what);
    if (!qu || !scale_u || !du || (needs_dh && !dh))
        return api_fail(CF_ERR_INVALID, "%s: the inputs and the output must be non-NULL", what);
    const Span t[] = {{"dh", dh, rows, C, lddh, 2},
                      dense("q", qu, rows, C, 1),
                      dense("scale", scale_u, rows, scales_of(C), 4),
                      {"the output", du, rows, C, lddu, 2}};
    CF_TRY(check_aligned(what, t, 4));
    CF_TRY(check_out(what, t[3], t, 3, t[0].name));
    if (!cf::act_fits(rows, C))
        return api_fail(CF_ERR_UNSUPPORTED, "%s: rows * ceil(C/64) * 8 must stay below 2^31", what);
    return api_done(cf::launch_act_backward(dh, lddh, cf::CkptIn{qu, scale_u}, du, lddu, rows, C, (int)act,
                                            dt == CF_BF16, (hipStream_t)stream),
                    what);
}

}  // namespace

extern "C" {

cf_status cf_layer_norm_forward(const void *x, void *y, const float *weight, const float *bias, float *stats,
                                int8_t *q, float *scale, int64_t rows, int C, int64_t ldx, int64_t ldy, float eps,
                                cf_dtype dt, void *stream) {
    const char *const what = "cf_layer_norm_forward";
    CF_TRY(check_rows(what, rows, C, "C"));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_ld(what, "ldx", ldx, 0, rows));
    CF_TRY(check_ld(what, "ldy", ldy, C, rows));
    if (!(eps >= 0.0f) || eps > 1.0e30f)
        return api_fail(CF_ERR_INVALID, "%s: eps must be a finite number that is not negative", what);
    if (rows == 0)
        return api_done(hipSuccess, what);
    if (!x || !y)
        return api_fail(CF_ERR_INVALID, "%s: x and y must be non-NULL", what);
    if (!q != !scale)
        return api_fail(CF_ERR_INVALID, "%s: a checkpoint needs both q and scale", what);
    const Span t[] = {{"x", x, rows, C, ldx, 2},
                      dense("weight", weight, 1, C, 4),
                      dense("bias", bias, 1, C, 4),
                      {"y", y, rows, C, ldy, 2},
                      dense("stats", stats, rows, 2, 4),
                      dense("q", q, rows, C, 1),
                      dense("scale", scale, rows, scales_of(C), 4)};
    CF_TRY(check_aligned(what, t, 7));
    if (!aligned(stats, 8))
        return api_fail(CF_ERR_INVALID, "%s: stats must be 8-byte aligned", what);
    for (int i = 3; i < 7; i++)
        CF_TRY(check_out(what, t[i], t, i, i == 3 ? t[0].name : ""));
    if (!cf::norm_fits(rows, C))
        return api_fail(CF_ERR_UNSUPPORTED, "%s: no kernel for rows=%lld C=%d (C up to %d, rows * C / 8 below 2^32)",
                        what, (long long)rows, C, CF_NORM_MAX_C);
    return api_done(cf::launch_norm_forward(x, ldx, y, ldy, weight, bias, stats, cf::Ckpt{q, scale}, rows, C, eps,
                                            dt == CF_BF16, (hipStream_t)stream),
                    what);
}

size_t cf_layer_norm_backward_workspace_bytes(int64_t rows, int C) {
    return rows <= 0 || C <= 0 || C > CF_NORM_MAX_C ? 0 : cf::norm_backward_workspace_bytes(rows, C);
}

cf_status cf_layer_norm_backward(const void *dy, const void *x, const int8_t *q, const float *scale,
                                 const float *stats, const float *weight, void *dx, float *dweight, float *dbias,
                                 void *ws, size_t ws_bytes, int64_t rows, int C, int64_t lddy, int64_t ldx,
                                 int64_t lddx, cf_dtype dt, void *stream) {
    const char *const what = "cf_layer_norm_backward";
    CF_TRY(check_rows(what, rows, C, "C"));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_ld(what, "lddy", lddy, 0, rows));
    if (x)
        CF_TRY(check_ld(what, "ldx", ldx, 0, rows));
    CF_TRY(check_ld(what, "lddx", lddx, C, rows));
    if (!dweight != !dbias)
        return api_fail(CF_ERR_INVALID, "%s: dweight and dbias go together", what);
    if (rows > 0 && (!dy || !stats || !dx))
        return api_fail(CF_ERR_INVALID, "%s: dy, stats and dx must be non-NULL", what);
    if (rows > 0 && (!x == !q || !q != !scale))
        return api_fail(CF_ERR_INVALID, "%s: give x, or q and scale", what);
    const Span t[] = {{"dy", dy, rows, C, lddy, 2},
                      {"x", x, rows, C, ldx, 2},
                      dense("q", q, rows, C, 1),
                      dense("scale", scale, rows, scales_of(C), 4),
                      dense("stats", stats, rows, 2, 4),
                      dense("weight", weight, 1, C, 4),
                      {"dx", dx, rows, C, lddx, 2},
                      dense("dweight", dweight, 1, C, 4),
                      dense("dbias", dbias, 1, C, 4)};
    CF_TRY(check_aligned(what, t, 9));
    if (!aligned(stats, 8))
        return api_fail(CF_ERR_INVALID, "%s: stats must be 8-byte aligned", what);
    for (int i = 6; i < 9; i++)
        CF_TRY(check_out(what, t[i], t, i, i == 6 ? t[0].name : ""));
    if (!cf::norm_fits(rows, C))
        return api_fail(CF_ERR_UNSUPPORTED, "%s: no kernel for rows=%lld C=%d (C up to %d, rows * C / 8 below 2^32)",
                        what, (long long)rows, C, CF_NORM_MAX_C);
    if (rows == 0 && !dweight)
        return api_done(hipSuccess, what);
    const size_t need = dweight ? cf_layer_norm_backward_workspace_bytes(rows, C) : 0;
    CF_TRY(check_ws(what, ws, ws_bytes, need, t, 9));
    cf::NormBackward a;
    a.dy = dy;
    a.lddy = lddy;
    a.x = x;
    a.ldx = ldx;
    a.ckpt = cf::CkptIn{q, scale};
    a.stats = stats;
    a.weight = weight;
    a.dx = dx;
    a.lddx = lddx;
    a.dweight = dweight;
    a.dbias = dbias;
    return api_done(cf::launch_norm_backward(a, rows, C, dt == CF_BF16, ws, (hipStream_t)stream), what);
}

cf_status cf_checkpoint_pack(const void *x, int8_t *q, float *scale, int64_t rows, int C, int64_t ldx, cf_dtype dt,
                             void *stream) {
    return act_forward("cf_checkpoint_pack", x, nullptr, q, scale, nullptr, nullptr, rows, C, ldx, C, dt, CF_ACT_NONE,
                       stream);
}

cf_status cf_checkpoint_unpack(const int8_t *q, const float *scale, void *x, int64_t rows, int C, int64_t ldx,
                               cf_dtype dt, void *stream) {
    return act_backward("cf_checkpoint_unpack", nullptr, q, scale, x, rows, C, 0, ldx, dt, CF_ACT_NONE, false, stream);
}

cf_status cf_act_forward(const void *u, void *h, int8_t *qu, float *scale_u, int8_t *qh, float *scale_h, int64_t rows,
                         int C, int64_t ldu, int64_t ldh, cf_dtype dt, cf_act act, void *stream) {
    return act_forward("cf_act_forward", u, h, qu, scale_u, qh, scale_h, rows, C, ldu, ldh, dt, act, stream);
}

cf_status cf_act_backward(const void *dh, const int8_t *qu, const float *scale_u, void *du, int64_t rows, int C,
                          int64_t lddh, int64_t lddu, cf_dtype dt, cf_act act, void *stream) {
    return act_backward("cf_act_backward", dh, qu, scale_u, du, rows, C, lddh, lddu, dt, act, true, stream);
}

size_t cf_linear_weight_grad_workspace_bytes(int64_t rows, int K, int C) {
    return rows <= 0 || K <= 0 || C <= 0 || K > 1 << 20 || C > 1 << 20 ? 0 : cf::wgrad_workspace_bytes(rows, K, C);
}

cf_status cf_linear_weight_grad(const void *dy, const int8_t *q, const float *scale, const float *stats,
                                const float *weight, const float *bias, void *dw, float *db, void *ws,
                                size_t ws_bytes, int64_t rows, int K, int C, int64_t lddy, cf_dtype dt,
                                void *stream) {
    const char *const what = "cf_linear_weight_grad";
    CF_TRY(check_rows(what, rows, C, "C"));
    CF_TRY(check_rows(what, rows, K, "K"));
    CF_TRY(check_dtype(what, (int)dt, CF_BF16));
    CF_TRY(check_ld(what, "lddy", lddy, 0, rows));
    if (!dw || !db)
        return api_fail(CF_ERR_INVALID, "%s: dw and db must be non-NULL", what);
    if (rows > 0 && (!dy || !q || !scale))
        return api_fail(CF_ERR_INVALID, "%s: dy, q and scale must be non-NULL", what);
    if (rows > 0 && !stats && (weight || bias))
        return api_fail(CF_ERR_INVALID, "%s: weight and bias are the layer norm's and need stats", what);
    const Span t[] = {{"dy", dy, rows, K, lddy, 2},
                      dense("q", q, rows, C, 1),
                      dense("scale", scale, rows, scales_of(C), 4),
                      dense("stats", stats, rows, 2, 4),
                      dense("weight", weight, 1, C, 4),
                      dense("bias", bias, 1, C, 4),
                      dense("dw", dw, K, C, 2),
                      dense("db", db, 1, K, 4)};
    CF_TRY(check_aligned(what, t, 8));
    if (!aligned(stats, 8))
        return api_fail(CF_ERR_INVALID, "%s: stats must be 8-byte aligned", what);
    for (int i = 6; i < 8; i++)
        CF_TRY(check_out(what, t[i], t, i));
    if (K > 1 << 20 || C > 1 << 20)
        return api_fail(CF_ERR_UNSUPPORTED, "%s: K=%d and C=%d must be at most 2^20", what, K, C);
    CF_TRY(check_ws(what, ws, ws_bytes, cf_linear_weight_grad_workspace_bytes(rows, K, C), t, 8));
    cf::WGrad a;
    a.dy = dy;
    a.lddy = lddy;
    a.x = cf::CkptIn{q, scale};
    a.stats = stats;
    a.weight = weight;
    a.bias = bias;
    a.dw = dw;
    a.db = db;
    return api_done(cf::launch_wgrad(a, rows, K, C, dt == CF_BF16, ws, (hipStream_t)stream), what);
}

size_t cf_log_probs_workspace_bytes(int64_t rows, int V, int top) {
    return rows <= 0 || V <= 0 || V > 1 << 30 || top < 0 || top > CF_TOP_MAX
               ? 0
               : cf::log_probs_workspace_bytes(rows, V, top);
}

cf_status cf_log_probs_forward(const void *z, const int64_t *tokens, float *logp, float *entropy, float *stats,
                               float *top_logp, int64_t *top_ids, int top, void *ws, size_t ws_bytes, int64_t rows,
                               int V, int64_t ldz, cf_logits_dtype dt, void *stream) {
    const char *const what = "cf_log_probs_forward";
    CF_TRY(check_rows(what, rows, V, "V"));
    CF_TRY(check_dtype(what, (int)dt, CF_LOGITS_F32));
    CF_TRY(check_ld(what, "ldz", ldz, 0, rows));
    if (top < 0 || top > V)
        return api_fail(CF_ERR_INVALID, "%s: top=%d must be between 0 and V=%d", what, top, V);
    if (top > CF_TOP_MAX)
        return api_fail(CF_ERR_UNSUPPORTED, "%s: top=%d must be at most %d", what, top, CF_TOP_MAX);
    if (rows == 0)
        return api_done(hipSuccess, what);
    if (!z || !entropy)
        return api_fail(CF_ERR_INVALID, "%s: z and entropy must be non-NULL", what);
    if (!tokens != !logp)
        return api_fail(CF_ERR_INVALID, "%s: tokens and logp go together", what);
    if ((top > 0) != (top_logp != nullptr) || (top > 0) != (top_ids != nullptr))
        return api_fail(CF_ERR_INVALID, "%s: top_logp and top_ids go with top > 0", what);
    const Span t[] = {{"z", z, rows, V, ldz, dt == CF_LOGITS_F32 ? (size_t)4 : (size_t)2},
                      dense("tokens", tokens, rows, 1, 8),
                      dense("logp", logp, rows, 1, 4),
                      dense("entropy", entropy, rows, 1, 4),
                      dense("stats", stats, rows, 2, 4),
                      dense("top_logp", top_logp, rows, top, 4),
                      dense("top_ids", top_ids, rows, top, 8)};
    CF_TRY(check_aligned(what, t, 7));
    if (!aligned(stats, 8))
        return api_fail(CF_ERR_INVALID, "%s: stats must be 8-byte aligned", what);
    for (int i = 2; i < 7; i++)
        CF_TRY(check_out(what, t[i], t, i));
    if (V > 1 << 30 || !cf::log_probs_fit(rows, V))
        return api_fail(CF_ERR_UNSUPPORTED, "%s: no kernel for rows=%lld V=%d", what, (long long)rows, V);
    CF_TRY(check_ws(what, ws, ws_bytes, cf_log_probs_workspace_bytes(rows, V, top), t, 7));
    cf::LogProbs a;
    a.z = z;
    a.ldz = ldz;
    a.tokens = tokens;
    a.logp = logp;
    a.entropy = entropy;
    a.stats = stats;
    a.top_logp = top_logp;
    a.top_ids = top_ids;
    return api_done(cf::launch_log_probs(a, rows, V, top, (int)dt, ws, (hipStream_t)stream), what);
}

cf_status cf_log_probs_backward(const void *z, const int64_t *tokens, const float *stats, const float *entropy,
                                const float *d_logp, const float *d_entropy, void *dz, int64_t rows, int V,
                                int64_t ldz, int64_t lddz, cf_logits_dtype dt, void *stream) {
    const char *const what = "cf_log_probs_backward";
    CF_TRY(check_rows(what, rows, V, "V"));
    CF_TRY(check_dtype(what, (int)dt, CF_LOGITS_F32));
    CF_TRY(check_ld(what, "ldz", ldz, 0, rows));
    CF_TRY(check_ld(what, "lddz", lddz, V, rows));
    if (rows == 0)
        return api_done(hipSuccess, what);
    if (!z || !stats || !entropy || !dz)
        return api_fail(CF_ERR_INVALID, "%s: z, stats, entropy and dz must be non-NULL", what);
    if (!d_logp && !d_entropy)
        return api_fail(CF_ERR_INVALID, "%s: d_logp or d_entropy must be non-NULL", what);
    if (d_logp && !tokens)
        return api_fail(CF_ERR_INVALID, "%s: d_logp needs tokens", what);
    const size_t size = dt == CF_LOGITS_F32 ? 4 : 2;
    const Span t[] = {{"z", z, rows, V, ldz, size},
                      dense("tokens", tokens, rows, 1, 8),
                      dense("stats", stats, rows, 2, 4),
                      dense("entropy", entropy, rows, 1, 4),
                      dense("d_logp", d_logp, rows, 1, 4),
                      dense("d_entropy", d_entropy, rows, 1, 4),
                      {"dz", dz, rows, V, lddz, size}};
    CF_TRY(check_aligned(what, t, 7));
    if (!aligned(stats, 8))
        return api_fail(CF_ERR_INVALID, "%s: stats must be 8-byte aligned", what);
    CF_TRY(check_out(what, t[6], t, 6, t[0].name));
    cf::LogProbsBackward a;
    a.z = z;
    a.ldz = ldz;
    a.tokens = tokens;
    a.stats = stats;
    a.entropy = entropy;
    a.d_logp = d_logp;
    a.d_entropy = d_entropy;
    a.dz = dz;
    a.lddz = lddz;
    if (V > 1 << 30 || !cf::log_probs_backward_fits(a, rows, V, (int)dt))
        return api_fail(CF_ERR_UNSUPPORTED, "%s: no kernel for rows=%lld V=%d", what, (long long)rows, V);
    return api_done(cf::launch_log_probs_backward(a, rows, V, (int)dt, (hipStream_t)stream), what);
}

}  // extern "C"
