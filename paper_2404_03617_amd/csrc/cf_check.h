// cf_check.h -- argument checks that the C ABI's operators on rows share
// (cf_train_api.hip, cf_head_api.hip).
#pragma once

#include "cf_api.h"

namespace cf {

inline bool aligned(const void *p, size_t n) { return ((uintptr_t)p & (n - 1)) == 0; }

// The memory of a [rows][cols] tensor with a row stride, in elements of `size`.
struct Span {
    const char *name;
    const void *p;
    int64_t rows, cols, ld;
    size_t size;
};

inline uintptr_t end_of(const Span &s) {
    return (uintptr_t)s.p + (size_t)(((s.rows > 0 ? s.rows - 1 : 0) * s.ld + s.cols) * (int64_t)s.size);
}

// Whether two tensors share bytes.  Views of one buffer with the same row
// stride do not where their columns are apart.
inline bool share(const Span &a, const Span &b) {
    if (!a.p || !b.p || a.rows <= 0 || b.rows <= 0)
        return false;
    const uintptr_t a0 = (uintptr_t)a.p, b0 = (uintptr_t)b.p;
    if (a0 >= end_of(b) || b0 >= end_of(a))
        return false;
    const uint64_t pitch = (uint64_t)a.ld * a.size;
    if (pitch == 0 || pitch != (uint64_t)b.ld * b.size || (uint64_t)a.cols * a.size > pitch ||
        (uint64_t)b.cols * b.size > pitch)
        return true;
    const uint64_t na = (uint64_t)a.cols * a.size, nb = (uint64_t)b.cols * b.size;
    const uint64_t d = a0 <= b0 ? (b0 - a0) % pitch : (a0 - b0) % pitch;  // columns of the later past the earlier's
    const uint64_t first = a0 <= b0 ? na : nb, second = a0 <= b0 ? nb : na;
    return d < first || d + second > pitch;
}

// An output against the other tensors of the call; `same` is the input that it
// may equal.
inline cf_status check_out(const char *what, const Span &out, const Span *others, int n, const char *same = "") {
    for (int i = 0; i < n; i++) {
        const Span &o = others[i];
        const bool in_place = o.name == same && o.p == out.p && (o.ld == out.ld || out.rows <= 1);
        if (!in_place && share(out, o))
            return api_fail(CF_ERR_INVALID, "%s: %s and %s overlap", what, out.name, o.name);
    }
    return CF_OK;
}

// Sizes and strides of [rows][C] tensors.
inline cf_status check_rows(const char *what, int64_t rows, int C, const char *c_name) {
    if (rows < 0 || C <= 0)
        return api_fail(CF_ERR_INVALID, "%s: rows must not be negative and %s must be positive (rows=%lld %s=%d)",
                        what, c_name, (long long)rows, c_name, C);
    if ((double)rows * C > 4.0e12)
        return api_fail(CF_ERR_INVALID, "%s: tensor too large", what);
    return CF_OK;
}

inline cf_status check_ld(const char *what, const char *name, int64_t ld, int64_t least, int64_t rows) {
    if (ld < least)
        return api_fail(CF_ERR_INVALID, "%s: %s=%lld must be at least %lld", what, name, (long long)ld,
                        (long long)least);
    if ((double)ld * (double)rows > 4.0e12)
        return api_fail(CF_ERR_INVALID, "%s: tensor too large", what);
    return CF_OK;
}

inline cf_status check_dtype(const char *what, int dt, int most) {
    if (dt < 0 || dt > most)
        return api_fail(CF_ERR_INVALID, "%s: unknown dtype %d", what, dt);
    return CF_OK;
}

inline cf_status check_act(const char *what, cf_act act) {
    if ((int)act != CF_ACT_GELU_ERF && (int)act != CF_ACT_RELU && (int)act != CF_ACT_NONE)
        return api_fail(CF_ERR_INVALID, "%s: unknown activation %d", what, (int)act);
    return CF_OK;
}

inline cf_status check_aligned(const char *what, const Span *t, int n) {
    for (int i = 0; i < n; i++)
        if (t[i].p && !aligned(t[i].p, t[i].size))
            return api_fail(CF_ERR_INVALID, "%s: %s is not aligned to its elements", what, t[i].name);
    return CF_OK;
}

// A workspace of `need` bytes, and the others apart from it.
inline cf_status check_ws(const char *what, const void *ws, size_t ws_bytes, size_t need, const Span *others, int n) {
    if (need == 0)
        return CF_OK;
    if (!ws || ws_bytes < need)
        return api_fail(CF_ERR_WORKSPACE, "%s: ws has %zu bytes, needs %zu", what, ws ? ws_bytes : (size_t)0, need);
    if (!aligned(ws, 16))
        return api_fail(CF_ERR_INVALID, "%s: ws must be 16-byte aligned", what);
    return check_out(what, Span{"ws", ws, 1, (int64_t)need, (int64_t)need, 1}, others, n);
}

inline Span dense(const char *name, const void *p, int64_t rows, int64_t cols, size_t size) {
    return Span{name, p, rows, cols, cols, size};
}

#define CF_TRY(call)                                                                                                   \
    do {                                                                                                               \
        const cf_status st_ = (call);                                                                                  \
        if (st_ != CF_OK)                                                                                              \
            return st_;                                                                                                \
    } while (0)

}  // namespace cf
