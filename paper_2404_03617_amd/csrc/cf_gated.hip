// cf_gated.hip -- the gated feed-forward block
//
//   y = (act(x Wg^T) * (x Wu^T)) Wd^T,   x [rows][C], Wg, Wu [H][C], Wd [C][H]
//
// as two products (cf_mm.h): the first makes gate and up channels in the same
// tile and leaves h = act(g) u; the second projects h.  Backward, from dy and
// the g and u of the forward pass:
//
//   dh = dy Wd, in the same launch dg = dh u act'(g), du = dh act(g) and h again
//   dWd = dy^T h;  dWg = dg^T x, dWu = du^T x (one launch);  dx = dg Wg + du Wu (one sum)
//
// h, dg and du are rounded to the type of x for the products that read them.
//
// g and u are kept in fp32: in 16 bits they would put two more roundings into every
// gradient (its distance from 64 bits 1.4 times that of a rounded exact one, 1.7 and
// more with them).  8192 x 4096 x 12288 in bf16: gate and up 1.43 ms (1155 TFLOP/s), down
// 0.68 (1217), gradients of gate and up 1.15, dx 1.29 (1281), the weights' 0.61 and
// 1.38 (1243): what passes behind the first and the third, 1.4 GB each, is not hidden
// by their products.
#include "cf_few.h"
#include "cf_head.h"
#include "cf_mm_run.h"

namespace cf {

using namespace mm;

namespace {

// Which operands need a packed copy.  Gate and up are read with one stride.
struct Copied {
    bool x, dy, wgu, wd;
};
Copied copied_of(const GatedFfn &a, const RowsIn &dy) {
    if (a.rows == 0)  // nothing is read
        return {false, false, false, false};
    return {!fits(a.x.p, a.x.ld, a.C), !fits(dy.p, dy.ld, a.C),
            !fits(a.w_gate.p, a.w_gate.ld, a.C) || !fits(a.w_up.p, a.w_up.ld, a.C) || a.w_gate.ld != a.w_up.ld,
            !fits(a.w_down.p, a.w_down.ld, a.H)};
}
Copied copied_at_most(int C, int H, bool aligned) {
    const bool c = C % 8 != 0 || !aligned, h = H % 8 != 0 || !aligned;
    return {c, c, c, h};
}

struct ForwardPlan {
    Room room;
    Operand x, wg, wu, wd;
    int pad;
    int64_t ld, lo;  // of h; to what rounding it takes (few rows)
    uint16_t *h;
    Plan up, down;  // of more rows
    void *part;
};
ForwardPlan forward_plan(const GatedFfn &a, Copied c, void *ws) {
    static_assert(PART_ROWS == few::ROWS, "products of few rows write h in two numbers, those of more in one");
    ForwardPlan p = {};
    const bool few = a.rows <= few::ROWS;
    if (few)  // read wherever they are
        c = {};
    p.room.p = (uint8_t *)ws;
    p.pad = up8(a.H);
    p.ld = stride_of(a.H);
    p.x = operand(a.x.p, a.x.ld, a.rows, a.C, c.x, p.room);
    p.wg = operand(a.w_gate.p, a.w_gate.ld, a.H, a.C, c.wgu, p.room);
    p.wu = operand(a.w_up.p, a.w_up.ld, a.H, a.C, c.wgu, p.room);
    p.wd = operand(a.w_down.p, a.w_down.ld, a.C, a.H, c.wd, p.room);
    p.lo = few ? a.rows * p.ld : 0;
    p.h = (uint16_t *)p.room.take((size_t)(few ? 2 : 1) * a.rows * p.ld * 2);
    if (few)
        return p;
    p.up = plan(a.rows, 2 * (int64_t)a.H, a.C, true, 1, 1, MORE);
    p.down = plan(a.rows, a.C, a.H, true);
    const size_t one = part_bytes(p.up, a.rows, a.H, 2), two = part_bytes(p.down, a.rows, a.C, 1);
    p.part = p.room.take(one > two ? one : two);
    return p;
}

struct BackwardPlan {
    Room room;
    Operand x, dy, wg, wu, wd;
    int pad;
    int64_t ld, lo;  // of h; to what rounding it takes, or 0; d has two of them a row
    uint16_t *d, *h;
    Plan dh, dwd, dwu, dx;
    void *part;
};
BackwardPlan backward_plan(const GatedFfn &a, const RowsIn &dy, const Copied &c, void *ws) {
    BackwardPlan p;
    p.room.p = (uint8_t *)ws;
    p.pad = up8(a.H);
    p.ld = stride_of(a.H);
    p.x = operand(a.x.p, a.x.ld, a.rows, a.C, c.x, p.room);
    p.dy = operand(dy.p, dy.ld, a.rows, a.C, c.dy, p.room);
    p.wg = operand(a.w_gate.p, a.w_gate.ld, a.H, a.C, c.wgu, p.room);
    p.wu = operand(a.w_up.p, a.w_up.ld, a.H, a.C, c.wgu, p.room);
    p.wd = operand(a.w_down.p, a.w_down.ld, a.C, a.H, c.wd, p.room);
    const bool lo = in_parts(a.rows);
    const int64_t rows = lo ? 2 * a.rows : a.rows;
    p.lo = lo ? a.rows * p.ld : 0;
    p.d = (uint16_t *)p.room.take((size_t)rows * 2 * p.ld * 2);
    p.h = (uint16_t *)p.room.take((size_t)rows * p.ld * 2);
    p.dh = plan(a.rows, a.H, a.C, true, 1, 1, GATE);
    p.dwd = plan(a.C, a.H, a.rows, true, 1, lo ? 2 : 1);
    p.dwu = plan(a.H, a.C, a.rows, true, lo ? 1 : 2, lo ? 2 : 1);
    p.dx = plan(rows, a.C, a.H, true, 1, 2);
    size_t part = part_bytes(p.dwd, a.C, a.H, 1);
    const size_t more[] = {part_bytes(p.dwu, a.H, a.C, lo ? 1 : 2), joined_bytes(p.dx, rows, a.C, 1, lo),
                           joined_bytes(p.dh, a.rows, a.H, 1, lo)};
    for (size_t m : more)
        part = part > m ? part : m;
    p.part = p.room.take(part);
    return p;
}

template <typename T>
hipError_t forward(const GatedFfn &a, const ForwardPlan &p, void *y, int64_t ldy, float *saved, int bf16, hipStream_t st) {
    CF_HIP(pack(p.x, bf16, st));
    CF_HIP(pack(p.wg, bf16, st));
    CF_HIP(pack(p.wu, bf16, st));
    CF_HIP(pack(p.wd, bf16, st));
    if (a.rows <= few::ROWS) {
        const few::Args up = {p.x.m.p, {p.wg.m.p, p.wu.m.p}, p.x.m.ld, {p.wg.m.ld, p.wu.m.ld}, 0, a.rows, a.H, a.C};
        CF_HIP((few::launch<T, 2, few::Gated>(up, GatedArgs{p.h, p.ld, p.lo, saved, a.H, p.pad, a.act}, st)));
        StoreArgs s = {};
        s.out[0] = (uint16_t *)y;
        s.ldo = ldy;
        const few::Args down = {p.h, {p.wd.m.p, p.wd.m.p}, p.ld, {p.wd.m.ld, p.wd.m.ld}, p.lo, a.rows, a.C, a.H};
        return a.rows <= 8 ? few::launch<T, 1, few::Store<true>>(down, s, st)
                           : few::launch<T, 1, few::Store<false>>(down, s, st);
    }
    const GatedArgs gate = {p.h, p.ld, 0, saved, a.H, p.pad, a.act};
    const bool split = p.up.splits > 1;
    Args up = args_of(p.up, a.rows, split ? a.H : 2 * a.H, a.C, p.x.m, a.rows, p.wg.m, a.H, false, split ? 2 : 1);
    up.b[1] = p.wu.m.p;
    if (split)
        CF_HIP((run_split<KC, KC>(up, gate, p.up, p.part, bf16, st)));
    else
        CF_HIP(launch_gated<T>(up, gate, p.up.tile, st));
    StoreArgs s = {};
    s.out[0] = s.out[1] = (uint16_t *)y;
    s.ldo = ldy;
    return run_store<KC, KC>(args_of(p.down, a.rows, a.C, a.H, Matrix{p.h, p.ld, p.pad}, a.rows, p.wd.m, a.C), s, p.down,
                             p.part, bf16, st);
}

template <typename T>
hipError_t backward(const GatedFfn &a, const BackwardPlan &p, const float *saved, const GatedGrads &g, int bf16,
                    hipStream_t st) {
    CF_HIP(pack(p.x, bf16, st));
    CF_HIP(pack(p.dy, bf16, st));
    CF_HIP(pack(p.wg, bf16, st));
    CF_HIP(pack(p.wu, bf16, st));
    CF_HIP(pack(p.wd, bf16, st));
    const Matrix h = {p.h, p.ld, p.pad}, d = {p.d, 2 * p.ld, p.pad};
    if (a.rows > 0) {
        const Args dh = args_of(p.dh, a.rows, a.H, a.C, p.dy.m, a.rows, p.wd.m, p.wd.m.ext);
        const GatedBackArgs e = {saved, p.d, p.h, p.ld, p.lo, a.H, p.pad, a.act};
        if (p.dh.splits > 1 || p.lo)
            CF_HIP((run_split<KC, RC>(dh, e, p.dh, p.part, bf16, st)));
        else
            CF_HIP(launch_gated_back<T>(dh, e, p.dh.tile, st));
        const int rows = p.lo ? 2 * a.rows : a.rows;
        Args dx = args_of(p.dx, rows, a.C, a.H, d, rows, p.wg.m, p.wg.m.ext, true);
        dx.a[1] = p.d + p.ld;
        dx.b[1] = p.wu.m.p;
        StoreArgs s = {};
        s.out[0] = s.out[1] = (uint16_t *)g.dx;
        s.ldo = g.lddx;
        s.fold = p.lo ? a.rows : 0;
        CF_HIP((run_store<KC, RC>(dx, s, p.dx, p.part, bf16, st)));
    }
    StoreArgs s = {};
    s.out[0] = s.out[1] = (uint16_t *)g.dw_down;
    s.ldo = a.H;
    Args down = args_of(p.dwd, a.C, a.H, a.rows, p.dy.m, p.dy.m.ext, h, p.pad, p.lo != 0);
    down.b[1] = p.h + p.lo;
    CF_HIP((run_store<RC, RC>(down, s, p.dwd, p.part, bf16, st)));
    s.ldo = a.C;
    if (p.lo) {
        for (int i = 0; i < 2; i++) {
            const Matrix di = {p.d + i * p.ld, 2 * p.ld, p.pad};
            Args w = args_of(p.dwu, a.H, a.C, a.rows, di, p.pad, p.x.m, p.x.m.ext, true);
            w.a[1] = di.p + 2 * p.lo;
            s.out[0] = (uint16_t *)(i ? g.dw_up : g.dw_gate);
            CF_HIP((run_store<RC, RC>(w, s, p.dwu, p.part, bf16, st)));
        }
        return hipSuccess;
    }
    Args w = args_of(p.dwu, a.H, a.C, a.rows, d, p.pad, p.x.m, p.x.m.ext, false, 2);
    w.a[1] = p.d + p.ld;
    s.out[0] = (uint16_t *)g.dw_gate;
    s.out[1] = (uint16_t *)g.dw_up;
    return run_store<RC, RC>(w, s, p.dwu, p.part, bf16, st);
}

}  // namespace

bool products_read(const void *p, int64_t ld, int cols) { return fits(p, ld, cols); }

bool gated_fits(int64_t rows, int C, int H) {
    return rows < (int64_t)1 << 30 && C <= 1 << 20 && H <= 1 << 20 && grid_fits(rows, C) && grid_fits(rows, 2 * (int64_t)H) &&
           grid_fits(2 * (int64_t)H, C) && pack_fits(rows, C) && pack_fits(H, C) && pack_fits(C, H);
}

size_t gated_workspace_bytes(int64_t rows, int C, int H, bool aligned) {
    GatedFfn a = {};
    a.rows = (int)rows;
    a.C = C;
    a.H = H;
    return forward_plan(a, copied_at_most(C, H, aligned), nullptr).room.used;
}

size_t gated_backward_workspace_bytes(int64_t rows, int C, int H, bool aligned) {
    GatedFfn a = {};
    a.rows = (int)rows;
    a.C = C;
    a.H = H;
    return backward_plan(a, RowsIn{}, copied_at_most(C, H, aligned), nullptr).room.used;
}

hipError_t launch_gated(const GatedFfn &a, void *y, int64_t ldy, float *saved, int bf16, void *ws, hipStream_t st) {
    const ForwardPlan p = forward_plan(a, copied_of(a, a.x), ws);
    return bf16 ? forward<BF16>(a, p, y, ldy, saved, bf16, st) : forward<F16>(a, p, y, ldy, saved, bf16, st);
}

hipError_t launch_gated_backward(const GatedFfn &a, RowsIn dy, const float *saved, const GatedGrads &g, int bf16,
                                 void *ws, hipStream_t st) {
    const BackwardPlan p = backward_plan(a, dy, copied_of(a, dy), ws);
    return bf16 ? backward<BF16>(a, p, saved, g, bf16, st) : backward<F16>(a, p, saved, g, bf16, st);
}

}  // namespace cf
