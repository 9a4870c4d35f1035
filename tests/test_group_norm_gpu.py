"""Group norm with an activation, forward and backward, against its definition
in 64 bits.  Tolerances: every sum in fp32 has an error of at most its longest
chain of additions (CHAIN) times 2^-24 of the sum of magnitudes; the rest is
first-order propagation of those, and one rounding to 16 bits."""
import math

import pytest
import torch

import paper_2404_03617_amd as cf

from _rows import DT, F32, ROUND, TINY, assert_within, randn

pytestmark = pytest.mark.gpu
CHAIN = 160  # additions one after the other: 16 vectors, 64 rows of a part, 64 parts, and lanes or channels of a group
ACT_ERROR = 4e-7  # of an activation and its slope in fp32, relative to max(1, |u|)


def act_of(u, act):
    """act(u), act'(u), and a bound of |act''| (or of the jump of the slope at 0)."""
    if act == "silu":
        s = torch.sigmoid(u)
        return u * s, s * (1 + u * (1 - s)), 0.5
    if act == "gelu":
        p = torch.special.ndtr(u)
        return u * p, p + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi), 0.8
    if act == "relu":
        return u.clamp_min(0), (u > 0).double(), 0.0
    return u, torch.ones_like(u), 0.0


def reference(x, dy, groups, w, b, eps, act):
    """x, dy [N, P, C] in 64 bits: (results, tolerances without the rounding to 16 bits) of y, dx, dw, db."""
    N, P, C = x.shape
    D = C // groups
    v = x.view(N, P, groups, D)
    n = P * D

    def avg(t):
        return t.mean((1, 3), keepdim=True)

    mean = avg(v)
    d = v - mean
    var = avg(d * d)
    rstd = 1 / torch.sqrt(var + eps)
    xh = d * rstd
    # the mean is off by e_mean, each difference by that and a rounding; the sum of squares by twice that and its own chain
    e_mean = CHAIN * F32 * avg(v.abs())
    e_d = e_mean + F32 * d.abs()
    e_var = 2 * avg(d.abs() * e_d) + CHAIN * F32 * var
    e_rstd = rstd * (0.5 * e_var / (var + eps) + 4 * F32)
    e_xh = e_d * rstd + d.abs() * e_rstd + F32 * xh.abs()
    wv, bv = w.view(groups, D), b.view(groups, D)
    u = xh * wv + bv
    e_u = e_xh * wv.abs() + 2 * F32 * (u.abs() + (xh * wv).abs())
    f, slope, bend = act_of(u, act)
    e_f = 1.13 * e_u + ACT_ERROR * u.abs().clamp_min(1)
    if dy is None:
        return [(f.reshape(N, P, C), e_f.reshape(N, P, C))]
    g0 = dy.view(v.shape)
    du = g0 * slope
    e_slope = bend * e_u + ACT_ERROR
    if act == "relu":
        e_slope = e_slope + (u.abs() <= e_u)
    e_du = g0.abs() * e_slope + F32 * du.abs()
    g = du * wv
    e_g = e_du * wv.abs() + F32 * g.abs()
    ga, gb = avg(g), avg(g * xh)
    e_ga = avg(e_g) + CHAIN * F32 * avg(g.abs())
    e_gb = avg(e_g * xh.abs() + g.abs() * e_xh) + CHAIN * F32 * avg((g * xh).abs())
    inner = g - ga - xh * gb
    size = g.abs() + ga.abs() + (xh * gb).abs()
    dx = rstd * inner
    e_dx = rstd * (e_g + e_ga + e_xh * gb.abs() + xh.abs() * e_gb + 4 * F32 * size) + e_rstd * inner.abs()
    more = CHAIN + N  # images are added too
    dw, db = (du * xh).sum((0, 1)).flatten(), du.sum((0, 1)).flatten()
    e_dw = (e_du * xh.abs() + du.abs() * e_xh + more * F32 * (du * xh).abs()).sum((0, 1)).flatten()
    e_db = (e_du + more * F32 * du.abs()).sum((0, 1)).flatten()
    return [(f.reshape(N, P, C), e_f.reshape(N, P, C)), (dx.reshape(N, P, C), e_dx.reshape(N, P, C)), (dw, e_dw), (db, e_db)]


def place(kind, t):
    """A tensor [N, .., C] dense, as channels of a wider one, or from an odd element on."""
    if kind == "dense":
        return t.cuda()
    C = t.shape[-1]
    if kind == "slice":
        wide = torch.full((*t.shape[:-1], C + 11), float("nan"), dtype=t.dtype, device="cuda")
        wide[..., 3:3 + C] = t.cuda()
        return wide[..., 3:3 + C]
    flat = torch.full((t.numel() + 1,), float("nan"), dtype=t.dtype, device="cuda")
    flat[1:] = t.cuda().reshape(-1)
    return flat[1:].view(t.shape)


def inputs(seed, shape, dt):
    C = shape[-1]
    x = (randn(seed, shape) * torch.exp(0.5 * randn(seed + 1, (C,))) + 0.3 * randn(seed + 2, (C,))).to(dt)
    return x, (0.1 * randn(seed + 3, shape)).to(dt), 0.5 + randn(seed + 4, (C,)).abs(), 0.2 * randn(seed + 5, (C,))


def check(x, dy, groups, w, b, act, kind="dense", eps=1e-6):
    shape, dt = x.shape, x.dtype
    N, C = shape[0], shape[-1]
    print("group norm", tuple(shape), groups, dt, act, kind, flush=True)
    wd = torch.ones(C).double() if w is None else w.double()
    bd = torch.zeros(C).double() if b is None else b.double()
    ref = reference(x.double().view(N, -1, C), dy.double().view(N, -1, C), groups, wd, bd, eps, act)
    xg, dyg = place(kind, x), place(kind, dy)
    wg, bg = None if w is None else w.cuda(), None if b is None else b.cuda()
    out = place(kind, torch.zeros_like(x))
    y, stats = cf.group_norm_forward_save(xg, groups, wg, bg, eps=eps, act=act, out=out)
    assert y is out and torch.equal(cf.group_norm_forward(xg, groups, wg, bg, eps=eps, act=act), y)
    dx, dw, db = cf.group_norm_backward(dyg, xg, stats, wg, bg, act=act)
    assert y.shape == shape and dx.shape == shape and stats.shape == (N, groups, 2)
    for got, (want, tol), what in zip((y, dx, dw, db), ref, ("y", "dx", "dweight", "dbias")):
        if what in ("y", "dx"):
            tol = (tol + ROUND[dt] * (want.abs() + tol) + TINY[dt]).view(shape)
            want = want.view(shape)
        assert_within(got, want, tol + 1e-30, what)
    # the parameters' gradients are a choice, and results repeat
    only, none, _ = cf.group_norm_backward(dyg, xg, stats, wg, bg, act=act, param_grads=False)
    again = cf.group_norm_backward(dyg, xg, stats, wg, bg, act=act)
    assert none is None and torch.equal(only, dx)
    assert all(torch.equal(p, q) for p, q in zip(again, (dx, dw, db)))
    return y, stats


SHAPES = [((1, 7, 7, 512), 32), ((2, 1, 8), 1), ((1, 1, 1, 5), 5), ((3, 5, 3, 12), 3), ((2, 9, 99), 9),
          ((1, 40, 37, 66), 6), ((2, 64, 64, 48), 4), ((5, 16), 4), ((4, 1), 1), ((1, 3, 4096), 1), ((2, 3, 2000), 2),
          ((2, 11, 2047), 89), ((1, 2, 3, 4, 40), 8), ((3, 1025, 8), 8), ((70, 4, 4, 64), 16), ((1, 100, 110, 24), 2)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("shape,groups", SHAPES, ids=str)
def test_shapes(shape, groups, dtype):
    act = ("silu", "gelu", "relu", "none")[(len(shape) + groups) % 4]
    x, dy, w, b = inputs(sum(shape) + groups, shape, DT[dtype])
    check(x, dy, groups, w, b, act)


@pytest.mark.parametrize("act", ["silu", "gelu", "relu", "none"])
@pytest.mark.parametrize("kind", ["dense", "slice", "shifted"])
def test_layouts_and_activations(kind, act):
    for dt, (shape, groups) in ((torch.float16, ((3, 13, 5, 44), 4)), (torch.bfloat16, ((2, 17, 121), 11))):
        x, dy, w, b = inputs(7, shape, dt)
        check(x, dy, groups, w, b, act, kind)
        check(x, dy, groups, None, None, act, kind)


@pytest.mark.parametrize("shape,groups", [((2, 150, 170, 40), 5), ((1, 40000, 16), 2), ((3, 9000, 130), 2)], ids=str)
def test_images_in_parts(shape, groups):
    """Images that several workgroups share."""
    for dt in (torch.float16, torch.bfloat16):
        x, dy, w, b = inputs(11, shape, dt)
        assert cf.lib().cf_group_norm_workspace_bytes(shape[0], x[0, ..., 0].numel(), shape[-1], groups) > 0
        check(x, dy, groups, w, b, "silu", "slice")


@pytest.mark.parametrize("dtype,shape,groups,act", [
    ("f16", (260, 17, 1032), 1, "gelu"), ("bf16", (33, 26, 26, 384), 8, "silu"), ("f16", (30, 26, 26, 387), 9, "none"),
    ("bf16", (33, 819, 320), 8, "relu"), ("f16", (40, 31, 1032), 8, "silu"), ("bf16", (33, 14, 14, 1280), 8, "gelu")],
    ids=str)
def test_widths_that_leave_threads_without_a_vector(dtype, shape, groups, act):
    """More groups than workgroups run at once, of up to 4096 vectors, more than 16
    of them a thread if 256 threads took them."""
    x, dy, w, b = inputs(sum(shape), shape, DT[dtype])
    out = torch.full(shape, float("nan"), dtype=DT[dtype], device="cuda")
    cf.group_norm_forward(x.cuda(), groups, w.cuda(), b.cuda(), act=act, out=out)
    assert not bool(out.isnan().any()), "pixels that were not written"
    check(x, dy, groups, w, b, act)


def test_offsets_are_taken_off_before_squares():
    """Values far from 0: the variance is of their differences."""
    for shape, groups in (((2, 30, 30, 32), 4), ((1, 40000, 16), 2)):
        x, dy, w, b = inputs(13, shape, torch.float16)
        x = (x * 0.125 + 1000).half()  # steps of 0.5 at 1000
        check(x, dy, groups, w, b, "none", eps=1e-3)


def test_outputs_in_place_and_nothing_else_is_written():
    x, dy, w, b = inputs(17, (2, 6, 7, 36), torch.bfloat16)
    w, b = w.cuda(), b.cuda()
    y, stats = cf.group_norm_forward_save(x.cuda(), 3, w, b, act="gelu")
    dx = cf.group_norm_backward(dy.cuda(), x.cuda(), stats, w, b, act="gelu")[0]
    xi, di = place("slice", x), place("slice", dy)
    wide = [torch.full((2, 6, 7, 47), 7.0, dtype=x.dtype, device="cuda") for _ in range(2)]
    for t, v in zip(wide, (x, dy)):
        t[..., 3:39] = v.cuda()
    xi, di = (t[..., 3:39] for t in wide)
    cf.group_norm_backward(di, xi, stats, w, b, act="gelu", out=di)
    cf.group_norm_forward(xi, 3, w, b, act="gelu", out=xi)
    assert torch.equal(xi, y) and torch.equal(di, dx)
    for t in wide:
        t[..., 3:39] = 7.0
        assert bool((t == 7.0).all())


def test_values_that_are_not_finite_stay_in_their_group():
    x, dy, w, b = inputs(19, (3, 20, 24), torch.bfloat16)
    clean = check(x, dy, 3, w, b, "silu")
    x[1, 4, 9] = float("inf")
    x[2, 5, 0] = float("nan")
    y, stats = cf.group_norm_forward_save(x.cuda(), 3, w.cuda(), b.cuda(), act="silu")
    bad = torch.zeros(3, 3, dtype=torch.bool)
    bad[1, 1] = bad[2, 0] = True
    off = bad[:, None, :, None].expand(3, 20, 3, 8).reshape(3, 20, 24)
    assert bool(y.cpu()[off].isnan().all()) and torch.equal(y.cpu()[~off], clean[0].cpu()[~off])
    assert torch.equal(stats.cpu().isnan().any(-1), bad)


def test_a_group_without_spread_and_empty_batches():
    x = torch.full((2, 10, 16), 3.0, dtype=torch.float16, device="cuda")
    b = torch.arange(16.0, device="cuda")
    y, stats = cf.group_norm_forward_save(x, 4, None, b)
    assert torch.equal(y, b.half().expand_as(y)) and torch.equal(stats[..., 0], torch.full((2, 4), 3.0, device="cuda"))
    for shape in ((0, 4, 4, 16), (3, 0, 16)):
        e = torch.empty(shape, dtype=torch.float16, device="cuda")
        y, stats = cf.group_norm_forward_save(e, 4)
        assert y.shape == e.shape and stats.shape == (shape[0], 4, 2)
        dx, dw, db = cf.group_norm_backward(e, e, stats, None, None)
        assert dx.shape == e.shape and bool((dw == 0).all()) and bool((db == 0).all())


def test_gradients_against_differences():
    """(loss(x + h v) - loss(x - h v)) / 2h of the definition in 64 bits along random directions."""
    x, dy, w, b = inputs(23, (2, 6, 5, 24), torch.float16)
    for act in ("silu", "gelu", "none"):
        _, stats = cf.group_norm_forward_save(x.cuda(), 4, w.cuda(), b.cuda(), act=act)
        dx, dw, db = (t.double().cpu() for t in cf.group_norm_backward(dy.cuda(), x.cuda(), stats, w.cuda(), b.cuda(), act=act))

        def loss(xv, wv, bv):
            y = reference(xv.view(2, -1, 24), None, 4, wv, bv, 1e-6, act)[0][0]
            return float((y * dy.double().view(2, -1, 24)).sum())

        at = [x.double(), w.double(), b.double()]
        for i, g in enumerate((dx, dw, db)):
            v = randn(29 + i, g.shape).double()
            h = 1e-5
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + h * v, at[i] - h * v
            want = (loss(*up) - loss(*down)) / (2 * h)
            # dx is rounded to fp16, 2^-11 of each value
            assert abs(float((g * v).sum()) - want) <= 2**-11 * float((g * v).abs().sum()) + 1e-5, (act, i)
