"""The gated feed-forward block, forward and backward.  With small whole numbers
every product and sum is exact and each result must be the definition's, rounded
once; with random numbers, against 64 bits: the error of a sum of n products in
fp32 is at most n 2^-24 of the sum of their magnitudes, and the factors h, da and
du are rounded to 16 bits."""
import math

import pytest
import torch

import paper_2404_03617_amd as cf

from _rows import DT, F32, ROUND, TINY, assert_within, randn, rows_in

pytestmark = pytest.mark.gpu


def act_of(u, act):
    if act == "silu":
        s = torch.sigmoid(u)
        return u * s, s * (1 + u * (1 - s))
    if act == "gelu":
        p = torch.special.ndtr(u)
        return u * p, p + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)
    if act == "relu":
        return u.clamp_min(0), (u > 0).double()
    return u, torch.ones_like(u)


def signs(seed, rows, cols, each):
    """A matrix of -1, 0 and 1 on the GPU in 64 bits, `each` of a row not 0 at most."""
    g = torch.Generator(device="cuda").manual_seed(seed)
    m = torch.zeros(rows, cols, dtype=torch.float64, device="cuda")
    at = torch.randint(0, cols, (rows, each), generator=g, device="cuda")
    return m.scatter_(1, at, torch.randint(0, 2, (rows, each), generator=g, device="cuda").double() * 2 - 1)


def mm(a, b):
    return torch.mm(a.contiguous(), b.contiguous())


def exact_case(rows, C, H, dt, act, seed=1, kind="dense"):
    print("gated", rows, C, H, dt, act, kind, flush=True)
    x = torch.randint(-1, 2, (rows, C), device="cuda", generator=torch.Generator("cuda").manual_seed(seed)).double()
    wg, wu, wd = signs(seed + 1, H, C, 3), signs(seed + 2, H, C, 3), signs(seed + 3, C, H, 3)
    dy = signs(seed + 4, rows, C, 2)
    a, u = mm(x, wg.t()), mm(x, wu.t())
    f, slope = act_of(a, act)
    h = f * u
    dh = mm(dy, wd)
    da, du = dh * u * slope, dh * f
    assert max(float(t.abs().max()) if t.numel() else 0 for t in (h, da, du)) <= 256  # whole numbers that bf16 has
    want = (mm(h, wd.t()), mm(da, wg) + mm(du, wu), mm(da.t(), x), mm(du.t(), x), mm(dy.t(), h))

    def given(t):
        return rows_in(kind, t.to(dt).cpu()) if kind != "dense" else t.to(dt)

    xg, wgg, wug, wdg, dyg = given(x), given(wg), given(wu), given(wd), given(dy)
    y, saved = cf.gated_ffn_forward_save(xg, wgg, wug, wdg, act=act)
    assert torch.equal(cf.gated_ffn_forward(xg, wgg, wug, wdg, act=act), y)
    assert torch.equal(saved.double(), torch.cat([a, u], 1)), "saved"
    got = (y, *cf.gated_ffn_backward(dyg, xg, saved, wgg, wug, wdg, act=act))
    for g, t, what in zip(got, want, ("y", "dx", "dw_gate", "dw_up", "dw_down")):
        assert g.dtype == dt and g.shape == t.shape
        off = g.double() != t.to(dt).double()
        assert not bool(off.any()), (what, off.nonzero()[:4].tolist(), int(off.sum()))


SIZES = [(1, 8, 8), (1, 1, 1), (3, 5, 7), (16, 64, 128), (17, 40, 72), (100, 130, 33), (128, 128, 128), (129, 136, 264),
         (256, 256, 256), (300, 520, 1000), (64, 2048, 96), (1000, 24, 40), (5, 4096, 16), (2, 16, 4099), (700, 96, 520),
         (40, 1000, 2500), (2100, 264, 520), (1, 1024, 4000), (33, 1032, 1), (31, 1, 1032)]


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,C,H", SIZES)
def test_whole_numbers(rows, C, H, dtype):
    exact_case(rows, C, H, DT[dtype], "relu" if rows % 2 else "none", rows + C + H)


@pytest.mark.parametrize("kind", ["slice", "shifted"])
def test_whole_numbers_in_other_layouts(kind):
    for dt, size in ((torch.float16, (70, 136, 264)), (torch.bfloat16, (9, 48, 130)), (torch.float16, (1, 256, 512))):
        exact_case(*size, dt, "relu", 3, kind)


def test_whole_numbers_over_large_tiles_and_many_rows():
    exact_case(4096, 1024, 2048, torch.bfloat16, "relu")
    exact_case(20000, 256, 512, torch.float16, "none")


def bounds(x, wg, wu, wd, dy, act, dt, inner=None):
    """Results in 64 bits and tolerances: errors of the sums, propagated, and of each rounding to 16 bits."""
    R, T = ROUND[dt], TINY[dt]
    inner = R if inner is None else inner
    C, H, rows = x.shape[1], wg.shape[0], x.shape[0]

    def product(a, ea, b, eb, n):  # of a b with errors ea, eb in the factors
        p = mm(a.abs(), b.abs())
        e = n * F32 * p
        if ea is not None:
            e = e + mm(ea, b.abs())
        if eb is not None:
            e = e + mm(a.abs(), eb)
        return mm(a, b), e

    a, ea = product(x, None, wg.t(), None, C)
    u, eu = product(x, None, wu.t(), None, C)
    f, s = act_of(a, act)
    size = a.abs().clamp_min(1)
    ef = 1.13 * ea + 4e-7 * size
    es = 0.8 * ea + 4e-7 * size + ((a.abs() <= ea).double() if act == "relu" else 0)
    h = f * u
    eh = ef * u.abs() + f.abs() * eu + 2 * F32 * h.abs()
    eh = eh + inner * (h.abs() + eh) + T
    y, ey = product(h, None, wd.t(), None, H)
    ey = ey + mm(eh, wd.t().abs())
    dh, edh = product(dy, None, wd, None, C)
    da, du = dh * u * s, dh * f
    eda = edh * (u * s).abs() + dh.abs() * (eu * s.abs() + u.abs() * es) + 3 * F32 * da.abs()
    edu = edh * f.abs() + dh.abs() * ef + 2 * F32 * du.abs()
    eda, edu = eda + inner * (da.abs() + eda) + T, edu + inner * (du.abs() + edu) + T
    g1, e1 = product(da, eda, wg, None, 2 * H)
    g2, e2 = product(du, edu, wu, None, 2 * H)
    dwg, edwg = product(da.t(), eda.t(), x, None, rows)
    dwu, edwu = product(du.t(), edu.t(), x, None, rows)
    dwd, edwd = product(dy.t(), None, h, eh, rows)
    out = [(y, ey), (g1 + g2, e1 + e2), (dwg, edwg), (dwu, edwu), (dwd, edwd)]
    return [(t, e + R * (t.abs() + e) + T) for t, e in out]


def random_case(rows, C, H, dt, seed=0):
    x, wg, wu = randn(seed, (rows, C), dt), randn(seed + 1, (H, C), dt, C**-0.5), randn(seed + 2, (H, C), dt, C**-0.5)
    return x, wg, wu, randn(seed + 3, (C, H), dt, H**-0.5), randn(seed + 4, (rows, C), dt, 0.1)


NAMES = ("y", "dx", "dw_gate", "dw_up", "dw_down")


@pytest.mark.parametrize("act", ["silu", "gelu", "relu", "none"])
@pytest.mark.parametrize("rows,C,H,dtype", [(1, 96, 200, "f16"), (50, 72, 130, "bf16"), (300, 256, 515, "f16"),
                                            (16, 512, 64, "bf16")])
def test_random_numbers(rows, C, H, dtype, act):
    dt = DT[dtype]
    given = random_case(rows, C, H, dt)
    ref = bounds(*(t.double() for t in given), act, dt)
    x, wg, wu, wd, dy = (t.cuda() for t in given)
    y, saved = cf.gated_ffn_forward_save(x, wg, wu, wd, act=act)
    got = (y, *cf.gated_ffn_backward(dy, x, saved, wg, wu, wd, act=act))
    again = cf.gated_ffn_backward(dy, x, saved, wg, wu, wd, act=act)
    assert all(torch.equal(p, q) for p, q in zip(got[1:], again))
    for g, (t, e), what in zip(got, ref, NAMES):
        assert_within(g, t, e, what)
        # two roundings of 2^-9 (2^-12) at most, the inner ones independent of each other
        assert float((g.double().cpu() - t).norm() / t.norm()) <= 2 * ROUND[dt], what


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,C,H", [(1, 96, 200), (16, 64, 130), (7, 33, 77), (2, 1032, 24)])
def test_few_rows_are_rounded_once(rows, C, H, dtype):
    """Up to 16 rows h, da and du are kept in two numbers of 16 bits: off by the
    square of a rounding (in fp16 by half of its least number, which is in the
    tolerance anyway)."""
    dt = DT[dtype]
    given = random_case(rows, C, H, dt, 21)
    ref = bounds(*(t.double() for t in given), "silu", dt, inner=ROUND[dt] ** 2)
    x, wg, wu, wd, dy = (t.cuda() for t in given)
    y, saved = cf.gated_ffn_forward_save(x, wg, wu, wd)
    got = (y, *cf.gated_ffn_backward(dy, x, saved, wg, wu, wd))
    for g, (t, e), what in zip(got, ref, NAMES):
        assert_within(g, t, e, what)


def test_leading_dimensions_outputs_and_workspaces():
    dt = torch.float16
    x, wg, wu, wd, dy = (t.cuda() for t in random_case(24, 64, 104, dt, 5))
    y, saved = cf.gated_ffn_forward_save(x, wg, wu, wd)
    grads = cf.gated_ffn_backward(dy, x, saved, wg, wu, wd)
    x4, dy4 = x.view(2, 3, 4, 64), dy.view(2, 3, 4, 64)
    wide = torch.full((2, 3, 4, 80), 7.0, dtype=dt, device="cuda")
    y4, saved4 = cf.gated_ffn_forward_save(x4, wg, wu, wd, out=wide[..., 8:72])
    assert torch.equal(y4.reshape(24, 64), y) and saved4.shape == (2, 3, 4, 208) and torch.equal(saved4.view(24, 208), saved)
    wide[..., 8:72] = 7.0
    assert bool((wide == 7.0).all())
    for name, aligned in (("gated_ffn_workspace_bytes", True), ("gated_ffn_workspace_bytes", False)):
        ws = torch.full((getattr(cf.heads, name)(24, 64, 104, aligned),), 255, dtype=torch.uint8, device="cuda")
        assert torch.equal(cf.gated_ffn_forward(x, wg, wu, wd, ws=ws), y)
    ws = torch.full((cf.heads.gated_ffn_backward_workspace_bytes(24, 64, 104, True),), 255, dtype=torch.uint8, device="cuda")
    for g, t in zip(cf.gated_ffn_backward(dy4, x4, saved4, wg, wu, wd, ws=ws), grads):
        assert torch.equal(g.reshape(t.shape), t)
    # gate and up as the halves of one matrix, with a stride of their own
    both = torch.cat([wg, wu], 1)
    assert torch.equal(cf.gated_ffn_forward(x, both[:, :64], both[:, 64:], wd), y)
    mixed = torch.cat([wg, wg], 1)[:, :64]  # another stride than up's
    assert torch.equal(cf.gated_ffn_forward(x, mixed, wu, wd), y)
    # one row for all
    one = x[:1].expand(5, 64)
    assert torch.equal(cf.gated_ffn_forward(one, wg, wu, wd), cf.gated_ffn_forward(one.contiguous(), wg, wu, wd))


def test_no_rows():
    x, wg, wu, wd, _ = (t.cuda() for t in random_case(2, 24, 36, torch.bfloat16))
    e = x[:0]
    y, saved = cf.gated_ffn_forward_save(e, wg, wu, wd)
    assert y.shape == (0, 24) and saved.shape == (0, 72)
    dx, *dw = cf.gated_ffn_backward(e, e, saved, wg, wu, wd)
    assert dx.shape == (0, 24) and all(bool((t == 0).all()) for t in dw)
    assert [tuple(t.shape) for t in dw] == [(36, 24), (36, 24), (24, 36)]


def test_gradients_against_differences():
    dt = torch.float16
    given = random_case(6, 24, 40, dt, 9)
    dy = given[4].double()
    for act in ("silu", "gelu"):
        x, wg, wu, wd, dyg = (t.cuda() for t in given)
        _, saved = cf.gated_ffn_forward_save(x, wg, wu, wd, act=act)
        grads = [t.double().cpu() for t in cf.gated_ffn_backward(dyg, x, saved, wg, wu, wd, act=act)]

        def loss(x, wg, wu, wd):
            return float((((act_of(x @ wg.t(), act)[0] * (x @ wu.t())) @ wd.t()) * dy).sum())

        at = [t.double() for t in given[:4]]
        _, dxe, dge, due, dde = bounds(*(t.double() for t in given), act, dt)
        for i, (g, e) in enumerate(zip(grads, (dxe[1], dge[1], due[1], dde[1]))):
            v = randn(40 + i, g.shape).double()
            up, down = list(at), list(at)
            up[i], down[i] = at[i] + 1e-5 * v, at[i] - 1e-5 * v
            want = (loss(*up) - loss(*down)) / 2e-5
            assert abs(float((g * v).sum()) - want) <= float((e * v.abs()).sum()) + 1e-6, (act, i)
