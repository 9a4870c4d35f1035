"""Log probabilities, entropy, alternatives and the gradient against 64 bits.

Tolerances.  An exponential errs by 2^-23 of itself and by its argument's
rounding (2 roundings of |d|, where the weight exp(d) |d| is below 0.37), a sum
over threads, waves and chunks by some 64 roundings: the sum of exponentials by
at most 2^-17 of itself, its logarithm by 2^-17, the entropy by twice that and
2^-17 of its own size, a log probability by 2^-17 and one rounding of its
parts.  ids are exact.  The gradient is rounded once to the logits' type."""
import pytest
import torch

import paper_2404_03617_amd as cf
from paper_2404_03617_amd import training

from _rows import DT, F32, ROUND, TINY, assert_within, guarded, outside_untouched, randn, rows_in

pytestmark = pytest.mark.gpu
INF = float("inf")
E = 2.0**-17

# rows, V: whole rows, rows in chunks, shorter than a vector, long and odd
SHAPES = [(1, 1), (3, 2), (5, 7), (1, 10), (40, 63), (700, 33), (128, 1000), (2, 1001), (1, 2049), (3, 8192), (2, 32003),
          (600, 4100), (1, 131072), (5, 100003)]


def reference(z, tokens):
    z = z.double()
    m = z.amax(1, keepdim=True)
    empty = m == -INF
    s = torch.where(empty, torch.zeros_like(z), torch.exp(z - m))
    total = s.sum(1, keepdim=True)
    logp = torch.where(empty, z, z - m - torch.log(total))
    p = torch.where(empty, torch.zeros_like(z), s / total)
    h = -torch.where(p > 0, p * logp, torch.zeros_like(p)).sum(1)
    lp = torch.where(tokens >= 0, logp.gather(1, tokens.clamp_min(0)[:, None])[:, 0], torch.zeros_like(h))
    return logp, p, h, lp, empty[:, 0]


def order(z, top):
    """ids by value, equal ones by index (a stable sort)."""
    return torch.sort(z.double() + 0.0, dim=1, descending=True, stable=True).indices[:, :top]


def tol_logp(z, logp):
    return torch.where(torch.isfinite(logp), E + 4 * F32 * (logp.abs() + z.double().abs().nan_to_num(0, 0, 0)), torch.ones_like(logp))


def check(z, tokens, top, kind="dense"):
    logp, p, h, lp, empty = reference(z, tokens)
    zd = rows_in(kind, z)
    r = cf.log_probs_forward(zd, tokens.cuda(), top=top)
    tl = tol_logp(z, logp)
    assert_within(r.entropy, h, 2 * E + E * h, "entropy")
    assert_within(r.logp, lp, torch.where(tokens >= 0, tl.gather(1, tokens.clamp_min(0)[:, None])[:, 0], 1e-30 * torch.ones_like(h)), "logp")
    if top:
        ids = order(z, top)
        assert torch.equal(r.top_ids.cpu(), ids)
        assert_within(r.top_logp, logp.gather(1, ids), tl.gather(1, ids), "top_logp")
    else:
        assert r.top_ids is None and r.top_logp is None
    lse = torch.logsumexp(z.double(), 1)
    assert_within(r.stats.cpu().double().sum(1), lse, torch.where(empty, torch.ones_like(lse), E + 4 * F32 * z.double().amax(1).abs()), "stats")
    return zd, r, logp, p, h, empty


def check_backward(z, tokens, zd, r, logp, p, h, empty, seed=1):
    rows, V = z.shape
    gl, gh = randn(seed, (rows,)), 0.3 * randn(seed + 1, (rows,))
    on = (tokens >= 0) & ~empty
    one = torch.zeros_like(p).scatter_(1, tokens.clamp_min(0)[:, None], 1.0) * on[:, None]
    g = torch.where(on, gl.double(), torch.zeros(rows, dtype=torch.float64))[:, None]
    slope = torch.where(p > 0, logp + h[:, None], torch.zeros_like(p))
    want = g * (one - p) - gh.double()[:, None] * p * slope
    err = 4 * E * p * (g.abs() + gh.double().abs()[:, None] * (1 + h[:, None] + slope.abs())) + 4 * F32 * g.abs() * one

    def tol(value):
        return ROUND[z.dtype] * (value.abs() + err) + err + TINY[z.dtype] + 1e-38

    got = cf.log_probs_backward(zd, tokens.cuda(), r, gl.cuda(), gh.cuda())
    assert_within(got, want, tol(want), "dlogits")
    out, wide = guarded(rows, V, z.dtype)
    cf.log_probs_backward(zd, tokens.cuda(), r, gl.cuda(), gh.cuda(), out=out)
    assert torch.equal(out, got) and outside_untouched(wide, V)
    only = cf.log_probs_backward(zd, None, r, None, gh.cuda())
    part = -gh.double()[:, None] * p * slope
    assert_within(only, part, tol(part), "entropy's")
    only = cf.log_probs_backward(zd, tokens.cuda(), r, gl.cuda())
    part = g * (one - p)
    assert_within(only, part, tol(part), "logp's")
    again = zd.clone()
    assert torch.equal(cf.log_probs_backward(again, tokens.cuda(), r, gl.cuda(), gh.cuda(), out=again), got)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("rows,V", SHAPES)
def test_forward_and_backward(rows, V, dtype):
    dt = DT[dtype]
    for n, kind in enumerate(("dense", "slice")):
        z = randn(rows + V + n, (rows, V), dt, 2.5)
        g = torch.Generator().manual_seed(V)
        tokens = torch.randint(-1 if rows > 1 else 0, V, (rows,), generator=g)
        for top in {0, 1, min(5, V), min(32, V)} if n == 0 else {min(8, V)}:
            got = check(z, tokens, top, kind)
        check_backward(z, tokens, *got)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("rows,V,top", [(70, 50, 8), (70, 64, 9), (70, 64, 17), (300, 128, 16), (300, 250, 32), (40, 512, 5),
                                        (1100, 1500, 5), (9, 1500, 5), (4200, 2600, 8), (4200, 1900, 3), (30, 3000, 0),
                                        (9, 3000, 8), (4200, 4096, 2)])
def test_rows_between_a_few_lanes_and_a_workgroup(rows, V, top, dtype):
    dt = DT[dtype]
    z = randn(rows + V, (rows, V), dt, 1.5)
    z[::7, ::3] = -INF
    z[1::5] = z[1::5].round()  # ties
    g = torch.Generator().manual_seed(V)
    tokens = 3 * torch.randint(0, V // 3, (rows,), generator=g) + 1
    check(z, tokens, top)


def masked_rows(V, dt):
    """Rows whose masks leave all, one, few or no classes, by -inf or by the
    type's lowest value; equal logits; large and small ones."""
    lowest = torch.finfo(dt).min
    base = randn(V, (V,), torch.float32, 2.0).to(dt)
    rows = [base.clone() for _ in range(14)]
    rows[1][:] = -INF
    rows[2][:] = lowest
    rows[3][:] = -INF
    rows[3][V // 2] = 3.0
    rows[4][:] = lowest
    rows[4][V - 1] = -2.0
    rows[5][3:] = -INF
    rows[6][:] = 0.0
    rows[7][::2] = -INF
    rows[7][1::2] = lowest
    rows[8][:] = -0.0
    rows[8][V // 3] = 0.0
    rows[9] = base.abs().round()  # many ties
    rows[10][:] = lowest
    rows[10][V // 4] = -INF
    rows[11] = (base.float() * 0 - 1000.0).to(dt)
    rows[11][5] = -990.0
    rows[12] = base + 60000.0 if dt == torch.float16 else (base.float() + 1e4).to(dt)
    rows[13] = torch.arange(V).float().remainder(7).to(dt)
    return torch.stack(rows)


@pytest.mark.parametrize("dtype", ["f16", "bf16", "f32"])
@pytest.mark.parametrize("V,repeat", [(33, 1), (700, 80), (1000, 1), (1900, 80), (3000, 80), (4100, 40), (20001, 1)])
def test_masks_ties_and_extremes(V, repeat, dtype):
    z = masked_rows(V, DT[dtype]).repeat(repeat, 1)
    g = torch.Generator().manual_seed(4)
    tokens = torch.randint(0, V, (z.shape[0],), generator=g)
    tokens[3::14] = V // 2
    for top in (1, 6, 32):
        got = check(z, tokens, top)
    # gradients where log p is finite or the row is empty
    keep = torch.isfinite(got[2].gather(1, tokens[:, None])[:, 0]) & (got[2].gather(1, tokens[:, None])[:, 0] > -1e30)
    z, tokens = z[keep], tokens[keep]
    check_backward(z, tokens, *check(z, tokens, 0))


@pytest.mark.parametrize("V", [70, 40000])
def test_many_large_logits_in_few_threads(V):
    """More logits above the bound than the list holds: every eighth vector of
    one thread in 64 is large (and all of them differ)."""
    z = randn(3, (2, V), torch.float32, 0.01)
    at = torch.arange(V)
    large = (at // 4) % 256 < 12
    z[:, large] = 5.0 + torch.arange(int(large.sum())).float().remainder(977) * 0.01
    check(z, torch.tensor([0, V - 1]), 32)


@pytest.mark.parametrize("rows", [1, 600])
def test_rows_that_are_not_finite(rows):
    V = 5000
    z = randn(2, (rows, V), torch.bfloat16)
    z[0, 77] = float("nan")
    if rows > 1:
        z[1, 4000] = INF
        z[2, [9, 4999]] = float("nan")
        z[3, 8] = INF
        z[3, 4] = -INF
    n = min(rows, 4)
    tokens = torch.zeros(rows, dtype=torch.int64)
    r = cf.log_probs_forward(z.cuda(), tokens.cuda(), top=4)
    assert bool(torch.isnan(r.logp[:n]).all()) and bool(torch.isnan(r.entropy[:n]).all())
    assert bool(torch.isnan(r.top_logp[:n]).all()) and bool(torch.isfinite(r.logp[n:]).all())
    assert r.top_ids[0, 0] == 77
    if rows > 1:
        assert r.top_ids[2, :2].tolist() == [9, 4999] and r.top_ids[1, 0] == 4000 and r.top_ids[3, 0] == 8
        assert torch.equal(r.top_ids[4:].cpu(), order(z[4:], 4))
    assert bool((r.top_ids >= 0).all()) and bool((r.top_ids < V).all())
    d = cf.log_probs_backward(z.cuda(), tokens.cuda(), r, torch.ones(rows, device="cuda"))
    assert bool(torch.isnan(d[:n]).all()) and bool(torch.isfinite(d[n:]).all())


def test_tokens_outside_the_vocabulary():
    z = randn(2, (3, 50), torch.float16)
    tokens = torch.tensor([50, -7, 49])
    r = cf.log_probs_forward(z.cuda(), tokens.cuda())
    assert torch.isnan(r.logp[0]) and r.logp[1] == 0 and torch.isfinite(r.logp[2])
    d = cf.log_probs_backward(z.cuda(), tokens.cuda(), r, torch.ones(3, device="cuda"))
    assert bool(torch.isnan(d[0]).all()) and bool((d[1] == 0).all()) and bool(torch.isfinite(d[2]).all())


def test_gradient_against_differences():
    """The gradient against central differences of logp and entropy."""
    rows, V, h = 4, 37, 1e-5
    z = randn(6, (rows, V))
    tokens = torch.tensor([0, 36, 5, -1])
    gl, gh = randn(7, (rows,)).double(), randn(8, (rows,)).double()
    v = randn(9, (rows, V)).double()

    def loss(s):
        _, _, ent, lp, _ = reference(z.double() + s * v, tokens)
        return (gl * lp + gh * ent).sum()

    want = float((loss(h) - loss(-h)) / (2 * h))
    r = cf.log_probs_forward(z.cuda(), tokens.cuda())
    d = cf.log_probs_backward(z.cuda(), tokens.cuda(), r, gl.float().cuda(), gh.float().cuda()).cpu().double()
    got = float((d * v).sum())
    print("  difference %.9g, gradient %.9g" % (want, got), flush=True)
    assert abs(want - got) <= 4 * E * float((d * v).abs().sum() + v.abs().sum() * 0.1) + 1e-8


def test_leading_dimensions_no_tokens_no_rows():
    z = randn(1, (2, 3, 40), torch.bfloat16).cuda()
    r = cf.log_probs_forward(z, top=3)
    assert r.logp is None and r.entropy.shape == (2, 3) and r.top_ids.shape == (2, 3, 3) and r.stats.shape == (2, 3, 2)
    t = torch.zeros(2, 3, dtype=torch.int64, device="cuda")
    assert cf.log_probs_forward(z, t).logp.shape == (2, 3)
    e = cf.log_probs_forward(z[:0], t[:0], top=2)
    assert e.logp.shape == (0, 3) and e.top_ids.shape == (0, 3, 2)
    assert cf.log_probs_backward(z[:0], t[:0], e, torch.empty(0, 3, device="cuda")).shape == (0, 3, 40)


def test_offsets_past_32_bits():
    rows, V = 9000, 250001
    z = torch.zeros(rows * V, dtype=torch.bfloat16, device="cuda").view(rows, V)
    some = torch.tensor([0, 8589, 8590, 8999]).cuda()
    vals = randn(3, (4, V), torch.bfloat16, 2.0)
    z[some] = vals.cuda()
    tokens = torch.zeros(rows, dtype=torch.int64)
    tokens[some.cpu()] = torch.tensor([1, V - 1, 77777, V - 2])
    r = cf.log_probs_forward(z, tokens.cuda(), top=3)
    small = cf.log_probs_forward(vals.cuda(), tokens[some.cpu()].cuda(), top=3)
    assert torch.equal(r.top_ids[some], small.top_ids)
    assert torch.allclose(r.logp[some], small.logp, rtol=1e-6, atol=2 * E)
    gl = torch.ones(rows, device="cuda")
    d = cf.log_probs_backward(z, tokens.cuda(), r, gl, out=z)
    logp, p, *_ = reference(vals, tokens[some.cpu()])
    want = torch.zeros_like(p).scatter_(1, tokens[some.cpu()][:, None], 1.0) - p
    assert_within(d[some], want, 2.0**-8 * want.abs() + 4 * E * p + 4 * F32, "dlogits")


def test_workspace_stream_and_graph():
    V = 30000
    z = randn(1, (6, V), torch.float16, 2.0).cuda()
    tokens = torch.arange(6).cuda()
    gl = torch.ones(6, device="cuda")
    need = training.log_probs_workspace_bytes(6, V, 5)
    assert need > 0

    def step(stream=None, ws=None):
        r = cf.log_probs_forward(z, tokens, top=5, stream=stream, ws=ws)
        return (*r, cf.log_probs_backward(z, tokens, r, gl, gl, stream=stream))

    ws = torch.full((need + 64,), 0xA5, dtype=torch.uint8, device="cuda")
    want = [t.clone() for t in step(ws=ws[:need])]
    assert bool((ws[need:] == 0xA5).all())
    with pytest.raises(ValueError):
        step(ws=ws[:need - 1])
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rec = step()
    first, other = z.clone(), randn(9, (6, V), torch.float16, 2.0).cuda()
    for v in (first, other, first):
        z.copy_(v)
        g.replay()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(rec, eager))


def test_refusals():
    z = torch.zeros(4, 40, dtype=torch.float16, device="cuda")
    t = torch.zeros(4, dtype=torch.int64, device="cuda")
    r = cf.log_probs_forward(z, t)
    for args, kw in (((z.double(), t), {}), ((z, t.int()), {}), ((z, t[:3]), {}), ((z.t(), t), {}), ((z, t.cpu()), {})):
        with pytest.raises(ValueError):
            cf.log_probs_forward(*args, **kw)
    for top, status in ((41, cf.CF_ERR_INVALID), (33, cf.CF_ERR_UNSUPPORTED), (-1, cf.CF_ERR_INVALID)):
        with pytest.raises(cf.CFError) as e:
            cf.log_probs_forward(z, t, top=top)
        assert e.value.status == status
    g = torch.ones(4, device="cuda")
    with pytest.raises(cf.CFError):
        cf.log_probs_backward(z, t, r)
    with pytest.raises(cf.CFError):
        cf.log_probs_backward(z, None, r, g)
    with pytest.raises(ValueError):
        cf.log_probs_backward(z, t, r, g[:3])
    with pytest.raises(ValueError):
        cf.log_probs_backward(z, t, r, g, out=z.bfloat16())
    buf = torch.zeros(5, 40, dtype=torch.float16, device="cuda")
    with pytest.raises(cf.CFError):
        cf.log_probs_backward(buf[:4], t, r, g, out=buf[1:])


def above_the_bound(z, top, lanes, together):
    """How many logits of each row [rows, V] are strictly above the n-th largest
    (n = top) of 64 maxima: `lanes` threads take vectors of 16 bytes in turn, and
    `together` neighbouring threads share a maximum."""
    vec = 16 // z.element_size()
    owner = (torch.arange(z.shape[1]) // vec) % lanes // together
    most = torch.full((z.shape[0], 64), -INF).scatter_reduce_(1, owner.expand(z.shape), z.float(), "amax")
    bound = most.sort(1, descending=True).values[:, top - 1:top]
    return (z.float() > bound).sum(1)


def check_repeated(z, top, repeat):
    """check() on the first rows of a call on many copies of them, and that every
    copy gets the same answer."""
    rows = z.shape[0]
    tokens = torch.arange(rows)
    r = cf.log_probs_forward(z.repeat(repeat, 1).cuda(), tokens.repeat(repeat).cuda(), top=top)
    logp, _, h, lp, _ = reference(z, tokens)
    ids, tl = order(z, top), tol_logp(z, logp)
    for name, got, want, tol in (("entropy", r.entropy, h, 2 * E + E * h), ("logp", r.logp, lp, tl.gather(1, tokens[:, None])[:, 0]),
                                 ("top_logp", r.top_logp, logp.gather(1, ids), tl.gather(1, ids))):
        assert_within(got[:rows], want, tol, name)
    assert torch.equal(r.top_ids[:rows].cpu(), ids)
    for t in (r.entropy, r.logp, r.top_logp, r.top_ids):
        assert torch.equal(t, t[:rows].repeat((repeat,) + (1,) * (t.dim() - 1)))


def rows_with_large(V, dt, lanes, few):
    """Small logits but for those of the first `few` threads of `lanes`."""
    z = randn(3, (3, V), torch.float32, 0.01)
    large = (torch.arange(V) // (16 // dt.itemsize)) % lanes < few
    z[:, large] = 5.0 + torch.arange(int(large.sum())).float().remainder(977) * 0.01
    z[1] = z[1].flip(0) if V % (lanes * 16 // dt.itemsize) == 0 else z[1]
    return z.to(dt)


@pytest.mark.parametrize("V,few,dtype", [(40000, 12, "f32"), (40000, 100, "f32"), (70000, 12, "bf16"), (70000, 120, "f16")])
def test_more_above_the_bound_than_the_list_holds(V, few, dtype):
    """Rows whole in a workgroup: more than 480 logits above the bound, in few
    threads, so that each alternative takes a pass over the row."""
    z = rows_with_large(V, DT[dtype], 256, few)
    assert int(above_the_bound(z, 32, 256, 4).min()) > 480
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    check_repeated(z, 32, (2 * cus + 2) // 3 + 1)


@pytest.mark.parametrize("V,dtype", [(32768, "bf16"), (16384, "f16")])
def test_more_above_the_bound_than_the_list_holds_in_a_chunk(V, dtype):
    """The same in chunks of 2048, a vector a thread."""
    z = rows_with_large(V, DT[dtype], 256, 100)
    for c in range(0, V, 2048):
        assert int(above_the_bound(z[:, c:c + 2048], 32, 256, 4).min()) > 480
    check_repeated(z, 32, 1)


@pytest.mark.parametrize("V,dtype,most", [(4000, "bf16", 256), (2000, "f16", 256), (2000, "f32", 256), (1000, "f32", 256),
                                          (1000, "bf16", 64), (500, "f16", 64)])
def test_more_above_the_bound_than_a_wave_collects(V, dtype, most):
    """Rows of a wave each: more keys above the bound than its list holds."""
    few = {"f32": 19, "f16": 19, "bf16": 12}[dtype]
    z = rows_with_large(V, DT[dtype], 64, few)
    assert int(above_the_bound(z, 20, 64, 1).min()) > most
    cus = torch.cuda.get_device_properties(0).multi_processor_count
    check_repeated(z, 20, (4 * cus + 2) // 3 + 1)
