"""8-bit checkpoints: the bytes and scales bit for bit, the values read back,
and the activation with its gradient against 64 bits.

Tolerances.  q, scale and what unpack gives are defined to the bit.  The fp32
GELU errs by at most 1e-7 max(1, |u|) and its slope by 5e-7 (tail 1.5e-8,
exponential and product a few roundings, |u| phi(u) < 0.25); one rounding to
the I/O type follows."""
import math

import pytest
import torch

import paper_2404_03617_amd as cf

from _rows import DT, F32, ROUND, TINY, assert_within, dequantise, guarded, outside_untouched, quantise, randn, rows_in

pytestmark = pytest.mark.gpu

SHAPES = [(1, 1), (2, 3), (1, 8), (5, 63), (300, 64), (7, 65), (33, 127), (64, 128), (9, 200), (21, 1000), (3, 4096),
          (2, 20011), (2000, 24)]


def tensor(seed, rows, C, dt):
    x = randn(seed, (rows, C)) * torch.exp(randn(seed + 1, (C,)))
    return x.to(dt)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("rows,C", SHAPES)
def test_pack_and_unpack(rows, C, dtype):
    dt = DT[dtype]
    x = tensor(rows + C, rows, C, dt)
    q, scale, _ = quantise(x)
    back = (q.float() * scale.repeat_interleave(64, 1)[:, :C]).to(dt)
    for kind in ("dense", "slice", "shifted"):
        ck = cf.checkpoint_pack(rows_in(kind, x))
        assert torch.equal(ck.q.cpu(), q) and torch.equal(ck.scale.cpu(), scale), kind
        assert torch.equal(cf.checkpoint_unpack(ck).cpu(), back)
        out, wide = guarded(rows, C, dt)
        cf.checkpoint_unpack(ck, out=out)
        assert torch.equal(out.cpu(), back) and outside_untouched(wide, C)
    worst = scale.repeat_interleave(64, 1)[:, :C].double() * 0.5 * (1 + 2**-15)
    assert bool(((dequantise(q, scale) - x.double()).abs() <= worst).all())


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_ties_tiny_blocks_and_values_that_are_not_finite(dtype):
    dt = DT[dtype]
    x = torch.zeros(8, 130, dtype=dt)
    x[0, :64] = torch.arange(64) * 0.5  # scale 31.5 / 127
    x[0, 64] = 127.0
    x[0, 65:128] = torch.arange(63) - 31.5  # halves: to even
    x[1, 3] = float("inf")
    x[1, 70] = 2.0
    x[2, 64] = float("nan")
    x[3] = torch.finfo(dt).max
    x[4, ::2] = torch.finfo(dt).tiny
    x[5] = -torch.finfo(dt).max
    x[6, 129] = -3.0
    if dt == torch.bfloat16:
        x[7] = 2.0**-120  # below the least block
        x[7, 128] = 2.0**-118
    q, scale, fine = quantise(x)
    ck = cf.checkpoint_pack(x.cuda())
    assert torch.equal(torch.isnan(ck.scale).cpu(), ~fine)
    assert torch.equal(ck.scale.cpu()[fine], scale[fine])
    cols = fine.repeat_interleave(64, 1)[:, :130]
    assert torch.equal(ck.q.cpu()[cols], q[cols])
    back = cf.checkpoint_unpack(ck).cpu()
    assert bool(torch.isnan(back[~cols]).all()) and bool(torch.isfinite(back[cols]).all())


def gelu(u):
    return u * torch.special.ndtr(u)


def gelu_slope(u):
    return torch.special.ndtr(u) + u * torch.exp(-u * u / 2) / math.sqrt(2 * math.pi)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
@pytest.mark.parametrize("act", ["gelu", "relu", "none"])
@pytest.mark.parametrize("rows,C", SHAPES)
def test_activation_and_its_gradient(rows, C, act, dtype):
    dt = DT[dtype]
    u, dh = tensor(rows * 3 + C, rows, C, dt), randn(C, (rows, C), dt)
    f = {"gelu": gelu, "relu": lambda v: v.clamp_min(0), "none": lambda v: v}[act]
    slope = {"gelu": gelu_slope, "relu": lambda v: (v > 0).double(), "none": torch.ones_like}[act]
    q, scale, _ = quantise(u)
    href, dref = f(u.double()), dh.double() * slope(dequantise(q, scale))
    exact = act != "gelu"
    th = ROUND[dt] * href.abs() + (0.0 if exact else 1e-7 * u.double().abs().clamp_min(1)) + TINY[dt]
    td = ROUND[dt] * dref.abs() + (0.0 if exact else 5e-7 * dh.double().abs()) + TINY[dt]
    for kind in ("dense", "slice"):
        ud, dd = rows_in(kind, u), rows_in(kind, dh)
        h, cu, ch = cf.act_forward_save(ud, act, checkpoint_out=True)
        assert_within(h, href, th, "%s h" % kind)
        assert torch.equal(cf.act_forward(ud, act), h)
        assert torch.equal(cu.q.cpu(), q) and torch.equal(cu.scale.cpu(), scale)
        qh, sh, _ = quantise(h.cpu())
        assert torch.equal(ch.q.cpu(), qh) and torch.equal(ch.scale.cpu(), sh)
        du = cf.act_backward(dd, cu, act)
        assert_within(du, dref, td, "%s du" % kind)
        out, wide = guarded(rows, C, dt)
        cf.act_backward(dd, cu, act, out=out)
        assert torch.equal(out, du) and outside_untouched(wide, C)
    d = dh.cuda()
    assert torch.equal(cf.act_backward(d, cu, act, out=d), du)
    v = u.cuda()
    assert torch.equal(cf.act_forward(v, act, out=v), h)


@pytest.mark.parametrize("dtype", ["f16", "bf16"])
def test_gelu_over_its_whole_range(dtype):
    """Every finite 16-bit number, and the gradient on a grid that the format
    keeps exactly (block maximum 127 / 8: u = q / 8)."""
    dt = DT[dtype]
    bits = torch.arange(65536, dtype=torch.int32).to(torch.int16)
    u = bits.view(dt)
    u = u[torch.isfinite(u)]
    u = torch.cat([u, u.new_zeros(-u.numel() % 64)]).view(-1, 64)
    href = gelu(u.double())
    h = cf.act_forward(u.cuda(), "gelu")
    assert_within(h, href, ROUND[dt] * href.abs() + 1e-7 * u.double().abs().clamp_min(1) + TINY[dt], "gelu")
    special = torch.tensor([[float("inf"), -float("inf"), float("nan"), 0.0]], dtype=dt)
    s = cf.act_forward(special.cuda(), "gelu").cpu()[0]
    assert s[0] == float("inf") and s[1] == 0 and torch.isnan(s[2]) and s[3] == 0
    k = (torch.arange(255) - 127).float()
    k = torch.cat([k, torch.full((65,), 127.0)]).view(5, 64)
    k[:, 0] = 127.0
    q, scale = k.to(torch.int8), torch.full((5, 1), 0.125)
    ref = gelu_slope(q.double() * 0.125)
    ones = torch.ones(5, 64, dtype=dt)
    got = cf.act_backward(ones.cuda(), cf.Checkpoint(q.cuda(), scale.cuda(), dt), "gelu")
    assert_within(got, ref, ROUND[dt] * ref.abs() + 5e-7, "gelu'")


def test_gradient_against_differences():
    """The slope at checkpointed values against central differences of GELU."""
    u = tensor(4, 40, 96, torch.float16)
    ck = cf.checkpoint_pack(u.cuda())
    v, h = dequantise(ck.q.cpu(), ck.scale.cpu()), 1e-4
    want = (gelu(v + h) - gelu(v - h)) / (2 * h)
    got = cf.act_backward(torch.ones_like(u).cuda(), ck, "gelu")
    assert_within(got, want, 2**-11 * want.abs() + 1e-6, "gelu' and the difference")


def test_no_rows_and_offsets_past_32_bits():
    e = torch.empty(0, 70, dtype=torch.bfloat16, device="cuda")
    h, cu, _ = cf.act_forward_save(e)
    assert h.shape == (0, 70) and cf.act_backward(e, cu).shape == (0, 70) and cf.checkpoint_unpack(cu).shape == (0, 70)
    rows, ld, C = 70000, 32768, 72
    buf = torch.zeros(rows * ld, dtype=torch.float16, device="cuda").view(rows, ld)
    u, out = buf[:, 5:5 + C], buf[:, 4096:4096 + C]
    some = torch.tensor([0, 65535, 65537, 69999]).cuda()
    vals = tensor(6, 4, C, torch.float16).cuda()
    u[some] = vals
    h, cu, ch = cf.act_forward_save(u, checkpoint_out=True, out=out)
    small = cf.act_forward_save(vals, checkpoint_out=True)
    assert torch.equal(h[some], small[0]) and torch.equal(cu.q[some], small[1].q) and torch.equal(ch.q[some], small[2].q)
    du = cf.act_backward(u, cu, out=out)
    assert torch.equal(du[some], cf.act_backward(vals, small[1]))


def test_side_stream_and_graph():
    u = tensor(5, 500, 130, torch.float16).cuda()
    dh = randn(6, (500, 130), torch.float16).cuda()

    def step(stream=None):
        h, cu, ch = cf.act_forward_save(u, checkpoint_out=True, stream=stream)
        return h, cf.act_backward(dh, cu, stream=stream), cf.checkpoint_unpack(ch, stream=stream)

    want = [t.clone() for t in step()]
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    got = step(side)
    torch.cuda.current_stream().wait_stream(side)
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        rec = step()
    first, other = u.clone(), tensor(9, 500, 130, torch.float16).cuda()
    for v in (first, other, first):
        u.copy_(v)
        g.replay()
        eager = step()
        torch.cuda.synchronize()
        assert all(torch.equal(a, b) for a, b in zip(rec, eager))


def test_refusals():
    x = torch.zeros(4, 70, dtype=torch.float16, device="cuda")
    ck = cf.checkpoint_pack(x)
    with pytest.raises(ValueError):
        cf.act_forward(x, "tanh")
    with pytest.raises(ValueError):
        cf.checkpoint_pack(x.float())
    with pytest.raises(TypeError):
        cf.act_backward(x, x)
    with pytest.raises(TypeError):
        cf.checkpoint_unpack(x)
    for bad in (cf.Checkpoint(ck.q[:3], ck.scale, ck.dtype), cf.Checkpoint(ck.q, ck.scale[:, :1], ck.dtype),
                cf.Checkpoint(ck.q.short(), ck.scale, ck.dtype), cf.Checkpoint(ck.q, ck.scale.half(), ck.dtype),
                cf.Checkpoint(ck.q.cpu(), ck.scale, ck.dtype)):
        with pytest.raises(ValueError):
            cf.act_backward(x, bad)
    with pytest.raises(ValueError):
        cf.checkpoint_unpack(cf.Checkpoint(ck.q, ck.scale, torch.float32))
    with pytest.raises(ValueError):
        cf.act_backward(x[:, :69], ck)
    buf = torch.zeros(5, 70, dtype=torch.float16, device="cuda")
    with pytest.raises(cf.CFError) as e:
        cf.act_forward(buf[:4], out=buf[1:])
    assert e.value.status == cf.CF_ERR_INVALID and "overlap" in str(e.value)
    two = torch.zeros(4, 140, dtype=torch.float16, device="cuda")
    cf.act_forward(two[:, :70], out=two[:, 70:])  # apart, though their rows alternate
