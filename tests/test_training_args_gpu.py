"""The native calls of the training and scoring operators take and refuse what
the Python path does: every malformed call raises the same error with them as
without, and every accepted one gives the same bytes."""
import pytest
import torch

import paper_2404_03617_amd as cf

from _rows import randn

pytestmark = pytest.mark.gpu


def flat(r):
    """The tensors of a result."""
    if isinstance(r, torch.Tensor):
        return [r]
    if isinstance(r, cf.Checkpoint):
        return [r.q, r.scale]
    return [] if r is None else [t for x in r for t in flat(x)]


def outcome(call, args):
    try:
        r = call(**args)
        torch.cuda.synchronize()
        return [t.clone() for t in flat(r)]
    except Exception as e:
        return type(e), str(e)


def spoiled(t):
    """Versions of an argument that a call may not be given in its place, and
    some that it may."""
    yield None
    yield "text"
    if isinstance(t, cf.Checkpoint):
        yield t.q
        yield cf.Checkpoint(t.q[:-1], t.scale, t.dtype)
        yield cf.Checkpoint(t.q, t.scale[:, :-1], t.dtype)
        yield cf.Checkpoint(t.q.float(), t.scale, t.dtype)
        yield cf.Checkpoint(t.q, t.scale.double(), t.dtype)
        yield cf.Checkpoint(t.q.cpu(), t.scale.cpu(), t.dtype)
        yield cf.Checkpoint(t.q, t.scale, torch.float32)
        yield cf.Checkpoint(t.q.t(), t.scale, t.dtype)
        return
    if not isinstance(t, torch.Tensor):
        return
    yield t.double()
    yield t.cpu()
    yield t[:-1]
    yield torch.cat([t, t[:1]])
    yield t[:0]
    yield t.unsqueeze(0)
    yield t.unsqueeze(-1)
    yield torch.stack([t, t], -1)[..., 0]  # not contiguous
    yield t.expand(2, *t.shape)
    yield t.new_zeros(())
    yield torch.nn.Parameter(t.clone(), requires_grad=False)
    if t.dim() > 1:
        yield torch.cat([t, t], -1)[..., : t.shape[-1]]  # rows of a wider tensor
        yield t[:1].expand(t.shape)


def calls():
    dt = torch.float16
    x, dy = randn(1, (40, 130), dt).cuda(), randn(2, (40, 130), dt).cuda()
    w, b = randn(3, (130,)).cuda(), randn(4, (130,)).cuda()
    y, stats, ck = cf.layer_norm_forward_save(x, w, b)
    g = randn(5, (40, 24), dt).cuda()
    z = randn(6, (30, 70), torch.bfloat16).cuda()
    t = (torch.arange(30) % 7 - 1).cuda()
    lp = cf.log_probs_forward(z, t)
    gl, gh = randn(7, (30,)).cuda(), randn(8, (30,)).cuda()
    out, dz = torch.empty_like(x), torch.empty_like(z)
    return {
        "norm": (cf.layer_norm_forward, dict(x=x, weight=w, bias=b, eps=1e-5, out=out)),
        "norm_save": (cf.layer_norm_forward_save, dict(x=x, weight=w, bias=b, checkpoint=True, out=out)),
        "norm_backward": (cf.layer_norm_backward, dict(dy=dy, x=x, stats=stats, weight=w, out=out)),
        "norm_backward, checkpoint": (cf.layer_norm_backward, dict(dy=dy, x=ck, stats=stats, weight=w, param_grads=False)),
        "pack": (cf.checkpoint_pack, dict(x=x)),
        "unpack": (cf.checkpoint_unpack, dict(ck=ck, out=out)),
        "act": (cf.act_forward, dict(u=x, act="relu", out=out)),
        "act_save": (cf.act_forward_save, dict(u=x, act="gelu", checkpoint_out=True, out=out)),
        "act_backward": (cf.act_backward, dict(dh=dy, u=ck, act="gelu", out=out)),
        "wgrad": (cf.linear_weight_grad, dict(dy=g, x=ck, stats=stats, weight=w, bias=b)),
        "log_probs": (cf.log_probs_forward, dict(logits=z, tokens=t, top=3)),
        "log_probs_backward": (cf.log_probs_backward, dict(logits=z, tokens=t, lp=lp, d_logp=gl, d_entropy=gh, out=dz)),
    }


@pytest.mark.parametrize("name", list(calls()) if torch.cuda.is_available() else ["none"])
def test_native_calls_accept_and_refuse_alike(name, monkeypatch):
    assert cf._args is not None
    call, args = calls()[name]
    variants = [args, {k: v for k, v in args.items() if k != "out"}]
    for key, value in args.items():
        variants += [{**args, key: s} for s in spoiled(value)]
    for top in (-1, 0, 33, 70, 71):
        if "top" in args:
            variants.append({**args, "top": top})
    for eps in (-1.0, float("nan"), 0.0):
        if "eps" in args:
            variants.append({**args, "eps": eps})
    cf.lib()
    native = [outcome(call, v) for v in variants]
    monkeypatch.setattr(cf, "_args", None)
    accepted = 0
    for i, v in enumerate(variants):
        want = outcome(call, v)
        if isinstance(want, list):
            assert isinstance(native[i], list), (i, native[i])
            assert len(want) == len(native[i])
            for a, b in zip(native[i], want):
                assert a.shape == b.shape and a.dtype == b.dtype
                assert torch.equal(a.view(torch.int8), b.view(torch.int8)), i
            accepted += 1
        else:
            assert native[i] == want, (i, native[i], want)
    assert accepted >= 2 and isinstance(native[0], list)


def test_choices_without_a_truth_value():
    """A tensor of several elements where a call asks yes or no: torch's own error."""
    x = randn(1, (4, 64), torch.float16).cuda()
    _, stats, ck = cf.layer_norm_forward_save(x)
    two = torch.ones(2)
    for call in (lambda: cf.layer_norm_forward_save(x, checkpoint=two),
                 lambda: cf.layer_norm_backward(x, ck, stats, param_grads=two),
                 lambda: cf.act_forward_save(x, checkpoint_out=two)):
        with pytest.raises(RuntimeError, match="ambiguous"):
            call()


def test_negated_views_are_refused():
    """A view whose memory holds the negatives of its values (the imaginary part of
    a conjugate) is not what a kernel would read."""
    z = torch.randn(5, 1, dtype=torch.complex64, device="cuda").conj().imag
    assert z.is_neg()
    with pytest.raises(ValueError, match="negated"):
        cf.log_probs_forward(z)
    x = randn(1, (5, 1), torch.float16).cuda()
    with pytest.raises(ValueError, match="negated"):
        cf.layer_norm_forward(x, z[0])
    assert cf.log_probs_forward(z.resolve_neg()).entropy.shape == (5,)
