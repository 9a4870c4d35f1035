"""Argument checks of the training and scoring operators on a host without a
GPU: the C ABI refuses before any HIP call (made-up addresses are never read),
and the binding refuses host tensors."""
import ctypes
import os

import pytest
import torch

import paper_2404_03617_amd as cf
from paper_2404_03617_amd import training

needs_library = pytest.mark.skipif(not os.path.exists(cf.library_path()), reason="libconvfirst.so not built")

A, B, Q, S, ST, W, OUT, WS, G1, G2 = (i << 43 for i in range(1, 11))  # apart by more than any tensor
OK, INVALID, UNSUPPORTED, WORKSPACE = cf.CF_OK, cf.CF_ERR_INVALID, cf.CF_ERR_UNSUPPORTED, cf.CF_ERR_WORKSPACE


def norm_forward(x=A, y=B, w=W, b=None, stats=ST, q=Q, scale=S, rows=10, C=100, ldx=100, ldy=100, eps=1e-6, dt=0):
    return cf.lib().cf_layer_norm_forward(x, y, w, b, stats, q, scale, rows, C, ldx, ldy, eps, dt, None)


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(x=None), INVALID), (dict(y=None), INVALID), (dict(rows=-1), INVALID), (dict(C=0), INVALID),
    (dict(dt=2), INVALID), (dict(dt=-1), INVALID), (dict(ldy=99), INVALID), (dict(ldx=-1), INVALID),
    (dict(eps=-1.0), INVALID), (dict(eps=float("nan")), INVALID), (dict(eps=float("inf")), INVALID),
    (dict(q=None), INVALID), (dict(scale=None), INVALID), (dict(x=A + 1), INVALID), (dict(w=W + 2), INVALID),
    (dict(stats=ST + 4), INVALID), (dict(y=A + 2), INVALID), (dict(y=A, ldy=101), INVALID), (dict(q=A), INVALID),
    (dict(stats=B), INVALID), (dict(y=W), INVALID), (dict(C=16385, ldx=16385, ldy=16385), UNSUPPORTED),
    (dict(rows=1 << 40), INVALID), (dict(rows=1 << 24, C=8000, ldx=8000, ldy=8000), UNSUPPORTED),
    (dict(x=None, y=None, rows=0), OK),
])
def test_norm_forward_rejects(kw, status):
    assert norm_forward(**kw) == status
    if status:
        assert cf.lib().cf_last_error().decode().startswith("cf_layer_norm_forward: ")
    else:
        assert cf.lib().cf_last_error() == b""


def norm_backward(dy=A, x=B, q=None, scale=None, stats=ST, w=W, dx=OUT, dw=G1, db=G2, ws=None, nbytes=0, rows=1, C=100,
                  lddy=100, ldx=100, lddx=100, dt=1):
    return cf.lib().cf_layer_norm_backward(dy, x, q, scale, stats, w, dx, dw, db, ws, nbytes, rows, C, lddy, ldx, lddx,
                                           dt, None)


@needs_library
@pytest.mark.parametrize("kw,status", [
    (dict(dy=None), INVALID), (dict(stats=None), INVALID), (dict(dx=None), INVALID), (dict(x=None), INVALID),
    (dict(q=Q, scale=S), INVALID), (dict(x=None, q=Q), INVALID), (dict(dw=None), INVALID), (dict(db=None), INVALID),
    (dict(dw=G1 + 2), INVALID), (dict(dx=B), INVALID), (dict(db=G1), INVALID),
    (dict(lddx=99), INVALID), (dict(rows=5000), WORKSPACE), (dict(rows=5000, ws=WS, nbytes=100), WORKSPACE),
    (dict(rows=5000, ws=WS + 8, nbytes=1 << 30), INVALID), (dict(rows=5000, ws=A, nbytes=1 << 30), INVALID),
    (dict(C=20000, lddy=20000, ldx=20000, lddx=20000), UNSUPPORTED),
])
def test_norm_backward_rejects(kw, status):
    assert norm_backward(**kw) == status


@needs_library
def test_activations_and_checkpoints_reject():
    L = cf.lib()

    def fwd(u=A, h=B, qu=Q, su=S, qh=None, sh=None, rows=4, C=70, ldu=70, ldh=70, dt=0, act=0):
        return L.cf_act_forward(u, h, qu, su, qh, sh, rows, C, ldu, ldh, dt, act, None)

    for kw in (dict(u=None), dict(h=None, qu=None, su=None), dict(su=None), dict(qh=G1), dict(act=3), dict(act=-1),
               dict(dt=2), dict(ldh=69), dict(rows=-2), dict(C=0), dict(h=A + 2), dict(qu=A), dict(qh=Q, sh=G1),
               dict(u=A + 1), dict(su=S + 2)):
        assert fwd(**kw) == INVALID, kw
    assert fwd(rows=1 << 31) == UNSUPPORTED
    assert fwd(rows=0, u=None) == OK
    for kw in (dict(dh=None), dict(q=None), dict(scale=None), dict(du=None), dict(ldd=69), dict(du=Q), dict(act=5),
               dict(du=A + 2)):
        v = dict(dh=A, q=Q, scale=S, du=OUT, ldd=70, act=0)
        v.update(kw)
        assert L.cf_act_backward(v["dh"], v["q"], v["scale"], v["du"], 4, 70, 70, v["ldd"], 0, v["act"], None) == INVALID
    assert L.cf_checkpoint_pack(None, Q, S, 4, 70, 70, 0, None) == INVALID
    assert L.cf_checkpoint_pack(A, None, None, 4, 70, 70, 0, None) == INVALID
    assert L.cf_checkpoint_unpack(Q, S, None, 4, 70, 70, 0, None) == INVALID
    assert L.cf_checkpoint_unpack(Q, S, A, 4, 70, 69, 0, None) == INVALID


@needs_library
def test_columns_of_one_buffer_do_not_overlap():
    """Rows of 140: columns 0..69 and 70..139 are apart, 0..69 and 69..138 not."""
    L = cf.lib()
    assert L.cf_act_forward(A, A + 138, None, None, None, None, 4, 70, 140, 140, 0, 0, None) == INVALID
    # apart: only the next check (a size without a grid) refuses
    assert L.cf_act_forward(A, A + 140, None, None, None, None, 1 << 28, 70, 140, 140, 0, 0, None) == UNSUPPORTED
    assert L.cf_act_forward(A + 140, A, None, None, None, None, 1 << 28, 70, 140, 140, 0, 0, None) == UNSUPPORTED
    assert L.cf_act_forward(A + 140, A + 2, None, None, None, None, 1 << 28, 70, 140, 140, 0, 0, None) == INVALID


@needs_library
def test_weight_grad_rejects():
    L = cf.lib()

    def call(dy=A, q=Q, scale=S, stats=ST, w=W, b=None, dw=OUT, db=G1, ws=None, nbytes=0, rows=64, K=64, C=64, lddy=64,
             dt=0):
        return L.cf_linear_weight_grad(dy, q, scale, stats, w, b, dw, db, ws, nbytes, rows, K, C, lddy, dt, None)

    for kw in (dict(dy=None), dict(q=None), dict(scale=None), dict(dw=None), dict(db=None), dict(stats=None),
               dict(stats=None, w=None, b=B), dict(rows=-1), dict(K=0), dict(C=0), dict(lddy=-1), dict(dt=2),
               dict(dw=A), dict(db=OUT), dict(stats=ST + 4), dict(dw=OUT + 1)):
        assert call(**kw) == INVALID, kw
    assert call(K=(1 << 20) + 1, lddy=(1 << 20) + 1) == UNSUPPORTED
    assert call(rows=400000) == WORKSPACE
    need = L.cf_linear_weight_grad_workspace_bytes(400000, 64, 64)
    assert need > 0 and call(rows=400000, ws=WS, nbytes=need - 1) == WORKSPACE
    assert call(rows=400000, ws=S + 1024, nbytes=need) == INVALID
    assert L.cf_linear_weight_grad_workspace_bytes(0, 64, 64) == 0
    assert L.cf_linear_weight_grad_workspace_bytes(10, 0, 64) == 0


@needs_library
def test_log_probs_reject():
    L = cf.lib()

    def call(z=A, t=B, lp=Q, h=S, st=ST, tl=None, ti=None, top=0, ws=None, nbytes=0, rows=600, V=100, ldz=100, dt=2):
        return L.cf_log_probs_forward(z, t, lp, h, st, tl, ti, top, ws, nbytes, rows, V, ldz, dt, None)

    for kw in (dict(z=None), dict(h=None), dict(t=None), dict(lp=None), dict(top=3), dict(tl=G1, ti=G2), dict(dt=3),
               dict(top=101, tl=G1, ti=G2), dict(top=-1), dict(V=0), dict(rows=-1), dict(z=A + 2), dict(t=B + 4),
               dict(h=Q), dict(st=S), dict(ldz=-4), dict(st=ST + 4)):
        assert call(**kw) == INVALID, kw
    assert call(top=33, tl=G1, ti=G2) == UNSUPPORTED
    assert call(rows=1 << 25) == UNSUPPORTED
    assert call(rows=1, V=100000, ldz=100000) == WORKSPACE
    assert call(rows=0, z=None) == OK

    def back(z=A, t=B, st=ST, h=S, gl=G1, gh=None, dz=OUT, rows=6, V=100, ldz=100, lddz=100, dt=0):
        return L.cf_log_probs_backward(z, t, st, h, gl, gh, dz, rows, V, ldz, lddz, dt, None)

    for kw in (dict(z=None), dict(st=None), dict(h=None), dict(dz=None), dict(gl=None), dict(t=None), dict(lddz=99),
               dict(dz=A + 2), dict(dz=A, lddz=104), dict(dt=3), dict(dz=G1)):
        assert back(**kw) == INVALID, kw


@pytest.fixture
def no_library(monkeypatch):
    def fail():
        raise AssertionError("the library must not be reached")

    monkeypatch.setattr(cf, "lib", fail)


def test_host_tensors_are_refused(no_library):
    x = torch.zeros(4, 64, dtype=torch.float16)
    ck = cf.Checkpoint(torch.zeros(4, 64, dtype=torch.int8), torch.zeros(4, 1), torch.float16)
    t = torch.zeros(4, dtype=torch.int64)
    for call in (lambda: cf.layer_norm_forward(x), lambda: cf.layer_norm_forward_save(x),
                 lambda: cf.layer_norm_backward(x, x, torch.zeros(4, 2)), lambda: cf.checkpoint_pack(x),
                 lambda: cf.checkpoint_unpack(ck), lambda: cf.act_forward(x), lambda: cf.act_forward_save(x),
                 lambda: cf.act_backward(x, ck), lambda: cf.linear_weight_grad(x, ck),
                 lambda: cf.log_probs_forward(x, t), lambda: cf.log_probs_backward(x, t, None)):
        with pytest.raises(ValueError, match="GPU"):
            call()


def test_types_are_refused(no_library):
    for call in (lambda: cf.layer_norm_forward([1.0]), lambda: cf.act_forward(None),
                 lambda: cf.log_probs_forward("logits"), lambda: cf.checkpoint_unpack(torch.zeros(3))):
        with pytest.raises(TypeError):
            call()
    with pytest.raises(ValueError, match="dtype"):
        cf.layer_norm_forward(torch.zeros(4, 64, dtype=torch.float64))


def test_checkpoint_sizes():
    ck = cf.Checkpoint(torch.zeros(6, 130, dtype=torch.int8), torch.zeros(6, 3), torch.float16)
    assert ck.shape == (6, 130) and ck.nbytes() == 6 * 130 + 4 * 18
    assert training.CKPT_BLOCK == 64


@needs_library
def test_no_rows_need_no_statistics():
    """The address of an empty tensor is null: with weight and bias of a norm but
    no statistics, only the next check (of the size) refuses a call without rows."""
    L, K = cf.lib(), (1 << 20) + 1
    for rows, status in ((0, UNSUPPORTED), (1, INVALID)):
        assert L.cf_linear_weight_grad(A, Q, S, None, W, B, OUT, G1, None, 0, rows, K, 64, K, 0, None) == status


@needs_library
def test_backward_of_long_rows_that_start_anywhere_has_a_grid():
    """Rows of 4096 fp32 logits that do not start at 16 bytes take two workgroups
    each: 2^23 of them are 2^32 threads."""
    L, rows, V = cf.lib(), 1 << 23, 4096
    for z, ldz in ((A + 4, V), (A, V + 1)):
        assert L.cf_log_probs_backward(z, B, ST, S, G1, None, OUT, rows, V, ldz, V, 2, None) == UNSUPPORTED


def test_the_two_copies_of_gelus_tail_agree():
    """GELU (cf_device.h) and its slope (cf_ckpt.hip) evaluate the same q(t)."""
    import re

    csrc = os.path.join(os.path.dirname(cf.__file__), "csrc")

    def tail(name, function):
        text = open(os.path.join(csrc, name)).read()
        body = text[text.index(function):]
        body = body[:body.index("exp2f")]
        return re.findall(r"fmaf\([^;]*?(-?0\.\d{6,})f(?:, t, (-?0\.\d+)f)?\)", body)

    a, b = tail("cf_device.h", "float gelu_f32("), tail("cf_ckpt.hip", "float gelu_slope(")
    assert a == b and len(a) == 5, (a, b)
