"""Operators for heads over features, forward and backward: group norm with an
activation, the gated feed-forward block, and log probabilities of classes or
tokens straight from features and a weight matrix.

Bindings over the C ABI of ``include/convfirst.h``, with the conventions of
training.py: tensors are [..., C] in fp16 or bf16 on the GPU, rows at one
stride; parameters of the norm, statistics and log probabilities are fp32;
weight matrices are in their layer's dtype and may be slices of wider ones.  act
is "silu", "gelu" (erf), "relu" or "none", in fp32.  A call runs on the device of
its tensors, whichever is current.
"""
from __future__ import annotations

import contextlib
from typing import NamedTuple, Optional

import torch

import paper_2404_03617_amd as _cf

from .training import _flat, _like, _native, _out_rows, _rows, _ws

ACTS = {"gelu": 0, "relu": 1, "none": 2, "silu": 3}


class LinearLogProbs(NamedTuple):
    """What linear_log_probs_forward returns, in fp32 and each [...] of the
    features' leading dimensions: logp (None without tokens) and lse, the log of
    the sum of exp(logits)."""
    logp: Optional[torch.Tensor]
    lse: torch.Tensor


def _act(act):
    if act not in ACTS:
        raise ValueError("act must be one of %s" % sorted(ACTS))
    return ACTS[act]


def _on(x):
    """The device of x as the current one, for what is allocated and launched."""
    return contextlib.nullcontext() if x.device.index == torch.cuda.current_device() else torch.cuda.device(x.device)


def _matrix(name, x, t, code, rows, cols):
    """(address, row stride) of a weight [rows, cols] (None: any number) of x's
    dtype and device."""
    p, n, C, ld, have = _rows(name, t, 2)
    if t.dim() != 2:
        raise ValueError("%s must be a matrix, got shape %s" % (name, tuple(t.shape)))
    if have != code:
        raise ValueError("%s must be %s, got %s" % (name, x.dtype, t.dtype))
    if C != cols or (rows is not None and n != rows):
        raise ValueError("%s must have shape [%s, %d], got %s" % (name, "*" if rows is None else rows, cols,
                                                                  tuple(t.shape)))
    if t.device != x.device:
        raise ValueError("%s is on %s but the input is on %s" % (name, t.device, x.device))
    return p, ld


def _some(name, x, t, *args):
    """_flat of an argument that must be there."""
    p = _flat(name, x, t, *args)
    if t is None:
        raise TypeError("%s must be a torch.Tensor" % name)
    return p


def _readable(*rows):
    """Whether the products read rows at these (address, stride) in place."""
    return int(all(p % 16 == 0 and ld % 8 == 0 and ld < 1 << 22 for p, ld in rows))


# ---------------------------------------------------------------------------
# Group norm


def _images(name, x):
    """(address, N, P, C, row stride, dtype code) of feature maps [N, ..., C]."""
    p, rows, C, ld, code = _rows(name, x, 2)
    if x.dim() < 2:
        raise ValueError("%s must be [N, ..., C]" % name)
    N = x.shape[0]
    return p, N, rows // N if N else 0, C, ld, code


def _groups(groups, C):
    if isinstance(groups, bool) or not isinstance(groups, int) or groups < 1 or C % groups:
        raise ValueError("groups must be a positive number that divides the %d channels, got %r" % (C, groups))
    return groups


def _group_norm(x, groups, weight, bias, eps, act, save, out, ws, stream):
    if stream is None and ws is None and act in ACTS:
        r = _native("group_norm", x, groups, weight, bias, eps, ACTS[act], save, out)
        if r is not None:
            return r
    xp, N, P, C, ldx, code = _images("x", x)
    G, a = _groups(groups, C), _act(act)
    w, b = _flat("weight", x, weight, 2, C, 0), _flat("bias", x, bias, 2, C, 0)
    with _on(x):
        y, yp, ldy = _out_rows(x, out, x.shape, code, stream)
        stats = _cf._new(x, (N, G, 2), stream, torch.float32) if save else None
        L = _cf.lib()
        keep, wp, nbytes = _ws(x, ws, L.cf_group_norm_workspace_bytes(N, P, C, G), stream)
        _cf._check(L.cf_group_norm_forward(xp, yp, w, b, _cf._ptr(stats), wp, nbytes, N, P, C, G, ldx, ldy, eps, code,
                                           a, _cf._stream(stream)))
    return y, stats


def group_norm_forward(x: torch.Tensor, groups: int, weight=None, bias=None, eps: float = 1e-6, act: str = "none",
                       out=None, ws=None, stream=None) -> torch.Tensor:
    """Group norm over feature maps [N, ..., C], channels last, and an
    activation, for inference: y = act(weight * (x - mean) / sqrt(var + eps) +
    bias), mean and var over all pixels of an image and the C / groups channels
    of a group; fp32 weight and bias [C] or None.  out may be x.  ws: a uint8
    workspace of group_norm_workspace_bytes()."""
    return _group_norm(x, groups, weight, bias, eps, act, False, out, ws, stream)[0]


def group_norm_forward_save(x: torch.Tensor, groups: int, weight=None, bias=None, eps: float = 1e-6,
                            act: str = "none", out=None, ws=None, stream=None):
    """group_norm_forward with what group_norm_backward needs besides x: (y,
    stats), stats fp32 [N, groups, 2] (mean and 1 / standard deviation)."""
    return _group_norm(x, groups, weight, bias, eps, act, True, out, ws, stream)


def group_norm_workspace_bytes(x_shape, groups: int) -> int:
    N, P, C = x_shape[0], _pixels(x_shape), x_shape[-1]
    return int(_cf.lib().cf_group_norm_workspace_bytes(N, P, C, groups))


def _pixels(shape):
    n = 1
    for s in shape[1:-1]:
        n *= s
    return n


def group_norm_backward(dy: torch.Tensor, x: torch.Tensor, stats: torch.Tensor, weight=None, bias=None,
                        act: str = "none", param_grads: bool = True, out=None, ws=None, stream=None):
    """Gradients of group_norm_forward_save: (dx, dweight, dbias), dx in dy's
    dtype, dweight and dbias fp32 [C] (None without param_grads), from the forward
    call's x, weight, bias, act and stats.  out may be dy.  ws: a uint8 workspace
    of group_norm_backward_workspace_bytes()."""
    if stream is None and ws is None and act in ACTS:
        r = _native("group_norm_backward", dy, x, stats, weight, bias, ACTS[act], param_grads, out)
        if r is not None:
            return r
    dyp, N, P, C, lddy, code = _images("dy", dy)
    xp, ldx = _like("x", dy, x, dy.shape, code)
    if not isinstance(stats, torch.Tensor) or stats.dim() != 3:
        raise ValueError("stats must be [N, groups, 2], as group_norm_forward_save returns it")
    G, a = _groups(int(stats.shape[1]), C), _act(act)
    sp = _some("stats", dy, stats, 2, N * G, 2)
    w, b = _flat("weight", dy, weight, 2, C, 0), _flat("bias", dy, bias, 2, C, 0)
    with _on(dy):
        dx, dxp, lddx = _out_rows(dy, out, dy.shape, code, stream)
        L = _cf.lib()
        dw = db = None
        if param_grads:
            dw, db = _cf._new(dy, (C,), stream, torch.float32), _cf._new(dy, (C,), stream, torch.float32)
        keep, wp, nbytes = _ws(dy, ws, L.cf_group_norm_backward_workspace_bytes(N, P, C, G), stream)
        _cf._check(L.cf_group_norm_backward(dyp, xp, sp, w, b, dxp, _cf._ptr(dw), _cf._ptr(db), wp, nbytes, N, P, C, G,
                                            lddy, ldx, lddx, code, a, _cf._stream(stream)))
    return dx, dw, db


def group_norm_backward_workspace_bytes(x_shape, groups: int) -> int:
    N, P, C = x_shape[0], _pixels(x_shape), x_shape[-1]
    return int(_cf.lib().cf_group_norm_backward_workspace_bytes(N, P, C, groups))


# ---------------------------------------------------------------------------
# Gated feed-forward block


def _gated_weights(x, w_gate, w_up, w_down, C, code):
    """(hidden channels, (address, stride) of each weight)"""
    if not isinstance(w_gate, torch.Tensor) or w_gate.dim() != 2:
        raise ValueError("w_gate must be a matrix [hidden, %d]" % C)
    H = int(w_gate.shape[0])
    if C < 1 or H < 1:
        raise ValueError("x and the weights must have channels, got C=%d hidden=%d" % (C, H))
    return H, (_matrix("w_gate", x, w_gate, code, H, C), _matrix("w_up", x, w_up, code, H, C),
               _matrix("w_down", x, w_down, code, C, H))


def _gated(x, w_gate, w_up, w_down, act, save, out, ws, stream):
    if stream is None and ws is None and act in ACTS:
        r = _native("gated", x, w_gate, w_up, w_down, ACTS[act], save, out)
        if r is not None:
            return r
    xp, rows, C, ldx, code = _rows("x", x, 2)
    a = _act(act)
    H, (g, u, d) = _gated_weights(x, w_gate, w_up, w_down, C, code)
    with _on(x):
        y, yp, ldy = _out_rows(x, out, x.shape, code, stream)
        saved = _cf._new(x, (*x.shape[:-1], 2 * H), stream, torch.float32) if save else None
        L = _cf.lib()
        plain = _readable((xp, ldx), g, u, d) if g[1] == u[1] else 0
        keep, wp, nbytes = _ws(x, ws, L.cf_gated_ffn_workspace_bytes(rows, C, H, plain), stream)
        _cf._check(L.cf_gated_ffn_forward(xp, g[0], u[0], d[0], yp, _cf._ptr(saved), wp, nbytes, rows, C, H, ldx, g[1],
                                          u[1], d[1], ldy, code, a, _cf._stream(stream)))
    return y, saved


def gated_ffn_forward(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                      act: str = "silu", out=None, ws=None, stream=None) -> torch.Tensor:
    """Gated feed-forward block for inference: y = (act(x w_gate^T) * (x
    w_up^T)) w_down^T over rows x [..., C], with w_gate and w_up [hidden, C] and
    w_down [C, hidden] in x's dtype.  out may not overlap x.  ws: a uint8 workspace
    of gated_ffn_workspace_bytes()."""
    return _gated(x, w_gate, w_up, w_down, act, False, out, ws, stream)[0]


def gated_ffn_forward_save(x: torch.Tensor, w_gate: torch.Tensor, w_up: torch.Tensor, w_down: torch.Tensor,
                           act: str = "silu", out=None, ws=None, stream=None):
    """gated_ffn_forward with what gated_ffn_backward needs besides its inputs:
    (y, saved), saved fp32 [..., 2 * hidden]: x w_gate^T and x w_up^T."""
    return _gated(x, w_gate, w_up, w_down, act, True, out, ws, stream)


def gated_ffn_workspace_bytes(rows: int, C: int, hidden: int, aligned: bool = False) -> int:
    """aligned: the call's tensors start at 16-byte aligned addresses, their row
    strides are multiples of 8 elements (below 2^22), and those of w_gate and w_up
    are the same; otherwise there is room for copies of them."""
    return int(_cf.lib().cf_gated_ffn_workspace_bytes(rows, C, hidden, int(bool(aligned))))


def gated_ffn_backward(dy: torch.Tensor, x: torch.Tensor, saved: torch.Tensor, w_gate: torch.Tensor,
                       w_up: torch.Tensor, w_down: torch.Tensor, act: str = "silu", out=None, ws=None, stream=None):
    """Gradients of gated_ffn_forward_save: (dx, dw_gate, dw_up, dw_down), all in
    dy's dtype, from the forward call's x, weights, act and saved.  ws: a uint8
    workspace of gated_ffn_backward_workspace_bytes()."""
    if stream is None and ws is None and act in ACTS:
        r = _native("gated_backward", dy, x, saved, w_gate, w_up, w_down, ACTS[act], out)
        if r is not None:
            return r
    dyp, rows, C, lddy, code = _rows("dy", dy, 2)
    xp, ldx = _like("x", dy, x, dy.shape, code)
    a = _act(act)
    H, (g, u, d) = _gated_weights(dy, w_gate, w_up, w_down, C, code)
    sp = _some("saved", dy, saved, 2, rows, 2 * H)
    with _on(dy):
        dx, dxp, lddx = _out_rows(dy, out, dy.shape, code, stream)
        dg, du, dd = (_cf._new(dy, shape, stream) for shape in ((H, C), (H, C), (C, H)))
        L = _cf.lib()
        plain = _readable((dyp, lddy), (xp, ldx), g, u, d) if g[1] == u[1] else 0
        keep, wp, nbytes = _ws(dy, ws, L.cf_gated_ffn_backward_workspace_bytes(rows, C, H, plain), stream)
        _cf._check(L.cf_gated_ffn_backward(dyp, xp, sp, g[0], u[0], d[0], dxp, dg.data_ptr(), du.data_ptr(),
                                           dd.data_ptr(), wp, nbytes, rows, C, H, lddy, ldx, g[1], u[1], d[1], lddx,
                                           code, a, _cf._stream(stream)))
    return dx, dg, du, dd


def gated_ffn_backward_workspace_bytes(rows: int, C: int, hidden: int, aligned: bool = False) -> int:
    """aligned: as for gated_ffn_workspace_bytes."""
    return int(_cf.lib().cf_gated_ffn_backward_workspace_bytes(rows, C, hidden, int(bool(aligned))))


# ---------------------------------------------------------------------------
# Log probabilities from features


def _classifier(x, weight, C, code):
    if not isinstance(weight, torch.Tensor) or weight.dim() != 2:
        raise ValueError("weight must be a matrix [classes, %d]" % C)
    V = int(weight.shape[0])
    if C < 1 or V < 1:
        raise ValueError("x must have channels and weight classes, got C=%d V=%d" % (C, V))
    return V, _matrix("weight", x, weight, code, V, C)


def linear_log_probs_forward(x: torch.Tensor, weight: torch.Tensor, tokens=None, ws=None,
                             stream=None) -> LinearLogProbs:
    """Log probabilities of given tokens (int64 [...], negative: none asked,
    logp 0) under the logits x weight^T of features x [..., C] and a classifier's
    weight [V, C] in x's dtype, whose logits are never kept, and their lse.  ws: a
    uint8 workspace of linear_log_probs_workspace_bytes()."""
    if stream is None and ws is None:
        r = _native("linear", x, weight, tokens)
        if r is not None:
            return LinearLogProbs(*r)
    xp, rows, C, ldx, code = _rows("x", x, 2)
    V, (w, ldw) = _classifier(x, weight, C, code)
    tp = _flat("tokens", x, tokens, 4, rows, 0)
    lead = x.shape[:-1]
    with _on(x):
        logp = None if tokens is None else _cf._new(x, lead, stream, torch.float32)
        lse = _cf._new(x, lead, stream, torch.float32)
        L = _cf.lib()
        need = L.cf_linear_log_probs_workspace_bytes(rows, C, V, _readable((xp, ldx), (w, ldw)))
        keep, wp, nbytes = _ws(x, ws, need, stream)
        _cf._check(L.cf_linear_log_probs_forward(xp, w, tp, _cf._ptr(logp), lse.data_ptr(), wp, nbytes, rows, C, V,
                                                 ldx, ldw, code, _cf._stream(stream)))
    return LinearLogProbs(logp, lse)


def linear_log_probs_workspace_bytes(rows: int, C: int, V: int, aligned: bool = False) -> int:
    """aligned: x and weight start at 16-byte aligned addresses and their row
    strides are multiples of 8 elements (below 2^22); otherwise there is room for
    copies of them."""
    return int(_cf.lib().cf_linear_log_probs_workspace_bytes(rows, C, V, int(bool(aligned))))


def linear_log_probs_backward(x: torch.Tensor, weight: torch.Tensor, tokens, lp: LinearLogProbs, d_logp=None,
                              d_lse=None, out=None, ws=None, stream=None):
    """The gradients (dx, dweight), in x's dtype, of sum(d_logp * lp.logp) +
    sum(d_lse * lp.lse); lp is what linear_log_probs_forward returned (for d_logp,
    with these tokens), d_logp and d_lse fp32 [...] or None.  Rows without a
    gradient (both 0, or d_logp of a negative token) add nothing to dweight, whatever
    their features hold.  In fp16 a row adds to dweight with all bits where gradient
    times feature is at least 2^-28 of the largest such product.  ws: a uint8
    workspace of linear_log_probs_backward_workspace_bytes()."""
    if stream is None and ws is None and type(lp) is LinearLogProbs:
        r = _native("linear_backward", x, weight, tokens, lp.logp, lp.lse, d_logp, d_lse, out)
        if r is not None:
            return r
    xp, rows, C, ldx, code = _rows("x", x, 2)
    V, (w, ldw) = _classifier(x, weight, C, code)
    tp = _flat("tokens", x, tokens, 4, rows, 0)
    pp, sp = _flat("lp.logp", x, lp.logp, 2, rows, 0), _some("lp.lse", x, lp.lse, 2, rows, 0)
    gl, gs = _flat("d_logp", x, d_logp, 2, rows, 0), _flat("d_lse", x, d_lse, 2, rows, 0)
    with _on(x):
        dx, dxp, lddx = _out_rows(x, out, x.shape, code, stream)
        dw = _cf._new(x, (V, C), stream)
        L = _cf.lib()
        need = L.cf_linear_log_probs_backward_workspace_bytes(rows, C, V, _readable((xp, ldx), (w, ldw)))
        keep, wp, nbytes = _ws(x, ws, need, stream)
        _cf._check(L.cf_linear_log_probs_backward(xp, w, tp, pp, sp, gl, gs, dxp, dw.data_ptr(), wp, nbytes, rows, C,
                                                  V, ldx, ldw, lddx, code, _cf._stream(stream)))
    return dx, dw


def linear_log_probs_backward_workspace_bytes(rows: int, C: int, V: int, aligned: bool = False) -> int:
    """aligned: as for linear_log_probs_workspace_bytes."""
    return int(_cf.lib().cf_linear_log_probs_backward_workspace_bytes(rows, C, V, int(bool(aligned))))
