"""Training and scoring operators: layer norm with its gradients, activations
kept in 8 bits for the backward pass and the gradients that read them, and log
probabilities of classes or tokens with entropy, alternatives and gradient.

Bindings over the C ABI of ``include/convfirst.h``, like the rest of the
package: torch supplies memory and streams, the library the arithmetic.
Tensors are [..., C] in fp16 or bf16 (logits in fp32 too) on the GPU: NHWC
activations, or rows of tokens.  Their last dimension is contiguous and the
others are rows at one stride, so slices of the channels of a wider tensor will
do, and as inputs rows that were expanded.  Parameters and statistics are fp32.
Gradients are what the calls named _backward and _grad return: as everywhere in
the package a tensor that requires gradients is read like any other, and results
have no autograd graph.
"""
from __future__ import annotations

import ctypes
from typing import NamedTuple, Optional

import torch

import paper_2404_03617_amd as _cf

CKPT_BLOCK = 64  # channels that share a scale of a checkpoint
_CODES = {torch.float16: 0, torch.bfloat16: 1, torch.float32: 2, torch.int8: 3, torch.int64: 4}
_DTYPE_OF = {v: k for k, v in _CODES.items()}


class Checkpoint:
    """Activations [..., C] in 8 bits: q int8 [..., C] and, for each 64
    channels of a row, scale fp32 [..., ceil(C / 64)]; dtype is that of the
    tensor kept.  Both are contiguous; x is near q * scale, within 1/254 of the
    largest magnitude of its 64 channels."""

    __slots__ = ("q", "scale", "dtype")

    def __init__(self, q: torch.Tensor, scale: torch.Tensor, dtype: torch.dtype):
        self.q, self.scale, self.dtype = q, scale, dtype

    @property
    def shape(self):
        return self.q.shape

    def nbytes(self) -> int:
        return self.q.numel() + 4 * self.scale.numel()


class LogProbs(NamedTuple):
    """What log_probs_forward returns, each [...] of the logits' leading
    dimensions, in fp32: logp (None without tokens), entropy, stats [..., 2]
    (the largest logit and the log of the sum of exp(logit - largest): their sum
    is the log of the partition sum), and top_logp and int64 top_ids [..., top]
    (None for top = 0)."""
    logp: Optional[torch.Tensor]
    entropy: torch.Tensor
    stats: torch.Tensor
    top_logp: Optional[torch.Tensor]
    top_ids: Optional[torch.Tensor]


# ---------------------------------------------------------------------------
# Native calls (csrc/host/cf_calls.cpp): checks, outputs and the library's call in
# one function.  They give None for what is not theirs (a stream or workspace of
# the caller's, anything wrong), and the functions below go on in Python.  A call
# on little data, back to back, through Python's checks and ctypes and through
# here: layer norm of one row of 512 9.6 and 4.1 us, weight gradient of 49 rows
# 13.5 and 5.8, scoring of 128 rows of 1000 with five alternatives 18.2 and 7.3,
# of one row of 131072 with eight 22.5 and 10.9.

_BOUND = ("cf_layer_norm_forward", "cf_layer_norm_backward", "cf_layer_norm_backward_workspace_bytes",
          "cf_act_forward", "cf_act_backward", "cf_checkpoint_unpack", "cf_linear_weight_grad",
          "cf_linear_weight_grad_workspace_bytes", "cf_log_probs_forward", "cf_log_probs_workspace_bytes",
          "cf_log_probs_backward", "cf_group_norm_forward", "cf_group_norm_workspace_bytes", "cf_group_norm_backward",
          "cf_group_norm_backward_workspace_bytes", "cf_gated_ffn_forward", "cf_gated_ffn_workspace_bytes",
          "cf_gated_ffn_backward", "cf_gated_ffn_backward_workspace_bytes", "cf_linear_log_probs_forward",
          "cf_linear_log_probs_workspace_bytes", "cf_linear_log_probs_backward",
          "cf_linear_log_probs_backward_workspace_bytes")


def _native(name, *args):
    """The native call's result; None where it is not for this one."""
    if _cf._args is None:
        return None
    r = getattr(_cf._args, name)(*args)
    if type(r) is int:
        _cf._check(r)
    return r


def _bind(L):
    """Gives the native calls the library's functions."""
    if _cf._args is not None:
        _cf._args.bind(tuple(ctypes.cast(getattr(L, f), ctypes.c_void_p).value for f in _BOUND))


# ---------------------------------------------------------------------------
# Argument checks: the native ones say yes, those below name what is wrong.


def _rows(name, t, kinds):
    """(address, rows, C, row stride, dtype code) of a tensor of rows whose
    dtype is one of the first `kinds` codes."""
    d = None if _cf._args is None else _cf._args.rows(t)
    if d is None:
        d = _rows_checked(name, t)
    if d[4] >= kinds:
        raise ValueError("%s must be %s" % (name, "float16 or bfloat16" if kinds == 2 else
                                            "float16, bfloat16 or float32"))
    return d


def _not_negated(name, t):
    """Memory that holds the negatives of a view's values is refused."""
    if t.is_neg():
        raise ValueError("%s is a negated view: resolve_neg() gives a tensor with its values" % name)


def _rows_checked(name, t):
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dim() < 1:
        raise ValueError("%s must be [..., C]" % name)
    if t.dtype not in _CODES:
        raise ValueError("%s has dtype %s" % (name, t.dtype))
    if t.device.type != "cuda":
        raise ValueError("%s must be a GPU tensor (got device %s)" % (name, t.device))
    _not_negated(name, t)
    C = t.shape[-1]
    if C > 1 and t.stride(-1) != 1:
        raise ValueError("%s must be contiguous in its last dimension" % name)
    n, ld = 1, None
    for size, stride in zip(reversed(t.shape[:-1]), reversed(t.stride()[:-1])):
        if size != 1:
            if ld is None:
                ld = stride
            elif stride != ld * n:
                raise ValueError("%s: the leading dimensions must be rows at one stride, got shape %s, strides %s"
                                 % (name, tuple(t.shape), t.stride()))
        n *= size
        if n == 0:
            break
    return t.data_ptr(), n, C, C if ld is None or n == 0 else ld, _CODES[t.dtype]


def _flat(name, x, t, code, n, last):
    """Address of a contiguous tensor of n rows of `last` elements (last = 0: n
    elements) of that dtype on x's device; None for None."""
    if t is None:
        return None
    p = None if _cf._args is None else _cf._args.flat(x, t, code, n, last)
    if p is not None:
        return p
    if not isinstance(t, torch.Tensor):
        raise TypeError("%s must be a torch.Tensor" % name)
    if t.dtype != _DTYPE_OF[code]:
        raise ValueError("%s must be %s, got %s" % (name, _DTYPE_OF[code], t.dtype))
    if t.numel() != n * (last or 1) or (last and (t.dim() < 1 or t.shape[-1] != last)):
        raise ValueError("%s has shape %s, expected %d%s elements" % (name, tuple(t.shape), n,
                                                                      " rows of %d" % last if last else ""))
    if not t.is_contiguous():
        raise ValueError("%s must be contiguous" % name)
    _not_negated(name, t)
    if t.device != x.device:
        raise ValueError("%s is on %s but the input is on %s" % (name, t.device, x.device))
    return t.data_ptr()


def _like(name, x, t, shape, code):
    """(address, row stride) of another tensor of rows: x's device, this shape
    and dtype."""
    p, _, C, ld, have = _rows(name, t, 3)
    if have != code:
        raise ValueError("%s must be %s, got %s" % (name, _DTYPE_OF[code], t.dtype))
    if t.shape != shape:
        raise ValueError("%s must have shape %s, got %s" % (name, tuple(shape), tuple(t.shape)))
    if t.device != x.device:
        raise ValueError("%s is on %s but the input is on %s" % (name, t.device, x.device))
    return p, ld


def _out_rows(x, out, shape, code, stream):
    """(tensor, address, row stride) of an output: the caller's, or a new one."""
    if out is None:
        out = _cf._new(x, shape, stream, _DTYPE_OF[code])
        return out, out.data_ptr(), shape[-1]
    return (out, *_like("out", x, out, shape, code))


def _blocks(C: int) -> int:
    return -(-C // CKPT_BLOCK)


def _new_checkpoint(x, stream):
    return Checkpoint(_cf._new(x, x.shape, stream, torch.int8),
                      _cf._new(x, (*x.shape[:-1], _blocks(x.shape[-1])), stream, torch.float32), x.dtype)


def _checkpoint(name, ck, x, rows, C):
    """Addresses of a checkpoint of `rows` rows of C channels on x's device."""
    return (_flat(name + ".q", x, ck.q, 3, rows, C), _flat(name + ".scale", x, ck.scale, 2, rows, _blocks(C)))


def _of_checkpoint(name, ck):
    """(rows, C, dtype code) of a checkpoint argument."""
    if not isinstance(ck, Checkpoint):
        raise TypeError("%s must be a Checkpoint" % name)
    if not isinstance(ck.q, torch.Tensor) or ck.q.dim() < 1 or ck.q.dtype != torch.int8:
        raise ValueError("%s.q must be an int8 tensor [..., C]" % name)
    if ck.q.device.type != "cuda":
        raise ValueError("%s must be on a GPU (got device %s)" % (name, ck.q.device))
    if ck.dtype not in _cf.DTYPES:
        raise ValueError("%s must be of float16 or bfloat16 activations" % name)
    C = ck.q.shape[-1]
    return (ck.q.numel() // C if C else 0), C, _CODES[ck.dtype]


def _act(act):
    if act not in _cf.ACTS:
        raise ValueError("act must be one of %s" % sorted(_cf.ACTS))
    return _cf.ACTS[act]


def _ws(x, ws, need, stream):
    """(tensor, address, bytes) of the caller's workspace or a new one."""
    ws = _cf._workspace(x, ws, need, stream)
    return (None, None, 0) if ws is None else (ws, ws.data_ptr(), ws.numel())


# ---------------------------------------------------------------------------
# Layer norm


def layer_norm_forward(x: torch.Tensor, weight=None, bias=None, eps: float = 1e-6, out=None,
                       stream=None) -> torch.Tensor:
    """Layer norm over the last dimension (C up to 16384), for inference: y =
    weight * (x - mean) / sqrt(var + eps) + bias, with fp32 weight and bias [C]
    or None.  out may be x."""
    if stream is None:
        y = _native("norm_forward", x, weight, bias, eps, out)
        if y is not None:
            return y
    xp, rows, C, ldx, code = _rows("x", x, 2)
    w, b = _flat("weight", x, weight, 2, C, 0), _flat("bias", x, bias, 2, C, 0)
    y, yp, ldy = _out_rows(x, out, x.shape, code, stream)
    _cf._check(_cf.lib().cf_layer_norm_forward(xp, yp, w, b, None, None, None, rows, C, ldx, ldy, eps, code,
                                               _cf._stream(stream)))
    return y


def layer_norm_forward_save(x: torch.Tensor, weight=None, bias=None, eps: float = 1e-6, checkpoint: bool = True,
                            out=None, stream=None):
    """layer_norm_forward with what layer_norm_backward needs: (y, stats,
    checkpoint), stats fp32 [..., 2] (mean and 1 / standard deviation of each
    row) and the 8-bit checkpoint of x, written in the same pass over x, or None
    where x itself is kept (checkpoint = False)."""
    if stream is None:
        r = _native("norm_forward_save", x, weight, bias, eps, checkpoint, out)
        if r is not None:
            return r[0], r[1], Checkpoint(r[2], r[3], x.dtype) if checkpoint else None
    xp, rows, C, ldx, code = _rows("x", x, 2)
    w, b = _flat("weight", x, weight, 2, C, 0), _flat("bias", x, bias, 2, C, 0)
    y, yp, ldy = _out_rows(x, out, x.shape, code, stream)
    stats = _cf._new(x, (*x.shape[:-1], 2), stream, torch.float32)
    ck = _new_checkpoint(x, stream) if checkpoint else None
    q, scale = (ck.q.data_ptr(), ck.scale.data_ptr()) if checkpoint else (None, None)
    _cf._check(_cf.lib().cf_layer_norm_forward(xp, yp, w, b, stats.data_ptr(), q, scale, rows, C, ldx, ldy, eps, code,
                                               _cf._stream(stream)))
    return y, stats, ck


def layer_norm_backward(dy: torch.Tensor, x, stats: torch.Tensor, weight=None, param_grads: bool = True, out=None,
                        ws=None, stream=None):
    """Gradients of a layer norm: (dx, dweight, dbias), dx in dy's dtype,
    dweight and dbias fp32 [C] (None without param_grads).  x is the norm's
    input or its Checkpoint, stats what layer_norm_forward_save returned.  out
    may be dy.  ws: a uint8 workspace of layer_norm_backward_workspace_bytes()."""
    if stream is None and ws is None:
        ck = (None, x.q, x.scale) if isinstance(x, Checkpoint) else (x, None, None)
        r = _native("norm_backward", dy, *ck, stats, weight, param_grads, out)
        if r is not None:
            return r
    dyp, rows, C, lddy, code = _rows("dy", dy, 2)
    xp, ldx, q, scale = None, C, None, None
    if isinstance(x, Checkpoint):
        q, scale = _checkpoint("x", x, dy, rows, C)
    else:
        xp, ldx = _like("x", dy, x, dy.shape, code)
    sp, w = _flat("stats", dy, stats, 2, rows, 2), _flat("weight", dy, weight, 2, C, 0)
    if sp is None:
        raise TypeError("stats must be a torch.Tensor")
    dx, dxp, lddx = _out_rows(dy, out, dy.shape, code, stream)
    L = _cf.lib()
    dw = db = keep = wp = None
    nbytes = 0
    if param_grads:
        dw, db = _cf._new(dy, (C,), stream, torch.float32), _cf._new(dy, (C,), stream, torch.float32)
        keep, wp, nbytes = _ws(dy, ws, L.cf_layer_norm_backward_workspace_bytes(rows, C), stream)
    _cf._check(L.cf_layer_norm_backward(dyp, xp, q, scale, sp, w, dxp, _cf._ptr(dw), _cf._ptr(db), wp, nbytes, rows,
                                        C, lddy, ldx, lddx, code, _cf._stream(stream)))
    return dx, dw, db


def layer_norm_backward_workspace_bytes(rows: int, C: int) -> int:
    return int(_cf.lib().cf_layer_norm_backward_workspace_bytes(rows, C))


# ---------------------------------------------------------------------------
# Checkpoints and activations


def checkpoint_pack(x: torch.Tensor, stream=None) -> Checkpoint:
    """x [..., C] in 8 bits."""
    if stream is None:
        r = _native("act_forward", x, _cf.ACTS["none"], False, True, False, None)
        if r is not None:
            return Checkpoint(r[1], r[2], x.dtype)
    xp, rows, C, ldx, code = _rows("x", x, 2)
    ck = _new_checkpoint(x, stream)
    _cf._check(_cf.lib().cf_checkpoint_pack(xp, ck.q.data_ptr(), ck.scale.data_ptr(), rows, C, ldx, code,
                                            _cf._stream(stream)))
    return ck


def checkpoint_unpack(ck: Checkpoint, out=None, stream=None) -> torch.Tensor:
    """The values that a checkpoint keeps, in the dtype of the tensor kept."""
    if stream is None and type(ck) is Checkpoint and ck.dtype in _cf.DTYPES:
        x = _native("unpack", ck.q, ck.scale, _CODES[ck.dtype], out)
        if x is not None:
            return x
    rows, C, code = _of_checkpoint("ck", ck)
    q, scale = _checkpoint("ck", ck, ck.q, rows, C)
    x, xp, ldx = _out_rows(ck.q, out, ck.q.shape, code, stream)
    _cf._check(_cf.lib().cf_checkpoint_unpack(q, scale, xp, rows, C, ldx, code, _cf._stream(stream)))
    return x


def act_forward(u: torch.Tensor, act: str = "gelu", out=None, stream=None) -> torch.Tensor:
    """h = act(u), "gelu" (erf), "relu" or "none", in fp32 and rounded once.
    out may be u."""
    if stream is None and act in _cf.ACTS:
        r = _native("act_forward", u, _cf.ACTS[act], True, False, False, out)
        if r is not None:
            return r[0]
    up, rows, C, ldu, code = _rows("u", u, 2)
    a = _act(act)
    h, hp, ldh = _out_rows(u, out, u.shape, code, stream)
    _cf._check(_cf.lib().cf_act_forward(up, hp, None, None, None, None, rows, C, ldu, ldh, code, a,
                                        _cf._stream(stream)))
    return h


def act_forward_save(u: torch.Tensor, act: str = "gelu", checkpoint_out: bool = False, out=None, stream=None):
    """act_forward with checkpoints in the same pass: (h, checkpoint of u for
    act_backward, checkpoint of h for linear_weight_grad of the next layer or,
    without checkpoint_out, None)."""
    if stream is None and act in _cf.ACTS:
        r = _native("act_forward", u, _cf.ACTS[act], True, True, checkpoint_out, out)
        if r is not None:
            return (r[0], Checkpoint(r[1], r[2], u.dtype),
                    Checkpoint(r[3], r[4], u.dtype) if checkpoint_out else None)
    up, rows, C, ldu, code = _rows("u", u, 2)
    a = _act(act)
    h, hp, ldh = _out_rows(u, out, u.shape, code, stream)
    cu = _new_checkpoint(u, stream)
    ch = _new_checkpoint(u, stream) if checkpoint_out else None
    qh, sh = (ch.q.data_ptr(), ch.scale.data_ptr()) if checkpoint_out else (None, None)
    _cf._check(_cf.lib().cf_act_forward(up, hp, cu.q.data_ptr(), cu.scale.data_ptr(), qh, sh, rows, C, ldu, ldh, code,
                                        a, _cf._stream(stream)))
    return h, cu, ch


def act_backward(dh: torch.Tensor, u: Checkpoint, act: str = "gelu", out=None, stream=None) -> torch.Tensor:
    """du = dh * act'(u) with u from its checkpoint.  out may be dh."""
    if stream is None and act in _cf.ACTS and type(u) is Checkpoint:
        du = _native("act_backward", dh, u.q, u.scale, _cf.ACTS[act], out)
        if du is not None:
            return du
    dhp, rows, C, lddh, code = _rows("dh", dh, 2)
    a = _act(act)
    if not isinstance(u, Checkpoint):
        raise TypeError("u must be a Checkpoint")
    q, scale = _checkpoint("u", u, dh, rows, C)
    du, dup, lddu = _out_rows(dh, out, dh.shape, code, stream)
    _cf._check(_cf.lib().cf_act_backward(dhp, q, scale, dup, rows, C, lddh, lddu, code, a, _cf._stream(stream)))
    return du


def _wider(x, dy):
    """Whether a checkpoint's values may lie beyond dy's range."""
    return x.dtype == torch.bfloat16 and getattr(dy, "dtype", None) == torch.float16


def linear_weight_grad(dy: torch.Tensor, x: Checkpoint, stats=None, weight=None, bias=None, ws=None, stream=None):
    """(dW, db) of a linear or point-wise layer y = x W^T + b with W [K, C]:
    dW = dy^T x [K, C] in dy's dtype, db = sums of dy [K] fp32, from the
    checkpoint of x.  With stats (and the norm's weight and bias) the checkpoint
    is of the input of a layer norm whose output was x.  The product takes x in
    dy's dtype, so a float16 dy needs a checkpoint of float16 activations.  ws: a
    uint8 workspace of linear_weight_grad_workspace_bytes()."""
    if stream is None and ws is None and type(x) is Checkpoint and x.dtype in _cf.DTYPES and not _wider(x, dy):
        r = _native("wgrad", dy, x.q, x.scale, stats, weight, bias)
        if r is not None:
            return r
    dyp, rows, K, lddy, code = _rows("dy", dy, 2)
    n, C, _ = _of_checkpoint("x", x)
    if K < 1 or C < 1:
        raise ValueError("dy and x must have channels, got K=%d C=%d" % (K, C))
    if n != rows:
        raise ValueError("dy has %d rows but x has %d" % (rows, n))
    if _wider(x, dy):
        raise ValueError("a checkpoint of bfloat16 activations needs a bfloat16 dy, got %s" % dy.dtype)
    q, scale = _checkpoint("x", x, dy, rows, C)
    sp = _flat("stats", dy, stats, 2, rows, 2)
    w, b = _flat("weight", dy, weight, 2, C, 0), _flat("bias", dy, bias, 2, C, 0)
    L = _cf.lib()
    dw, db = _cf._new(dy, (K, C), stream), _cf._new(dy, (K,), stream, torch.float32)
    keep, wp, nbytes = _ws(dy, ws, L.cf_linear_weight_grad_workspace_bytes(rows, K, C), stream)
    _cf._check(L.cf_linear_weight_grad(dyp, q, scale, sp, w, b, dw.data_ptr(), db.data_ptr(), wp, nbytes, rows, K, C,
                                       lddy, code, _cf._stream(stream)))
    return dw, db


def linear_weight_grad_workspace_bytes(rows: int, K: int, C: int) -> int:
    return int(_cf.lib().cf_linear_weight_grad_workspace_bytes(rows, K, C))


# ---------------------------------------------------------------------------
# Log probabilities


def log_probs_forward(logits: torch.Tensor, tokens=None, top: int = 0, ws=None, stream=None) -> LogProbs:
    """Log probabilities of given tokens (int64 [...], negative: none asked)
    under logits [..., V] in fp16, bf16 or fp32, with the entropy of each row
    and its `top` (at most 32) most probable tokens in order, equal ones by
    index.  Logits of -inf have probability 0.  ws: a uint8 workspace of
    log_probs_workspace_bytes()."""
    if stream is None and ws is None:
        r = _native("log_probs", logits, tokens, top)
        if r is not None:
            return LogProbs(*r)
    zp, rows, V, ldz, code = _rows("logits", logits, 3)
    lead = logits.shape[:-1]
    tp = _flat("tokens", logits, tokens, 4, rows, 0)
    f32, n = torch.float32, int(top)
    logp = None if tp is None else _cf._new(logits, lead, stream, f32)
    entropy, stats = _cf._new(logits, lead, stream, f32), _cf._new(logits, (*lead, 2), stream, f32)
    top_logp = top_ids = None
    if n > 0:
        top_logp, top_ids = _cf._new(logits, (*lead, n), stream, f32), _cf._new(logits, (*lead, n), stream, torch.int64)
    L = _cf.lib()
    keep, wp, nbytes = _ws(logits, ws, L.cf_log_probs_workspace_bytes(rows, V, n), stream)
    _cf._check(L.cf_log_probs_forward(zp, tp, _cf._ptr(logp), entropy.data_ptr(), stats.data_ptr(),
                                      _cf._ptr(top_logp), _cf._ptr(top_ids), n, wp, nbytes, rows, V, ldz, code,
                                      _cf._stream(stream)))
    return LogProbs(logp, entropy, stats, top_logp, top_ids)


def log_probs_workspace_bytes(rows: int, V: int, top: int = 0) -> int:
    return int(_cf.lib().cf_log_probs_workspace_bytes(rows, V, top))


def log_probs_backward(logits: torch.Tensor, tokens, lp: LogProbs, d_logp=None, d_entropy=None, out=None,
                       stream=None) -> torch.Tensor:
    """The gradient of sum(d_logp * lp.logp) + sum(d_entropy * lp.entropy) with
    respect to the logits, in their dtype; lp is what log_probs_forward returned
    for them, d_logp and d_entropy fp32 [...] or None.  out may be logits."""
    if stream is None and type(lp) is LogProbs:
        dz = _native("log_probs_backward", logits, tokens, lp.stats, lp.entropy, d_logp, d_entropy, out)
        if dz is not None:
            return dz
    zp, rows, V, ldz, code = _rows("logits", logits, 3)
    tp = _flat("tokens", logits, tokens, 4, rows, 0)
    sp, ep = _flat("lp.stats", logits, lp.stats, 2, rows, 2), _flat("lp.entropy", logits, lp.entropy, 2, rows, 0)
    gl, gh = _flat("d_logp", logits, d_logp, 2, rows, 0), _flat("d_entropy", logits, d_entropy, 2, rows, 0)
    dz, dzp, lddz = _out_rows(logits, out, logits.shape, code, stream)
    _cf._check(_cf.lib().cf_log_probs_backward(zp, tp, sp, ep, gl, gh, dzp, rows, V, ldz, lddz, code,
                                               _cf._stream(stream)))
    return dz
