"""Performance cases of the training and scoring operators: what a program
calls that fine-tunes a norm, an FFN and a classifier over ConvFirst features,
or that scores classes or tokens from their logits.

A case is a dict of plain values.  ``kind`` names what one pass does:

  norm         layer_norm_forward                              y
  norm_train   layer_norm_forward_save, layer_norm_backward    y, dx, dweight, dbias
               (`ckpt`: the backward pass reads the 8-bit checkpoint of x that
               the forward pass wrote, else x itself)
  pack         checkpoint_pack, checkpoint_unpack              the values that come back
  act_train    act_forward_save, act_backward                  h, du
  wgrad        linear_weight_grad                              dW, db
               (`norm`: the linear layer's input was the layer norm of the
               checkpointed tensor)
  score        log_probs_forward                               logp, entropy, top values and ids
  score_train  log_probs_forward, log_probs_backward           logp, entropy, dlogits

``own`` false: the same in elementary torch operations in 32 bits, rounded
once at the end.  The 8-bit checkpoint of a row keeps, for each block of 64
channels with the largest magnitude a, q = rint(x * (127 / a)) and the scale
a * (1 / 127); a block with a < 2^-119 is kept as zeros.
"""
import math

import torch

own = False

DTYPES = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
BLOCK = 64
EPS = 1e-6


def listed():
    return [
        # The norm before a classifier, on one image's features: what a call costs when there is no work.
        dict(name="norm_1x512_f16", kind="norm", rows=1, C=512, dtype="f16"),
        # Inference over the pixels of a batch-128 third stage.
        dict(name="norm_25088x256_bf16", kind="norm", rows=128 * 14 * 14, C=256, dtype="bf16"),
        # A training step's norm over the pixels of a batch-128 first stage: narrow rows, many of them.
        dict(name="norm_train_401408x64_f16", kind="norm_train", rows=128 * 56 * 56, C=64, dtype="f16", ckpt=True),
        # Wide rows of an odd length, x itself kept: no row but the first is aligned.
        dict(name="norm_train_2999x4095_bf16", kind="norm_train", rows=2999, C=4095, dtype="bf16", ckpt=False),
        # Checkpoint and recall of a second stage's activations.
        dict(name="pack_100352x128_bf16", kind="pack", rows=128 * 28 * 28, C=128, dtype="bf16"),
        # The hidden layer (E = 4) of a batch-128 last stage: activation, checkpoint, gradient.
        dict(name="act_train_6272x2048_f16", kind="act_train", rows=128 * 7 * 7, C=2048, dtype="f16", act="gelu"),
        # Expand layer of the last stage, the pixels of one image: next to no rows to sum over.
        dict(name="wgrad_49x2048x512_f16", kind="wgrad", rows=49, K=2048, C=512, dtype="f16", norm=False),
        # Expand layer of a batch-128 first stage after its norm: a small matrix summed over very many rows.
        dict(name="wgrad_401408x256x64_f16", kind="wgrad", rows=128 * 56 * 56, K=256, C=64, dtype="f16", norm=True),
        # A large square layer over a large batch of tokens: bound by the matrix cores.
        dict(name="wgrad_16384x4096x4096_bf16", kind="wgrad", rows=16384, K=4096, C=4096, dtype="bf16", norm=False),
        # One decoded token of a large vocabulary with its alternatives.
        dict(name="score_1x131072_bf16", kind="score", rows=1, V=131072, dtype="bf16", top=8),
        # Evaluation of a classifier with 1000 classes: top 5 of a batch, some classes masked.
        dict(name="score_128x1000_f16", kind="score", rows=128, V=1000, dtype="f16", top=5),
        # Loss with an entropy term and its gradient over a large odd vocabulary.
        dict(name="score_train_4096x100003_bf16", kind="score_train", rows=4096, V=100003, dtype="bf16"),
    ]


def _log(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))))


def draw(rng):
    """One more call of the same entry points: from one row to those of a
    batch of 128, widths from a narrow stage's to a large layer's, two in three
    of them multiples of 8, and no more work than the largest case listed."""
    kind = rng.choice(["norm", "norm_train", "norm_train", "pack", "act_train", "wgrad", "wgrad", "score", "score",
                       "score_train"])

    def width(lo, hi):
        w = _log(rng, lo, hi)
        return max(lo, w // 8 * 8) if rng.random() < 0.67 else w

    c = dict(kind=kind, dtype=rng.choice(["f16", "bf16"]))
    if kind in ("score", "score_train"):
        c["dtype"] = rng.choice(["f16", "bf16", "bf16", "f32"])
        c["V"] = width(10, 262144)
        c["rows"] = _log(rng, 1, max(1, min(65536, (1 << 27) // c["V"])))
        if kind == "score":
            c["top"] = rng.choice([0, 1, 5, 8, 20])
            c["top"] = min(c["top"], c["V"])
    elif kind == "wgrad":
        c.update(K=width(16, 8192), C=width(16, 8192), norm=rng.random() < 0.5)
        most = min(2.5e11 / (2.0 * c["K"] * c["C"]), 2.0e8 / (c["K"] + c["C"]))
        c["rows"] = _log(rng, 1, max(1, min(401408, int(most))))
    else:
        c["C"] = width(8, 16384)
        c["rows"] = _log(rng, 1, max(1, min(401408, (1 << 26) // c["C"])))
        if kind == "norm_train":
            c["ckpt"] = rng.random() < 0.6
        if kind == "act_train":
            c["act"] = rng.choice(["gelu", "gelu", "relu"])
    return c


# ---------------------------------------------------------------------------
# Inputs


def _gen(seed):
    return torch.Generator(device="cuda").manual_seed(seed)


def _randn(g, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=g, device="cuda") * scale).to(dtype)


def _uniform(g, shape, lo, hi):
    return torch.rand(shape, generator=g, device="cuda") * (hi - lo) + lo


def _activations(g, rows, C, dtype):
    """A residual stream: channels of different sizes (a few of them large), a
    small offset of each channel."""
    size = torch.exp(0.5 * torch.randn((C,), generator=g, device="cuda")).clamp_(max=8.0)
    offset = 0.3 * torch.randn((C,), generator=g, device="cuda")
    x = torch.randn((rows, C), generator=g, device="cuda")
    return x.mul_(size).add_(offset).to(dtype)


def _blocks(x):
    """[rows, C] padded with zeros to whole blocks: [rows, blocks, 64]."""
    n = -(-x.shape[1] // BLOCK)
    return torch.nn.functional.pad(x, (0, n * BLOCK - x.shape[1])).view(x.shape[0], n, BLOCK)


def _quantise(x):
    """(q int8 [rows, C], scale fp32 [rows, blocks]) of x in 32 bits."""
    b = _blocks(x)
    a = b.abs().amax(-1)
    ok = a >= 2.0**-119
    inv = torch.where(ok, torch.full_like(a, 127.0) / a, torch.zeros_like(a))
    scale = torch.where(ok, a * (1.0 / 127.0), torch.zeros_like(a))
    q = torch.round(b * inv[..., None]).to(torch.int8)
    return q.view(x.shape[0], -1)[:, : x.shape[1]].contiguous(), scale


def _dequantise(q, scale):
    return q.to(scale.dtype) * scale.repeat_interleave(BLOCK, 1)[:, : q.shape[1]]


def prepare(case, seed):
    g, dtype, rows = _gen(seed), DTYPES[case["dtype"]], case["rows"]
    s = dict(case=case)
    if case["kind"] in ("score", "score_train"):
        V = case["V"]
        z = _randn(g, (rows, V), torch.float32, 2.5)
        s["tokens"] = torch.randint(0, V, (rows,), generator=g, device="cuda")
        if V >= 64:  # classes that may not be chosen, by either mask in use; no row asks for one of them
            mask = torch.rand((V,), generator=g, device="cuda")
            z[:, mask < 0.03] = float("-inf")
            z[:, mask > 0.97] = torch.finfo(dtype).min
            allowed = ((mask >= 0.03) & (mask <= 0.97)).nonzero()[:, 0]
            s["tokens"] = allowed[s["tokens"] % allowed.numel()]
        s["logits"] = z.to(dtype)
        s["tokens"][torch.rand((rows,), generator=g, device="cuda") < 0.05] = -1  # padding
        if rows >= 64:
            s["logits"][rows // 2] = float("-inf")  # a row whose mask leaves nothing
        if case["kind"] == "score_train":
            s["d_logp"] = _uniform(g, (rows,), -1.5, -0.5) / rows
            s["d_entropy"] = torch.full((rows,), -0.01 / rows, device="cuda")
            if dtype == torch.float16:  # scaled loss
                s["d_logp"], s["d_entropy"] = s["d_logp"] * 4096.0, s["d_entropy"] * 4096.0
        return s
    C = case["C"]
    x = _activations(g, rows, C, dtype)
    s["weight"], s["bias"] = _uniform(g, (C,), 0.5, 1.5), 0.1 * torch.randn((C,), generator=g, device="cuda")
    if case["kind"] == "wgrad":
        xf = x.float()
        s["q"], s["scale"] = _quantise(xf)
        mean = xf.mean(1)
        s["stats"] = torch.stack([mean, torch.rsqrt((xf - mean[:, None]).square().mean(1) + EPS)], 1)
        s["dy"] = _randn(g, (rows, case["K"]), dtype, 0.02)
        return s
    s["x"] = x
    if case["kind"] in ("norm_train", "act_train"):
        s["dy"] = _randn(g, (rows, C), dtype, 0.02)
    return s


# ---------------------------------------------------------------------------
# One pass


def run(state):
    return _run_own(state) if own else _run_plain(state)


def _run_own(s):
    import paper_2404_03617_amd as cf

    case = s["case"]
    kind = case["kind"]
    if kind == "norm":
        return cf.layer_norm_forward(s["x"], s["weight"], s["bias"], eps=EPS)
    if kind == "norm_train":
        y, stats, ck = cf.layer_norm_forward_save(s["x"], s["weight"], s["bias"], eps=EPS, checkpoint=case["ckpt"])
        dx, dw, db = cf.layer_norm_backward(s["dy"], ck if case["ckpt"] else s["x"], stats, s["weight"])
        return y, dx, dw, db
    if kind == "pack":
        return cf.checkpoint_unpack(cf.checkpoint_pack(s["x"]))
    if kind == "act_train":
        h, ck, _ = cf.act_forward_save(s["x"], case["act"])
        return h, cf.act_backward(s["dy"], ck, case["act"])
    if kind == "wgrad":
        ck = cf.Checkpoint(s["q"], s["scale"], s["dy"].dtype)
        if case["norm"]:
            return cf.linear_weight_grad(s["dy"], ck, stats=s["stats"], weight=s["weight"], bias=s["bias"])
        return cf.linear_weight_grad(s["dy"], ck)
    lp = cf.log_probs_forward(s["logits"], s["tokens"], top=case.get("top", 0))
    if kind == "score":
        return (lp.logp, lp.entropy) + ((lp.top_logp, lp.top_ids) if case["top"] else ())
    return lp.logp, lp.entropy, cf.log_probs_backward(s["logits"], s["tokens"], lp, s["d_logp"], s["d_entropy"])


def _gelu_grad(u):
    return 0.5 * (1.0 + torch.erf(u * math.sqrt(0.5))) + u * torch.exp(-0.5 * u * u) / math.sqrt(2.0 * math.pi)


def _run_plain(s):
    case, kind = s["case"], s["case"]["kind"]
    if kind == "wgrad":
        dy, x = s["dy"].float(), _dequantise(s["q"], s["scale"])
        if case["norm"]:
            x = (x - s["stats"][:, :1]) * s["stats"][:, 1:] * s["weight"] + s["bias"]
        return (dy.t() @ x).to(s["dy"].dtype), dy.sum(0)
    if kind in ("score", "score_train"):
        return _score_plain(s)
    x, dtype = s["x"].float(), s["x"].dtype
    if kind == "pack":
        return _dequantise(*_quantise(x)).to(dtype)
    if kind == "act_train":
        u = _dequantise(*_quantise(x))
        if case["act"] == "relu":
            return x.clamp_min(0.0).to(dtype), (s["dy"].float() * (u > 0)).to(dtype)
        h = 0.5 * x * (1.0 + torch.erf(x * math.sqrt(0.5)))
        return h.to(dtype), (s["dy"].float() * _gelu_grad(u)).to(dtype)
    mean = x.mean(1, keepdim=True)
    rstd = torch.rsqrt((x - mean).square().mean(1, keepdim=True) + EPS)
    y = ((x - mean) * rstd * s["weight"] + s["bias"]).to(dtype)
    if kind == "norm":
        return y
    dy = s["dy"].float()
    xh = ((_dequantise(*_quantise(x)) if case["ckpt"] else x) - mean) * rstd
    gw = dy * s["weight"]
    dx = rstd * (gw - gw.mean(1, keepdim=True) - xh * (gw * xh).mean(1, keepdim=True))
    return y, dx.to(dtype), (dy * xh).sum(0), dy.sum(0)


def _score_plain(s):
    case, tokens = s["case"], s["tokens"]
    z = s["logits"].float()
    m = z.amax(1, keepdim=True)
    empty = m == float("-inf")
    d = z - torch.where(empty, torch.zeros_like(m), m)
    e = torch.exp(d)
    total = e.sum(1, keepdim=True)
    ls = torch.log(total)
    logp = torch.where(empty, d, d - ls)
    p = torch.where(empty, torch.zeros_like(e), e / total)
    plogp = torch.where(p > 0, p * logp, torch.zeros_like(p))
    entropy = -plogp.sum(1)
    given = tokens >= 0
    lp = torch.where(given, logp.gather(1, tokens.clamp_min(0)[:, None])[:, 0], torch.zeros_like(entropy))
    if case["kind"] == "score":
        if not case["top"]:
            return lp, entropy
        # one whole number a class, larger for larger logits and, among equal ones, for lower ids
        bits = (z + 0.0).view(torch.int32).long()
        order = torch.where(bits >= 0, bits, -(bits & 0x7FFFFFFF) - 1)
        key = (order << 32) | (0xFFFFFFFF - torch.arange(z.shape[1], device=z.device))
        ids = 0xFFFFFFFF - (key.topk(case["top"], dim=1).values & 0xFFFFFFFF)
        return lp, entropy, logp.gather(1, ids), ids
    glp = torch.where(given & ~empty[:, 0], s["d_logp"], torch.zeros_like(entropy))[:, None]
    gh = s["d_entropy"][:, None]
    dz = -glp * p - gh * (plogp + p * entropy[:, None])
    dz.scatter_add_(1, tokens.clamp_min(0)[:, None], glp)
    return lp, entropy, dz.to(s["logits"].dtype)


# ---------------------------------------------------------------------------
# What a pass cannot do without


def work(case):
    """Each input read once and each output written once; a checkpoint is
    written by the forward call and read by the backward call."""
    R, kind = case["rows"], case["kind"]
    if kind in ("score", "score_train"):
        n, b = R * case["V"], 4 if case["dtype"] == "f32" else 2
        if kind == "score":
            return {"bytes": n * b + R * (16 + 12 * case["top"]), "flops": 5 * n}
        return {"bytes": n * 3 * b + R * 24, "flops": 10 * n}
    n, C = R * case["C"], case["C"]
    ckpt = n + 4 * R * -(-C // BLOCK)
    if kind == "norm":
        return {"bytes": 4 * n + 8 * C, "flops": 8 * n}
    if kind == "norm_train":
        return {"bytes": 8 * n + (2 * ckpt if case["ckpt"] else 2 * n) + 16 * R + 16 * C, "flops": 22 * n}
    if kind == "pack":
        return {"bytes": 4 * n + 2 * ckpt, "flops": 5 * n}
    if kind == "act_train":
        return {"bytes": 8 * n + 2 * ckpt, "flops": 40 * n if case["act"] == "gelu" else 8 * n}
    K = case["K"]
    return {"bytes": 2 * R * K + ckpt + 2 * K * C + 4 * K + (8 * R + 8 * C if case["norm"] else 0),
            "flops": 2.0 * R * K * C}


# ---------------------------------------------------------------------------
# The definitions in 64 bits


def exact(case, seed):
    s = prepare(case, seed)
    kind, R = case["kind"], case["rows"]
    f = torch.float64
    if kind == "wgrad":
        dw = torch.zeros((case["K"], case["C"]), dtype=f, device="cuda")
        db = torch.zeros((case["K"],), dtype=f, device="cuda")
        for a in range(0, R, 16384):  # some rows at a time: 64-bit copies are large
            at = slice(a, a + 16384)
            x = _dequantise(s["q"][at], s["scale"][at].to(f))
            if case["norm"]:
                mean, rstd = s["stats"][at].to(f).unbind(1)
                x = torch.addcmul(s["bias"].to(f), (x - mean[:, None]) * rstd[:, None], s["weight"].to(f))
            dy = s["dy"][at].to(f)
            dw += torch.mm(dy.t().contiguous(), x)
            db += dy.sum(0)
        return dw, db
    if kind in ("score", "score_train"):
        return _exact_score(case, s)
    out, dw, db = [], 0.0, 0.0
    step = max(1, (1 << 24) // case["C"])
    for a in range(0, R, step):
        x16 = s["x"][a:a + step]
        x = x16.to(f)
        back = _dequantise(*_quantise(x16.float())).to(f) if kind != "norm" and case.get("ckpt", True) else x
        if kind == "pack":
            q, scale = _quantise(x16.float())
            out.append((_dequantise(q, scale.to(f)),))
            continue
        if kind == "act_train":
            dh = s["dy"][a:a + step].to(f)
            if case["act"] == "relu":
                out.append((torch.relu(x), torch.where(back > 0, dh, torch.zeros_like(dh))))
            else:
                pdf = torch.exp(-back.square() / 2) / math.sqrt(2 * math.pi)
                out.append((x * torch.special.ndtr(x), dh * (torch.special.ndtr(back) + back * pdf)))
            continue
        var, mean = torch.var_mean(x, 1, correction=0, keepdim=True)
        sd = torch.sqrt(var + EPS)
        w = s["weight"].to(f)
        y = w * (x - mean) / sd + s["bias"].to(f)
        if kind == "norm":
            out.append((y,))
            continue
        dy, n = s["dy"][a:a + step].to(f), case["C"]
        xh = (back - mean) / sd
        dxh = dy * w
        out.append((y, (n * dxh - dxh.sum(1, keepdim=True) - xh * (dxh * xh).sum(1, keepdim=True)) / (n * sd)))
        dw, db = dw + (dy * xh).sum(0), db + dy.sum(0)
    parts = [torch.cat(p) for p in zip(*out)]
    if kind in ("norm", "pack"):
        return parts[0]
    return tuple(parts) + ((dw, db) if kind == "norm_train" else ())


def _exact_score(case, s):
    f, out = torch.float64, []
    step = max(1, (1 << 25) // case["V"])
    for a in range(0, case["rows"], step):
        z, t = s["logits"][a:a + step].to(f), s["tokens"][a:a + step]
        some = (z > float("-inf")).any(1, keepdim=True)
        lse = torch.logsumexp(z, 1, keepdim=True)
        logp = torch.where(some, z - lse, z)
        p = torch.where(some, torch.softmax(z, 1), torch.zeros_like(z))
        entropy = torch.special.entr(p).sum(1, keepdim=True)
        at = t.clamp_min(0)[:, None]
        picked = torch.where(t[:, None] >= 0, logp.gather(1, at), torch.zeros_like(lse))[:, 0]
        if case["kind"] == "score":
            top = torch.sort(logp, 1, descending=True).values[:, : case["top"]]
            out.append((picked, entropy[:, 0]) + ((top,) if case["top"] else ()))
            continue
        one = torch.zeros_like(z).scatter_(1, at, 1.0) * ((t[:, None] >= 0) & some)
        glp = s["d_logp"][a:a + step].to(f)[:, None] * ((t[:, None] >= 0) & some)
        gh = s["d_entropy"][a:a + step].to(f)[:, None]
        slope = torch.where(p > 0, logp + entropy, torch.zeros_like(p))
        out.append((picked, entropy[:, 0], glp * (one - p) - gh * p * slope))
    parts = tuple(torch.cat(p) for p in zip(*out))
    return parts + ((None,) if case["kind"] == "score" and case["top"] else ())
