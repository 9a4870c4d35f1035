"""Inputs and references in 64 bits for the tests of the row operators."""
import numpy as np
import torch

DT = {"f16": torch.float16, "bf16": torch.bfloat16, "f32": torch.float32}
ROUND = {torch.float16: 2.0**-11, torch.bfloat16: 2.0**-8, torch.float32: 2.0**-24}  # of one rounding to nearest
TINY = {torch.float16: 2.0**-25, torch.bfloat16: 2.0**-133, torch.float32: 2.0**-149}  # below the normal range
F32 = 2.0**-24


def randn(seed, shape, dtype=torch.float32, scale=1.0):
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(shape, generator=g) * scale).to(dtype)


def rows_in(kind, x):
    """x [rows, C] on the GPU as a contiguous tensor, as columns of a wider one
    (from an odd element on), or shifted by one element."""
    rows, C = x.shape
    if kind == "dense":
        return x.cuda()
    if kind == "slice":
        wide = torch.full((rows, C + 11), float("nan"), dtype=x.dtype, device="cuda")
        wide[:, 3:3 + C] = x.cuda()
        return wide[:, 3:3 + C]
    flat = torch.full((rows * C + 1,), float("nan"), dtype=x.dtype, device="cuda")
    flat[1:] = x.cuda().reshape(-1)
    return flat[1:].view(rows, C)


def guarded(rows, C, dtype, pad=5):
    """An output as columns of a wider buffer of sevens, and the buffer."""
    wide = torch.full((rows + 1, C + pad), 7.0, dtype=dtype, device="cuda")
    return wide[:rows, 2:2 + C], wide


def outside_untouched(wide, C):
    w = wide.clone()
    w[:-1, 2:2 + C] = 7.0
    return bool((w == 7.0).all())


def quantise(x):
    """(q, scale) of x [rows, C] by the format's definition: one float32
    rounding an operation (numpy)."""
    v = x.float().numpy()
    rows, C = v.shape
    n = -(-C // 64)
    b = np.zeros((rows, n * 64), np.float32)
    b[:, :C] = v
    b = b.reshape(rows, n, 64)
    a = np.abs(b).max(-1)
    fine = np.isfinite(b).all(-1)
    ok = fine & (a >= np.float32(2.0**-119))
    safe = np.where(ok, a, np.float32(1.0))
    inv = np.where(ok, np.float32(127.0) / safe, np.float32(0.0)).astype(np.float32)
    scale = np.where(ok, a * np.float32(np.float32(1.0) / np.float32(127.0)), np.float32(0.0)).astype(np.float32)
    scale[~fine] = np.nan
    with np.errstate(invalid="ignore"):
        q = np.rint(np.where(ok[..., None], b, np.float32(0.0)) * inv[..., None]).astype(np.int8)
    return torch.from_numpy(q.reshape(rows, -1)[:, :C].copy()), torch.from_numpy(scale), torch.from_numpy(fine)


def dequantise(q, scale):
    """Values in 64 bits."""
    return q.double() * scale.double().repeat_interleave(64, 1)[:, : q.shape[1]]


def assert_within(got, ref, tol, what):
    """|got - ref| <= tol, elementwise, with the same NaNs and infinities."""
    got, ref, tol = got.detach().cpu().double(), ref.double(), torch.as_tensor(tol, dtype=torch.float64)
    assert got.shape == ref.shape, (what, got.shape, ref.shape)
    fine = torch.isfinite(ref)
    assert torch.equal(torch.isnan(got), torch.isnan(ref)), what + ": NaN in other places"
    inf = torch.isinf(ref)
    assert torch.equal(got[inf], ref[inf]), what + ": other infinities"
    assert bool(torch.isfinite(got[fine]).all()), what + ": not finite"
    over = ((got - ref).abs() / tol.expand_as(ref).clamp_min(1e-300))[fine]
    worst = float(over.max()) if over.numel() else 0.0
    print("  %s: worst error %.3g of the tolerance" % (what, worst), flush=True)
    assert worst <= 1.0, "%s: %.3g times the tolerance" % (what, worst)
