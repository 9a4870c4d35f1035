"""The example's training step: its gradients against autograd in 64 bits on
the same head, and a loss that falls."""
import importlib.util
import os

import pytest
import torch

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def example():
    spec = importlib.util.spec_from_file_location("finetune_head", os.path.join(ROOT, "examples", "finetune_head.py"))
    m = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(m)
    return m


@pytest.mark.parametrize("dtype", [torch.float16, torch.bfloat16])
def test_gradients_of_a_step(dtype):
    """Checkpoints keep 8 bits (1/254 of a block's largest value), activations
    and their gradients are rounded to 16 bits at each of five layers, so the
    gradients agree with those of the exact head to some 2 percent in norm."""
    m = example()
    head = m.Head(64, 256, 10, dtype, seed=1)
    head.p["lw"] += 0.2 * torch.randn(64, device="cuda", generator=torch.Generator("cuda").manual_seed(5))
    g = torch.Generator().manual_seed(2)
    x = torch.randn(4, 5, 6, 64, generator=g).to(dtype).cuda()
    labels = torch.randint(-1, 10, (4, 5, 6), generator=g).cuda()
    loss, grads, dx = head.step(x, labels, scale=256.0)
    q = {k: v.double().cpu().requires_grad_() for k, v in head.p.items()}
    xd = x.double().cpu().reshape(-1, 64).requires_grad_()
    t = labels.cpu().reshape(-1)
    y = torch.nn.functional.layer_norm(xd, (64,), q["lw"], q["lb"], 1e-6)
    h = torch.nn.functional.gelu(y @ q["w1"].t() + q["b1"])
    want = torch.nn.functional.cross_entropy(h @ q["w2"].t() + q["b2"], t, ignore_index=-1)
    want.backward()
    assert abs(float(loss) - want.item()) <= 0.02 * want.item()
    for k, v in list(grads.items()) + [("x", dx)]:
        ref = xd.grad if k == "x" else q[k].grad
        off = float((v.double().cpu() / 256.0 - ref).norm() / ref.norm())
        print("  d%s: %.2e of the gradient's norm" % (k, off), flush=True)
        assert off <= 0.02, k


def test_the_loss_falls(monkeypatch, capsys):
    m = example()
    monkeypatch.setattr("sys.argv", ["finetune_head.py", "--steps", "21", "--batch", "8"])
    m.main()
    losses = [float(line.split("loss ")[1].split(";")[0]) for line in capsys.readouterr().out.splitlines()]
    assert len(losses) == 3 and losses[-1] < 0.8 * losses[0], losses


def test_evaluation_leaves_out_rows_without_a_label():
    m = example()
    g = torch.Generator().manual_seed(3)
    z = (2.0 * torch.randn(6, 9, 40, generator=g)).half().cuda()
    labels = torch.randint(0, 40, (6, 9), generator=g)
    labels[0, 0] = z[0, 0].argmax().cpu()
    none = torch.rand(6, 9, generator=g) < 0.4
    none[0, 0] = False
    padded = torch.where(none, -1 - labels, labels).cuda()
    want = m.evaluate(z[~none.cuda()], labels[~none].cuda())
    got = m.evaluate(z, padded)
    assert float(want[2]) > 0
    for a, b in zip(got, want):  # the same rows in another order of adding
        assert abs(float(a) - float(b)) <= 1e-5 * abs(float(b)), (got, want)
    nothing = m.evaluate(z, torch.full_like(padded, -1))
    assert all(float(v) == 0.0 for v in nothing)
