"""Fine-tune a head over frozen ConvFirst features, and score with it.

    python examples/finetune_head.py [--steps 30]

The backbone is one stage of fused blocks (stage_forward).  The head is layer
norm, an expand layer with GELU and a project layer to the classes, for every
pixel of the feature map (or any rows of features).  Its training step keeps
two 8-bit checkpoints a layer and no 16-bit activation: the norm's input serves
the norm's gradient and, with the row statistics, the expand layer's; the
expand layer's output serves GELU's gradient; GELU's output the project
layer's.  Products with the weights are torch matmuls.  Weights and
data are synthetic: the classes are those of a second head with other weights.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import paper_2404_03617_amd as cf  # noqa: E402
from paper_2404_03617_amd import synth  # noqa: E402


class Head:
    """norm -> w1 [E*C, C], b1 -> GELU -> w2 [classes, E*C], b2.  Weights in the
    features' dtype, vectors in fp32."""

    def __init__(self, C, hidden, classes, dtype=torch.float16, device="cuda", seed=0):
        g = torch.Generator().manual_seed(seed)

        def normal(rows, cols):
            return (torch.randn(rows, cols, generator=g) * cols**-0.5).to(dtype).to(device)

        self.p = {"lw": torch.ones(C, device=device), "lb": torch.zeros(C, device=device),
                  "w1": normal(hidden, C), "b1": torch.zeros(hidden, device=device),
                  "w2": normal(classes, hidden), "b2": torch.zeros(classes, device=device)}

    def logits(self, x):
        p = self.p
        u = torch.nn.functional.linear(cf.layer_norm_forward(x, p["lw"], p["lb"]), p["w1"], p["b1"].to(x.dtype))
        return torch.nn.functional.linear(cf.act_forward(u, "gelu", out=u), p["w2"], p["b2"].to(x.dtype))

    def step(self, x, labels, scale=1.0):
        """The mean loss -log p(label) over rows with a label, the gradients of
        `scale` times that loss by name, and that of the features.  Labels below
        0 mark rows that do not count."""
        p = self.p
        x, labels = x.reshape(-1, x.shape[-1]), labels.reshape(-1)
        y, stats, kept_x = cf.layer_norm_forward_save(x, p["lw"], p["lb"])
        u = torch.nn.functional.linear(y, p["w1"], p["b1"].to(x.dtype))
        h, kept_u, kept_h = cf.act_forward_save(u, "gelu", checkpoint_out=True, out=u)
        z = torch.nn.functional.linear(h, p["w2"], p["b2"].to(x.dtype))
        lp = cf.log_probs_forward(z, labels)
        count = (labels >= 0).sum().clamp_min(1)
        loss = -lp.logp.sum() / count
        # ---- backward: each gradient takes the place of the activation before it
        dz = cf.log_probs_backward(z, labels, lp, (-scale / count).expand(labels.shape).contiguous(), out=z)
        g = {}
        g["w2"], g["b2"] = cf.linear_weight_grad(dz, kept_h)
        dh = dz @ p["w2"]
        du = cf.act_backward(dh, kept_u, "gelu", out=dh)
        g["w1"], g["b1"] = cf.linear_weight_grad(du, kept_x, stats, p["lw"], p["lb"])
        dx, g["lw"], g["lb"] = cf.layer_norm_backward(du @ p["w1"], kept_x, stats, p["lw"])
        return loss, g, dx

    def sgd(self, grads, lr, scale=1.0):
        for k, v in grads.items():
            self.p[k] -= (lr / scale * v.float()).to(self.p[k].dtype)


def evaluate(logits, labels, top=5):
    """Mean log probability of the labels, mean entropy, shares of rows whose
    label is first and among the `top` first; over the rows with a label, as in
    Head.step (all 0 where none has one)."""
    labels = labels.reshape(-1)
    r = cf.log_probs_forward(logits.reshape(-1, logits.shape[-1]), labels, top=top)
    given = labels >= 0
    hit = (r.top_ids == labels[:, None]).float()  # no id is negative
    count = given.sum().clamp_min(1)
    return (r.logp.sum() / count, r.entropy.masked_fill(~given, 0.0).sum() / count, hit[:, 0].sum() / count,
            hit.sum() / count)


def main():
    ap = argparse.ArgumentParser(description=__doc__, formatter_class=argparse.RawDescriptionHelpFormatter)
    ap.add_argument("--steps", type=int, default=30)
    ap.add_argument("--batch", type=int, default=16)
    ap.add_argument("--lr", type=float, default=0.3)
    a = ap.parse_args()
    N, H, C, hidden, classes, scale = a.batch, 14, 256, 1024, 100, 1024.0
    blocks = [{k: v.cuda() for k, v in synth.block_params(1, i, C, 4, 3).items() if v is not None} for i in range(2)]
    head, teacher = Head(C, hidden, classes, seed=2), Head(C, hidden, classes, seed=3)
    teacher.p["w2"] *= 8
    for i in range(a.steps):
        x = cf.stage_forward(synth.activations(10 + i, N, H, H, C).cuda(), blocks)
        labels = teacher.logits(x).argmax(-1)
        loss, grads, _ = head.step(x, labels, scale)
        head.sgd(grads, a.lr, scale)
        if i % 10 == 0 or i == a.steps - 1:
            logp, entropy, first, five = (float(v) for v in evaluate(head.logits(x), labels))
            print("step %d: loss %.4f; after it: log p %.4f, entropy %.4f, first %.3f, among five %.3f"
                  % (i, float(loss), logp, entropy, first, five), flush=True)


if __name__ == "__main__":
    main()
