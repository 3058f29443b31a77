"""Cluster, train, cluster again, with a layer of experts: inputs of different kinds go through different weights.

As train_encoder.py, but the encoder's hidden layer is a layer of experts.  A router sends each row to k of them, by sigmoid scores and
a bias that is moved after each step so that all experts get rows; an expert is two products in bfloat16 with gated units
between them, whose inputs are kept in 8 bits for the backward pass.  Everything but the router's and the head's products is
this package's.

    python examples/train_experts.py
"""
from __future__ import annotations

import os
import sys

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
if ROOT not in sys.path:
    sys.path.insert(0, ROOT)

import torch

import paper_2609_36074_b200 as gem
import synth
from train_encoder import cluster

HALF = torch.bfloat16


class Encoder:
    """x -> layer norm -> x + experts -> layer norm: the features.  Weights in float32, gradients beside them; the experts' products
    run on bfloat16 copies."""

    def __init__(self, d: int, d_hidden: int, experts: int, k: int, clusters: int, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)

        def normal(*shape):
            return torch.randn(*shape, generator=gen, device="cuda") / shape[-2] ** 0.5

        ones, zeros = (lambda n: torch.ones(n, device="cuda")), (lambda n: torch.zeros(n, device="cuda"))
        self.k, self.bias = k, zeros(experts)
        self.p = {
            "norm1.w": ones(d), "norm1.b": zeros(d), "router": normal(d, experts),
            "up": normal(experts, d, 2 * d_hidden), "down": normal(experts, d_hidden, d),
            "norm2.w": ones(d), "norm2.b": zeros(d), "head": normal(d, clusters),
        }

    def features(self, x):
        """The features and what the backward pass needs."""
        p = self.p
        a, mean1, rstd1 = gem.layer_norm(x, p["norm1.w"], p["norm1.b"])
        logits = a @ p["router"]
        r = gem.route(logits, self.k, "sigmoid", bias=self.bias)
        a16, up, down = a.to(HALF), p["up"].to(HALF), p["down"].to(HALF)
        h, units = gem.activation(gem.expert_product(a16, up, r.offset, r.row), "silu", gated=True)
        y = gem.expert_product(h, down, r.offset)
        s = a + gem.combine(y, r.place, r.weight)
        f, mean2, rstd2 = gem.layer_norm(s, p["norm2.w"], p["norm2.b"])
        return f, (x, mean1, rstd1, a, logits, r, a16, up, down, units, y, s, mean2, rstd2)

    def gradients(self, x, labels):
        """(loss, gradients by name, rows by expert) of the mean cross entropy on the labels."""
        p = self.p
        f, (x, mean1, rstd1, a, logits, r, a16, up, down, units, y, s, mean2, rstd2) = self.features(x)
        z = f @ p["head"]
        loss, _, dz = gem.label_cross_entropy(z, labels, dlogits=z)                      # written over the logits
        g = {"head": f.t() @ dz}
        ds, g["norm2.w"], g["norm2.b"] = gem.layer_norm_backward(dz @ p["head"].t(), s, mean2, rstd2, p["norm2.w"])
        dy, dweight = gem.combine_backward(ds.to(HALF), y, r.place, r.weight, r.offset)
        h = gem.activation_backward(None, units, "silu", gated=True, need_y=True)[1]     # again, from the 8 bits
        dh, g["down"] = gem.expert_product_backward(dy, h, down, r.offset)
        du, _ = gem.activation_backward(dh, units, "silu", gated=True)
        dplace, g["up"] = gem.expert_product_backward(du, a16, up, r.offset, r.row)
        dlogits = gem.route_backward(dweight, logits, r.expert, "sigmoid")
        g["router"] = a.t() @ dlogits
        da = ds + gem.combine(dplace, r.place) + dlogits @ p["router"].t()
        _, g["norm1.w"], g["norm1.b"] = gem.layer_norm_backward(da, x, mean1, rstd1, p["norm1.w"], need_dx=False)
        return loss, g, r.offset[1:] - r.offset[:-1]

    def step(self, x, labels, rate: float, max_norm: float, balance: float = 0.01):
        loss, g, rows = self.gradients(x, labels)
        names = sorted(g)
        out = [torch.empty_like(self.p[n]) for n in names]                               # clipped, in float32
        norm = gem.clip_grad_norm([g[n] for n in names], max_norm, out=out)
        for n, v in zip(names, out):
            self.p[n].sub_(v, alpha=rate)
        rows = rows.float()
        self.bias.add_(torch.sign(rows.mean() - rows), alpha=balance)
        return loss, norm


def main(rounds: int = 2, steps: int = 30, n: int = 8192, d: int = 64, clusters: int = 16, experts: int = 8, k: int = 2, batch: int = 2048, seed: int = 0):
    """Returns the mean loss of each round's first and last four steps."""
    data, _, _ = synth.make_mixture(synth.MixtureSpec("example", n, d, clusters, "equal", 9.0, "unit", 1, seed))
    x = torch.from_numpy(data).cuda()
    enc = Encoder(d, 96, experts, k, clusters, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for r in range(rounds):
        labels = cluster(enc.features(x)[0], clusters)
        losses, norm = [], None
        for _ in range(steps):
            pick = torch.randint(0, n, (batch,), generator=gen, device="cuda")
            loss, norm = enc.step(x[pick], labels[pick], rate=0.5, max_norm=1.0)
            losses.append(loss)
        losses = torch.stack(losses).cpu()
        out.append((losses[:4].mean().item(), losses[-4:].mean().item()))
        print(f"round {r}: {labels.unique().numel()} clusters, loss {out[-1][0]:.4f} -> {out[-1][1]:.4f}, last gradient norm {norm.item():.4f}")
    return out


if __name__ == "__main__":
    main()
