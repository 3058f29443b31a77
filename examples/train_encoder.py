"""Cluster, train, cluster again: an encoder that learns the clusters of its own features.

Each round clusters the encoder's features with the NLR iteration, reads one label a row out, and trains the encoder and a
linear head on those labels.  The matrix products are torch's; everything between them is this package's: layer norm and its
gradient, cross entropy on the int32 labels with its gradient, and the norm of all gradients with clipping.

    python examples/train_encoder.py
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


class Encoder:
    """x -> layer norm -> product -> tanh -> layer norm: the features.  Weights in float32, gradients beside them."""

    def __init__(self, d_in: int, d_hidden: int, k: int, seed: int = 0):
        gen = torch.Generator(device="cuda").manual_seed(seed)
        ones, zeros = (lambda n: torch.ones(n, device="cuda")), (lambda n: torch.zeros(n, device="cuda"))
        self.p = {
            "norm1.w": ones(d_in), "norm1.b": zeros(d_in),
            "hidden": torch.randn(d_in, d_hidden, generator=gen, device="cuda") / d_in ** 0.5,
            "norm2.w": ones(d_hidden), "norm2.b": zeros(d_hidden),
            "head": torch.randn(d_hidden, k, generator=gen, device="cuda") / d_hidden ** 0.5,
        }

    def features(self, x):
        """The features and what the backward pass needs."""
        p = self.p
        a, mean1, rstd1 = gem.layer_norm(x, p["norm1.w"], p["norm1.b"])
        h = torch.tanh(a @ p["hidden"])
        f, mean2, rstd2 = gem.layer_norm(h, p["norm2.w"], p["norm2.b"])
        return f, (x, mean1, rstd1, a, h, mean2, rstd2)

    def gradients(self, x, labels):
        """(loss, gradients by name) of the mean cross entropy on the labels."""
        p = self.p
        f, (x, mean1, rstd1, a, h, mean2, rstd2) = self.features(x)
        logits = f @ p["head"]
        loss, _, dlogits = gem.label_cross_entropy(logits, labels, dlogits=logits)       # written over the logits
        g = {"head": f.t() @ dlogits}
        dh, g["norm2.w"], g["norm2.b"] = gem.layer_norm_backward(dlogits @ p["head"].t(), h, mean2, rstd2, p["norm2.w"])
        dz = dh * (1.0 - h * h)
        g["hidden"] = a.t() @ dz
        _, g["norm1.w"], g["norm1.b"] = gem.layer_norm_backward(dz @ p["hidden"].t(), x, mean1, rstd1, p["norm1.w"], need_dx=False)
        return loss, g

    def step(self, x, labels, rate: float, max_norm: float):
        loss, g = self.gradients(x, labels)
        names = sorted(g)
        norm = gem.clip_grad_norm([g[n] for n in names], max_norm)
        for n in names:
            self.p[n].sub_(g[n], alpha=rate)
        return loss, norm


def cluster(features, k: int, iterations: int = 400):
    """One int32 label a row: the row argmax of the NLR factor, from the data-informed start."""
    hp = synth.default_hparams(k)
    gen = torch.Generator(device="cuda").manual_seed(0)
    u = torch.randn(features.shape[0], k, generator=gen, device="cuda")
    solver = gem.GemNlr(features.contiguous(), u, k, alpha=hp["alpha"], beta=hp["beta"], eps_d=hp["eps_d"], eps_c=hp["eps_c"],
                        T=iterations, T_min=hp["T_min"], x_inplace=0)
    solver.spectral_norm()
    if solver.init_range() != gem.OK:
        raise RuntimeError("the features have too low a rank for this start")
    solver.run()
    labels = solver.labels()
    torch.cuda.synchronize()
    solver.destroy()
    return labels


def main(rounds: int = 2, steps: int = 30, n: int = 8192, d: int = 64, k: int = 16, batch: int = 2048, seed: int = 0):
    """Returns the mean loss of each round's first and last epoch-like stretch of four steps."""
    data, _, _ = synth.make_mixture(synth.MixtureSpec("example", n, d, k, "equal", 9.0, "unit", 1, seed))
    x = torch.from_numpy(data).cuda()
    enc = Encoder(d, 96, k, seed)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = []
    for r in range(rounds):
        labels = cluster(enc.features(x)[0], k)
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
