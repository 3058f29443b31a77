"""The training operators together, as the example uses them: one step's gradients against 64-bit autograd, and a run."""
import os
import sys

import pytest
import torch

import paper_2609_36074_b200 as gem

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu


def test_gradients_of_a_step_against_autograd():
    import train_encoder as ex
    torch.backends.cuda.matmul.allow_tf32 = False
    enc = ex.Encoder(40, 56, 11, seed=3)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(300, 40, generator=gen, device="cuda") * 2 + 0.5
    labels = torch.randint(-1, 11, (300,), generator=gen, device="cuda", dtype=torch.int32)
    loss, g = enc.gradients(x, labels)
    p = {n: w.double().requires_grad_(True) for n, w in enc.p.items()}

    def norm(v, w, b):
        c = v - v.mean(1, keepdim=True)
        return c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * w + b

    h = torch.tanh(norm(x.double(), p["norm1.w"], p["norm1.b"]) @ p["hidden"])
    logp = torch.log_softmax(norm(h, p["norm2.w"], p["norm2.b"]) @ p["head"], 1)
    kept = labels >= 0
    want = -logp[kept].gather(1, labels[kept].long()[:, None]).mean()
    want.backward()
    # products of 40 to 300 terms in 32 bits between the operators: some hundred roundings of 2^-24 each way
    assert abs(loss.item() - want.item()) <= 1e-5
    for n in g:
        assert (g[n].double() - p[n].grad).norm() <= 2e-5 * p[n].grad.norm(), n
    want = torch.cat([v.grad.reshape(-1) for v in p.values()]).norm()
    got = gem.clip_grad_norm([g[n] for n in sorted(g)], 0.1)
    assert abs(got.item() - want.item()) <= 2e-5 * want.item()
    total = torch.cat([v.reshape(-1) for v in g.values()]).double().norm()
    assert abs(total.item() - 0.1) <= 1e-5


def test_rounds_of_clustering_and_training():
    import train_encoder as ex
    for first, last in ex.main(rounds=2, steps=30, n=4096, batch=1024):
        assert last < 0.7 * first
