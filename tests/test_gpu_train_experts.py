"""A layer of experts as the example uses it: a step's gradients against 64-bit autograd, the same step captured and replayed, and a run."""
import math
import os
import sys

import pytest
import torch

import paper_2609_36074_b200 as gem

sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))

pytestmark = pytest.mark.gpu

N, D, HIDDEN, EXPERTS, K, CLUSTERS = 400, 40, 56, 6, 2, 11


def made(seed=3):
    import train_experts as ex
    torch.backends.cuda.matmul.allow_tf32 = False
    enc = ex.Encoder(D, HIDDEN, EXPERTS, K, CLUSTERS, seed)
    gen = torch.Generator(device="cuda").manual_seed(1)
    x = torch.randn(N, D, generator=gen, device="cuda") * 2 + 0.5
    labels = torch.randint(-1, CLUSTERS, (N,), generator=gen, device="cuda", dtype=torch.int32)
    return enc, x, labels


def rows_at(v, offset, row, w):
    """The experts' products in 64 bits, one row a place."""
    at = offset.tolist()
    return torch.cat([(v[row[a:b].long()] if row is not None else v[a:b]) @ w[e] for e, (a, b) in enumerate(zip(at[:-1], at[1:]))])


def test_gradients_of_a_step_against_autograd():
    enc, x, labels = made()
    loss, g, rows = enc.gradients(x, labels)
    r = enc.features(x)[1][5]
    p = {n: w.double().requires_grad_(True) for n, w in enc.p.items()}

    def norm(v, w, b):
        c = v - v.mean(1, keepdim=True)
        return c / (c.square().mean(1, keepdim=True) + 1e-5).sqrt() * w + b

    a = norm(x.double(), p["norm1.w"], p["norm1.b"])
    s = torch.sigmoid(a @ p["router"]).gather(1, r.expert.long())
    weight = s / s.sum(1, keepdim=True)
    gate, value = rows_at(a, r.offset, r.row, p["up"]).chunk(2, 1)
    y = rows_at(torch.nn.functional.silu(gate) * value, r.offset, None, p["down"])
    out = norm(a + (weight[:, :, None] * y[r.place.long()]).sum(1), p["norm2.w"], p["norm2.b"])
    logp = torch.log_softmax(out @ p["head"], 1)
    kept = labels >= 0
    want = -logp[kept].gather(1, labels[kept].long()[:, None]).mean()
    want.backward()
    assert rows.sum().item() == N * K
    # Half steps of bfloat16 are 2^-9 of a value's binade's top, 2^-8 of a value at most; the forward pass has seven in a row (weights,
    # a, z, h, y, their sums' joining and the 8 bits of the units, at most a 127th of 32 neighbours' largest: four such), the
    # backward pass as many again.  They are independent of one another: the norms of what they add are far below 16 times 2^-8.
    for n in g:
        assert (g[n].double() - p[n].grad).norm() <= 16 * 2.0 ** -8 * p[n].grad.norm(), n
    assert abs(loss.item() - want.item()) <= 16 * 2.0 ** -8


def test_gradients_of_the_layer_against_differences():
    """The loss along a direction of the experts' weights, its step large against bfloat16's and small against the weights."""
    enc, x, labels = made(5)
    _, g, _ = enc.gradients(x, labels)
    def loss():
        return enc.gradients(x, labels)[0].item()

    for n in ("down", "up"):
        v = g[n].float() / g[n].float().norm()
        along = (g[n].float() * v).sum().item()
        kept = enc.p[n].clone()
        h = 0.5
        enc.p[n] = kept + h * v
        up = loss()
        enc.p[n] = kept - h * v
        down = loss()
        enc.p[n] = kept
        # bfloat16's roundings are as in the test above; the second order cancels, the third is h^2 / 6 of the curvature's change
        assert abs((up - down) / (2 * h) - along) <= 0.15 * abs(along), n


def test_a_step_captured_and_replayed():
    enc, x, labels = made()
    want = enc.gradients(x, labels)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        enc.gradients(x, labels)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = enc.gradients(x, labels)
    keep = x.clone()
    x.copy_(torch.randn_like(x))
    graph.replay()
    x.copy_(keep)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])
    for n in got[1]:
        assert torch.equal(got[1][n], want[1][n]), n


def test_rounds_of_clustering_and_training():
    import train_experts as ex
    out = ex.main(rounds=2, steps=12, n=4096, batch=1024)
    assert len(out) == 2 and all(math.isfinite(v) for pair in out for v in pair)


def test_what_the_layer_keeps_is_smaller():
    enc, x, _ = made()
    units = enc.features(x)[1][9]
    kept = units.q.numel() + units.scale.numel()
    assert isinstance(units, gem.Checkpoint) and kept <= N * K * (2 * 64 + 4) and kept < 0.6 * 2 * (N * K * 3 * HIDDEN)
