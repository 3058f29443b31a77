"""Rows so wide that one block goes through them term by term.

Terms that are alike round the same way, one after the other: a 32-bit sum of 2^17 of them is off by parts in a thousand.  Here
a 32-bit sum takes at most 64 terms before it goes on in 64 bits; with the roundings of the
terms themselves 128 u is a bound on every sum's relative error (u = 2^-24, terms of one sign)."""
import math

import pytest
import torch

import paper_2609_36074_b200 as gem

pytestmark = pytest.mark.gpu

U = 2.0 ** -24
WIDE = (1 << 25) + 3


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=lambda t: str(t)[6:])
def test_mean_and_variance(dtype):
    x = torch.empty(2, WIDE, dtype=dtype, device="cuda")
    x[0], x[1] = 3.3, -0.7
    x[1, ::2] = 1.3
    y, mean, rstd = gem.layer_norm(x, eps=1e-2)
    v = x.double()
    want = v.mean(1)
    var = (v - want[:, None]).square().mean(1)
    size = v.abs().mean(1)
    assert ((mean.double() - want).abs() <= 128 * U * size).all()
    # the squares about a mean that is off by e add e^2 and e times the terms' own sum about it (0)
    rst = 1.0 / (var + 1e-2).sqrt()
    assert ((rstd.double() - rst).abs() <= (128 * U + (128 * U * size).square() / 1e-2 + 8 * U) * rst).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=lambda t: str(t)[6:])
def test_gradient(dtype):
    gen = torch.Generator(device="cuda").manual_seed(0)
    x = torch.randn(1, WIDE, generator=gen, device="cuda").to(dtype)
    dy = torch.full((1, WIDE), 0.3, device="cuda").to(dtype)
    _, mean, rstd = gem.layer_norm(x)
    dx = gem.layer_norm_backward(dy, x, mean, rstd)[0].double()
    g, r = dy.double(), rstd.double()[:, None]
    h = (x.double() - mean.double()[:, None]) * r
    c1, c2 = g.mean(), (g * h).mean()
    want = r * (g - c1 - h * c2)
    e = 128 * U * (g.abs().mean() + h.abs() * (g * h).abs().mean()) + 8 * U * (g.abs() + c1.abs() + (h * c2).abs())
    step = 2.0 ** -8 if dtype is torch.bfloat16 else U
    assert ((dx - want).abs() <= r * e + step * want.abs() * 1.01 + 1e-38).all()


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16], ids=lambda t: str(t)[6:])
def test_loss_of_clusters_alike(dtype):
    z = torch.full((2, WIDE), 0.5, dtype=dtype, device="cuda")
    z[1, 7] = 20.0                                    # one far ahead: the others' share is 2^25 small terms
    labels = torch.tensor([5, 6], dtype=torch.int32, device="cuda")
    _, row, dz = gem.label_cross_entropy(z, labels, mean=False)
    v = z.double()
    total = torch.logsumexp(v, 1)
    want = total - v[torch.arange(2), labels.long()]
    # the sum's relative error is the logarithm's absolute one; exp's argument is exact to 3 u times itself
    assert ((row.double() - want).abs() <= 128 * U + 3 * U * 20 + 4 * U * (total.abs() + 20)).all()
    assert abs(want[0].item() - math.log(WIDE)) < 1e-9
    p = (v - total[:, None]).exp()
    p[torch.arange(2), labels.long()] -= 1.0
    step = 2.0 ** -8 if dtype is torch.bfloat16 else U
    assert ((dz.double() - p).abs() <= p.abs() * ((128 + 60 + 16) * U + 1.01 * step) + 1e-38).all()
