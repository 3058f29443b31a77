"""Clipping with a limit or a norm without bound."""
import pytest
import torch

import paper_2609_36074_b200 as gem

pytestmark = pytest.mark.gpu

INF = float("inf")


@pytest.mark.parametrize("size", [100, 300000])          # one launch, several
def test_an_infinite_norm_leaves_zeros_whatever_the_limit(size):
    for limit in (1.0, INF):
        g = torch.ones(size, device="cuda")
        g[3] = -INF
        out = torch.empty_like(g)
        assert gem.clip_grad_norm([g], limit, out=[out]) == INF
        assert (out[:3] == 0).all() and (out[4:] == 0).all() and out[3].isnan()


@pytest.mark.parametrize("size", [100, 300000])
def test_no_limit_leaves_everything(size):
    g = torch.randn(size, device="cuda")
    keep = g.clone()
    norm = gem.clip_grad_norm([g], INF)
    assert torch.equal(g, keep) and norm.isfinite()
    out = torch.empty_like(g)
    gem.clip_grad_norm([g], INF, out=[out])
    assert torch.equal(out, keep)


@pytest.mark.parametrize("size", [100, 300000])
def test_a_nan_shows_whatever_the_limit(size):
    g = torch.ones(size, device="cuda")
    g[5] = float("nan")
    assert gem.clip_grad_norm([g], INF).isnan() and g.isnan().all()
