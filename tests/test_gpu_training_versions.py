"""Tensors that the training operators write into count as changed in place: what autograd saved of them is not used any more."""
import pytest
import torch

import paper_2609_36074_b200 as gem

pytestmark = pytest.mark.gpu


def saved(shape, seed=0):
    """(input, an output that its own backward pass needs)"""
    a = torch.randn(shape, generator=torch.Generator(device="cuda").manual_seed(seed), device="cuda", requires_grad=True)
    return a, a.tanh()


def refused(out):
    with pytest.raises(RuntimeError, match="modified by an inplace operation"):
        out.sum().backward()


def test_gradient_written_over_logits():
    for other_stream in (None, torch.cuda.Stream()):
        _, z = saved((40, 100))
        later = z * 1.0
        torch.cuda.synchronize()
        gem.label_cross_entropy(z.detach(), torch.zeros(40, dtype=torch.int32, device="cuda"), dlogits=z.detach(), stream=other_stream)
        torch.cuda.synchronize()
        refused(later)


def test_gradient_written_into_a_part_of_another():
    _, z = saved((40, 130))
    later = z * 1.0
    logits = torch.randn(40, 100, device="cuda")
    gem.label_cross_entropy(logits, torch.zeros(40, dtype=torch.int32, device="cuda"), dlogits=z.detach()[:, 30:])
    refused(later)


def test_output_of_the_norm():
    _, z = saved((40, 96))
    later = z * 1.0
    gem.layer_norm(torch.randn(40, 96, device="cuda"), out=z.detach())
    refused(later)


def test_clipping_in_place_and_into_outputs():
    for into in (False, True):
        _, z = saved((500,))
        later = z * 1.0
        if into:
            gem.clip_grad_norm([torch.randn(500, device="cuda")], 1e6, out=[z.detach()])
        else:
            gem.clip_grad_norm([torch.randn(30, device="cuda"), z.detach()], 1.0)
        refused(later)


def test_what_is_only_read_stays_usable():
    a, z = saved((40, 100))
    later = z * 1.0
    d = z.detach()
    _, mean, rstd = gem.layer_norm(d)
    gem.layer_norm_backward(d, d, mean, rstd)
    gem.label_cross_entropy(d, torch.zeros(40, dtype=torch.int32, device="cuda"))
    gem.label_cross_entropy(d, torch.zeros(40, dtype=torch.int32, device="cuda"), dlogits=d, need_grad=False)
    gem.grad_norm([d])
    gem.clip_grad_norm([d], 1.0, out=[torch.empty_like(d)])
    later.sum().backward()
    assert torch.allclose(a.grad, 1 - z.detach() ** 2)


def test_tensors_without_versions():
    with torch.inference_mode():
        g = torch.ones(100, device="cuda")
        assert abs(gem.clip_grad_norm([g], 1.0, eps=0.0).item() - 10) <= 1e-5
        assert (g - 0.1).abs().max() <= 1e-7
