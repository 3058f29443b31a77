"""What the expert layer's functions refuse of tensors that are on the GPU; nothing is launched."""
import pytest
import torch

import paper_2609_36074_b200 as gem

pytestmark = pytest.mark.gpu

BF16 = torch.bfloat16


def no(*args, **kw):
    with pytest.raises(ValueError):
        args[0](*args[1:], **kw)


def test_route():
    z = torch.randn(6, 16, device="cuda")
    i = torch.zeros(6, 2, dtype=torch.int32, device="cuda")
    for kw in (dict(k=0), dict(k=17), dict(k=2, score="tanh"), dict(k=2, groups=3), dict(k=2, groups=4, kept_groups=5), dict(k=9, groups=4, kept_groups=2), dict(k=2, groups=4, group_best=3),
               dict(k=2, scale=float("nan")), dict(k=2, bias=torch.zeros(16, device="cuda", dtype=BF16)), dict(k=2, bias=torch.zeros(8, device="cuda")), dict(k=2, bias=torch.zeros(16))):
        no(gem.route, z, **kw)
    no(gem.route, z.int(), 2)
    no(gem.route, z.t(), 2)
    no(gem.route, z.view(2, 3, 16), 2)
    no(gem.route, torch.randn(2, 513, device="cuda"), 2)
    v = torch.zeros(6, 2, device="cuda")
    no(gem.route_backward, v, z, i.long())
    no(gem.route_backward, v[:, :1], z, i)
    no(gem.route_backward, v.half(), z, i)
    no(gem.route_backward, v, z, i[:5])
    no(gem.route_backward, v, z, i, "max")


def test_products():
    x, w = torch.randn(6, 16, device="cuda").to(BF16), torch.randn(3, 16, 8, device="cuda").to(BF16)
    o, row = torch.zeros(4, dtype=torch.int32, device="cuda"), torch.zeros(5, dtype=torch.int32, device="cuda")
    dy = torch.zeros(6, 8, device="cuda", dtype=BF16)
    no(gem.expert_product, x.float(), w, o)
    no(gem.expert_product, x.double(), w.double(), o)
    no(gem.expert_product, x, w.half(), o)
    no(gem.expert_product, x[:, :15], w, o)
    no(gem.expert_product, x, w[:, :, ::2], o)
    no(gem.expert_product, x, w[0], o)
    no(gem.expert_product, x, w, o[:3])
    no(gem.expert_product, x, w, o.long())
    no(gem.expert_product, x, w, o, row.long())
    no(gem.expert_product, x, w, o, row.view(1, 5))
    no(gem.expert_product, x, w, o, out=dy[:5])
    no(gem.expert_product, x, w.cpu(), o)
    no(gem.expert_product, x, w, o, stream=torch.cuda.Stream(), out=dy.float())
    no(gem.expert_product_backward, dy[:5], x, w, o)
    no(gem.expert_product_backward, dy.half(), x, w, o)
    no(gem.expert_product_backward, dy, x, w, o, row)


def test_combine():
    y, p = torch.randn(8, 16, device="cuda"), torch.zeros(4, 2, dtype=torch.int32, device="cuda")
    v, o = torch.zeros(4, 2, device="cuda"), torch.zeros(3, dtype=torch.int32, device="cuda")
    no(gem.combine, y, p.long())
    no(gem.combine, y, p[0])
    no(gem.combine, y, p, v[:, :1])
    no(gem.combine, y, p, v.half())
    no(gem.combine, y, p, v, out=y[:4].half())
    no(gem.combine, y.int(), p)
    no(gem.combine, y, torch.zeros(4, 33, dtype=torch.int32, device="cuda"))
    no(gem.combine_backward, y[:3], y, p, v, o)
    no(gem.combine_backward, y[:4].half(), y, p, v, o)
    no(gem.combine_backward, y[:4], y, p, v, o[0])
    no(gem.combine_backward, y[:4], y, p, v, o.long())


def test_activation():
    z = torch.randn(4, 33, device="cuda")
    no(gem.activation, z, "relu")
    no(gem.activation, z, "silu", True)
    no(gem.activation, z.int(), "silu")
    no(gem.activation, z, "silu", out=z[:3])
    no(gem.activation, z.t(), "silu")
    saved = gem.checkpoint(z)
    no(gem.activation_backward, z, saved, "silu", True)
    no(gem.activation_backward, z[:3], saved, "silu")
    no(gem.activation_backward, z.half(), saved, "silu")
    no(gem.activation_backward, z, saved._replace(q=saved.q[:, :32]), "silu")
    no(gem.activation_backward, z, saved._replace(scale=saved.scale.int()), "silu")
    no(gem.restore, gem.activation(torch.randn(4, 32, device="cuda"), "silu", True)[1])
