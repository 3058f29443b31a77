"""Host-only checks of the expert layer's entry points: what they refuse before anything is launched."""
import ctypes as C
import math

import pytest
import torch

import paper_2609_36074_b200 as gem
from paper_2609_36074_b200 import experts

P = 1 << 20          # stands for an aligned device address; every call below is refused before it is looked at


def refuses(name, good, bad, nothing=()):
    fn = experts._load()[name]
    for kw in bad:
        assert set(kw) <= set(good), kw
        assert fn(*{**good, **kw}.values(), None) == gem.E_INVALID, kw
    for kw in nothing:
        assert fn(*{**good, **kw}.values(), None) == gem.OK, kw


def test_route_refuses():
    fns = experts._load()
    size = fns["route_scratch_bytes"](1000, 16)
    assert size > 0 and fns["route_scratch_bytes"](4, 16) == 0 and fns["route_scratch_bytes"](1000, 513) == fns["route_scratch_bytes"](-1, 4) == 0
    good = dict(z=P, type=0, ld=16, bias=P, n=1000, experts=16, k=4, score=0, groups=4, kept=2, best=2, renorm=1, scale=1.0, expert=P, weight=P, offset=P,
                row=P, place=P, scratch=P, size=size)
    refuses("route", good, (
        dict(z=None), dict(z=P + 2), dict(type=3), dict(type=-1), dict(ld=-1), dict(bias=P + 1), dict(n=-1), dict(experts=0), dict(experts=513, groups=1, kept=1), dict(k=0),
        dict(k=9), dict(k=33, experts=64), dict(score=2), dict(score=-1), dict(groups=0), dict(groups=3), dict(groups=33, experts=66), dict(kept=0), dict(kept=5),
        dict(best=0), dict(best=3), dict(renorm=2), dict(scale=math.inf), dict(scale=math.nan), dict(expert=None), dict(weight=P + 2), dict(offset=None), dict(offset=P + 1),
        dict(row=None), dict(place=P + 3), dict(n=1 << 29), dict(n=(1 << 29) - (1 << 14))))
    fn = fns["route"]
    for kw in (dict(scratch=None), dict(scratch=P + 16), dict(size=size - 1), dict(size=0)):
        assert fn(*{**good, **kw}.values(), None) == gem.E_WORKSPACE, kw


def test_route_backward_refuses():
    good = dict(dw=P, z=P, type=0, ld=16, expert=P, n=10, experts=16, k=4, score=0, renorm=1, scale=1.0, dz=2 * P, ldd=16)
    refuses("route_backward", good, (
        dict(dw=None), dict(dw=P + 1), dict(z=None), dict(z=P + 1), dict(type=7), dict(ld=-2), dict(expert=None), dict(expert=P + 2), dict(n=-1), dict(experts=0),
        dict(experts=1000), dict(k=0), dict(k=33), dict(score=3), dict(renorm=-1), dict(scale=math.inf), dict(dz=None), dict(dz=P), dict(dz=2 * P + 2), dict(ldd=15)),
        (dict(n=0, z=None, dw=None, dz=None),))


def test_expert_product_refuses():
    good = dict(x=P, type=2, ldx=64, x_rows=100, w=2 * P, ldw=32, sw=64 * 32, turned=0, offset=P, row=None, places=100, experts=4, d_in=64, d_out=32, y=3 * P, ldy=32, scratch=None, size=0)
    refuses("expert_product", good, (
        dict(x=None), dict(x=P + 1), dict(type=-1), dict(type=3), dict(ldx=-1), dict(x_rows=99), dict(x_rows=-1), dict(x_rows=1 << 31, places=5), dict(w=None), dict(w=P + 1),
        dict(ldw=-1), dict(sw=-1), dict(turned=2), dict(offset=None), dict(offset=P + 2), dict(row=P + 2), dict(places=-1), dict(places=1 << 31, x_rows=1 << 31),
        dict(experts=0), dict(experts=513), dict(d_in=0), dict(d_out=0), dict(d_in=(1 << 30) + 1), dict(y=None), dict(y=P), dict(y=2 * P), dict(y=3 * P + 1), dict(ldy=31)),
        (dict(places=0, x=None, y=None),))


def test_expert_product_backward_refuses():
    good = dict(dy=P, lddy=32, x=2 * P, type=1, ldx=64, x_rows=100, w=3 * P, ldw=32, sw=64 * 32, turned=0, offset=P, row=None, places=100, experts=4, d_in=64, d_out=32,
                dx=4 * P, lddx=64, dw=5 * P, lddw=32, sdw=64 * 32, scratch=None, size=0)
    refuses("expert_product_backward", good, (
        dict(dy=None), dict(dy=P + 1), dict(lddy=-1), dict(x=None), dict(x=P + 1), dict(type=3), dict(ldx=-1), dict(x_rows=50), dict(w=None), dict(w=P + 1), dict(ldw=-1),
        dict(sw=-1), dict(turned=-1), dict(offset=None), dict(row=P + 1), dict(places=-1), dict(experts=0), dict(experts=600), dict(d_in=0), dict(d_out=-1),
        dict(dx=None, dw=None), dict(dx=P), dict(dx=4 * P + 1), dict(lddx=63), dict(dw=P), dict(dw=2 * P), dict(dw=4 * P), dict(dw=5 * P + 1), dict(lddw=31), dict(sdw=64 * 32 - 1),
        dict(turned=1, lddw=63)),
        (dict(places=0, dw=None),))


def test_products_want_scratch_where_rows_do_not_begin_on_16_bytes():
    fns = experts._load()
    size = fns["expert_product_scratch_bytes"]
    assert size(P, 2, 64, 100, P, 32, 64 * 32, 0, 4, 64, 32) == 0
    assert size(P, 0, 64, 100, P, 32, 64 * 32, 0, 4, 64, 32) == 3 * (100 * 64 * 2 + 4 * 64 * 32 * 2)
    assert size(P, 5, 64, 100, P, 32, 64 * 32, 0, 4, 64, 32) == 0 and size(P, 0, 64, 1 << 30, P, 32, 64 * 32, 0, 4, 64, 32) == 0
    copy_x, copy_w = 100 * 64 * 2, 4 * 64 * 32 * 2
    for kw in (dict(x=P + 2), dict(ldx=65), dict(ldx=0)):
        a = {**dict(x=P, ldx=64), **kw}
        assert size(a["x"], 1, a["ldx"], 100, P, 32, 64 * 32, 0, 4, 64, 32) == copy_x, kw
    for kw in (dict(w=P + 8), dict(ldw=33, sw=64 * 33), dict(sw=0), dict(sw=64 * 32 + 1)):
        a = {**dict(w=P, ldw=32, sw=64 * 32), **kw}
        assert size(P, 2, 64, 100, a["w"], a["ldw"], a["sw"], 0, 4, 64, 32) == copy_w, kw
    assert size(P, 2, 65, 0, P, 32, 65 * 32, 0, 4, 65, 32) == 0 and size(P, 2, 64, -1, P, 32, 0, 0, 4, 64, 32) == 0
    both = fns["expert_product_backward_scratch_bytes"](P, 33, 100, P, 2, 65, 100, P, 33, 65 * 33, 0, 4, 65, 33)
    assert both == sum(-(-n // 256) * 256 for n in (100 * 40 * 2, 100 * 72 * 2, 4 * 65 * 40 * 2))
    good = dict(x=P, type=2, ldx=65, x_rows=100, w=2 * P, ldw=32, sw=65 * 32, turned=0, offset=P, row=None, places=100, experts=4, d_in=65, d_out=32, y=3 * P, ldy=32,
                scratch=P, size=-(-100 * 72 * 2 // 256) * 256)
    fn = fns["expert_product"]
    for kw in (dict(scratch=None), dict(scratch=P + 16), dict(size=good["size"] - 1), dict(size=0), dict(type=0)):
        assert fn(*{**good, **kw}.values(), None) == gem.E_WORKSPACE, kw
    assert fn(*{**good, **dict(type=0, x_rows=1 << 30, row=P, places=1 << 30)}.values(), None) == gem.E_INVALID


def test_combine_refuses():
    good = dict(y=P, type=0, ldy=16, places=40, place=P, weight=P, n=10, k=4, d=16, out=2 * P, ldo=16)
    refuses("combine", good, (
        dict(y=None), dict(y=P + 2), dict(type=4), dict(ldy=-1), dict(places=-1), dict(places=1 << 31), dict(place=None), dict(place=P + 1), dict(weight=P + 2), dict(n=-1), dict(k=0),
        dict(k=33), dict(d=0), dict(d=(1 << 30) + 1), dict(out=None), dict(out=P), dict(out=2 * P + 1), dict(ldo=15)), (dict(n=0, place=None, out=None),))
    good = dict(dout=P, ldo=16, y=2 * P, type=0, ldy=16, places=40, place=P, weight=P, offset=P, experts=4, n=10, k=4, d=16, dy=3 * P, lddy=16, dw=P)
    refuses("combine_backward", good, (
        dict(dout=None), dict(dout=P + 2), dict(ldo=-1), dict(y=None), dict(y=P + 1), dict(type=9), dict(ldy=-1), dict(places=-1), dict(place=None), dict(weight=P + 1),
        dict(offset=None), dict(offset=P + 1), dict(experts=0), dict(n=-1), dict(k=0), dict(k=40), dict(d=0), dict(dy=P), dict(dy=2 * P), dict(dy=3 * P + 1), dict(lddy=15),
        dict(dw=P + 1), dict(dy=None, dw=None)), (dict(n=0, dy=None, place=None),))


def test_activation_refuses():
    blocks = gem.lib().gem_nlr_checkpoint_blocks
    blocks.argtypes, blocks.restype = [C.c_int32, C.c_int32], C.c_int64
    for d in (1, 31, 32, 33, 100, 4096):
        assert blocks(d, 0) == experts._blocks(d, False) and blocks(d, 1) == experts._blocks(d, True)
    assert blocks(100, 1) == 8 and blocks(0, 0) == blocks(4, 2) == 0
    good = dict(z=P, type=0, ldz=32, n=5, d=16, kind=1, gated=1, y=2 * P, ldy=16, q=P, scale=P)
    refuses("activation", good, (
        dict(z=None), dict(z=P + 1), dict(type=3), dict(ldz=-1), dict(n=-1), dict(d=0), dict(d=(1 << 29) + 1), dict(kind=4), dict(kind=-1), dict(gated=2), dict(y=P), dict(y=2 * P + 2),
        dict(ldy=15), dict(y=None, q=None, scale=None), dict(q=None), dict(scale=None), dict(q=P + 8)), (dict(n=0, z=None),))
    good = dict(dy=P, type=0, lddy=16, z=None, ldz=0, q=P, scale=P, n=5, d=16, kind=1, gated=1, dz=2 * P, lddz=32, y=3 * P, ldy=16)
    refuses("activation_backward", good, (
        dict(dy=None), dict(dz=None), dict(dy=P + 1), dict(type=5), dict(lddy=-1), dict(z=4 * P, ldz=32), dict(q=None, scale=None), dict(scale=None), dict(q=P + 4), dict(n=-1), dict(d=0),
        dict(kind=9), dict(gated=-1), dict(dz=P), dict(dz=2 * P + 1), dict(lddz=31), dict(dz=3 * P), dict(y=3 * P + 1), dict(ldy=15), dict(y=P),
        dict(dy=None, dz=None, y=None), dict(q=None, scale=None, z=2 * P, ldz=32), dict(q=None, scale=None, z=4 * P + 1, ldz=32)), (dict(n=0, dy=None, dz=None),))


def test_tensors_on_the_host_are_refused():
    x, i = torch.randn(4, 8), torch.zeros(4, 2, dtype=torch.int32)
    w, o = torch.randn(2, 8, 8).half(), torch.zeros(3, dtype=torch.int32)
    for call in (lambda: gem.route(x, 2), lambda: gem.route_backward(x[:, :2], x, i), lambda: gem.expert_product(x.half(), w, o), lambda: gem.combine(x, i),
                 lambda: gem.expert_product_backward(x.half(), x.half(), w, o), lambda: gem.combine_backward(x, x, i, None, o), lambda: gem.activation(x, "silu"),
                 lambda: gem.activation_backward(x, x, "silu"), lambda: gem.checkpoint(x),
                 lambda: gem.restore(gem.Checkpoint(torch.zeros(4, 32, dtype=torch.int8), torch.zeros(4, 1, dtype=torch.uint8), (4, 8), torch.float32, False))):
        with pytest.raises(ValueError):
            call()
