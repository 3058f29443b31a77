"""Host-only checks of the training entry points: what they refuse before anything is launched, and their scratch sizes."""
import ctypes as C

import pytest
import torch

import paper_2609_36074_b200 as gem
from paper_2609_36074_b200 import training

P = 1 << 20          # stands for an aligned device address; every call below is refused before it is looked at


def test_scratch_sizes():
    fn = training._load()
    for n, d in ((0, 1), (1, 1), (1, 768), (10 ** 6, 768), (2 ** 40, 16384)):
        assert 0 <= fn["layer_norm_backward_scratch_bytes"](n, d) <= 2 * 4 * d * 4096
        assert 0 <= fn["label_cross_entropy_scratch_bytes"](n, d) <= 1 << 20
    # small calls are one launch that needs none; larger ones do
    assert fn["layer_norm_backward_scratch_bytes"](24, 768) == fn["label_cross_entropy_scratch_bytes"](24, 768) == 0
    assert fn["layer_norm_backward_scratch_bytes"](40000, 768) > 0 < fn["label_cross_entropy_scratch_bytes"](40000, 768)
    assert fn["layer_norm_backward_scratch_bytes"](-1, 4) == 0 and fn["layer_norm_backward_scratch_bytes"](4, 0) == 0
    assert fn["label_cross_entropy_scratch_bytes"](-1, 4) == 0 and fn["label_cross_entropy_scratch_bytes"](4, 0) == 0
    assert fn["clip_grad_norm_scratch_bytes"](-1) == 0
    sizes = [fn["clip_grad_norm_scratch_bytes"](c) for c in (0, 1, 64, 1000, 1001, 100000)]
    assert sizes[0] > 0 and sizes == sorted(sizes)


def test_layer_norm_refuses():
    fn = training._load()["layer_norm"]
    good = dict(x=P, type=0, ld=8, w=P, b=P, wtype=0, n=4, d=8, eps=1e-5, y=2 * P, ldy=8, mean=P, rstd=P)

    def call(**kw):
        return fn(*{**good, **kw}.values(), None)

    for kw in (dict(x=None), dict(x=P + 1), dict(type=3), dict(type=-1), dict(ld=-1), dict(wtype=2), dict(wtype=7), dict(n=-1),
               dict(d=0), dict(d=-4), dict(d=2 ** 31 - 1, ld=2 ** 31, ldy=2 ** 31), dict(eps=-1.0), dict(eps=float("nan")), dict(eps=float("inf")), dict(y=None), dict(y=P),
               dict(ldy=7), dict(w=P + 2), dict(b=P + 1), dict(mean=P + 2), dict(rstd=P + 1), dict(type=2, wtype=1)):
        assert call(**kw) == gem.E_INVALID, kw
    assert call(n=0, x=None, y=None) == gem.OK


def test_layer_norm_backward_refuses():
    fns = training._load()
    size = fns["layer_norm_backward_scratch_bytes"](40000, 8)
    good = dict(dy=P, lddy=8, x=P, ld=8, type=0, mean=P, rstd=P, w=P, wtype=0, n=40000, d=8, dx=2 * P, lddx=8, dw=P, db=P, scratch=P,
                size=size)

    def call(**kw):
        return fns["layer_norm_backward"](*{**good, **kw}.values(), None)

    for kw in (dict(dy=None), dict(x=None), dict(mean=None), dict(rstd=None), dict(type=4), dict(wtype=1), dict(n=-1), dict(d=0), dict(d=2 ** 30 + 1, lddx=2 ** 31),
               dict(lddx=7), dict(dx=P), dict(dx=None, dw=None, db=None), dict(dy=P + 2), dict(x=P + 3), dict(dw=P + 1),
               dict(db=P + 2), dict(w=P + 1), dict(lddy=-8), dict(ld=-1), dict(mean=P + 1), dict(dx=2 * P + 2)):
        assert call(**kw) == gem.E_INVALID, kw
    for kw in (dict(scratch=None), dict(scratch=P + 4), dict(size=size - 1), dict(size=0)):
        assert call(**kw) == gem.E_WORKSPACE, kw


def test_cross_entropy_refuses():
    fns = training._load()
    size = fns["label_cross_entropy_scratch_bytes"](40000, 8)
    good = dict(z=P, type=0, ld=8, labels=P, n=40000, k=8, mean=1, loss=P, row=P, dz=2 * P, ldd=8, scratch=P, size=size)

    def call(**kw):
        return fns["label_cross_entropy"](*{**good, **kw}.values(), None)

    for kw in (dict(z=None), dict(z=P + 2), dict(type=5), dict(ld=-1), dict(labels=None), dict(labels=P + 2), dict(n=-1), dict(k=0), dict(k=2 ** 30 + 1, ldd=2 ** 31),
               dict(mean=2), dict(loss=None), dict(loss=P + 1), dict(row=None), dict(row=P + 2), dict(dz=P + 1), dict(ldd=7),
               dict(dz=P, ld=9)):
        assert call(**kw) == gem.E_INVALID, kw
    for kw in (dict(scratch=None), dict(scratch=P + 8), dict(size=size - 1)):
        assert call(**kw) == gem.E_WORKSPACE, kw


def test_clip_refuses():
    fns = training._load()
    size = fns["clip_grad_norm_scratch_bytes"](2)

    def call(second=(P, 2 * P, 10, 0, 0), count=2, max_norm=1.0, eps=0.0, norm=P, scratch=P, size=size, table=True):
        t = (training.Tensor * 2)()
        t[0], t[1] = (P, 2 * P, 5, 2, 0), second
        return fns["clip_grad_norm"](t if table else None, count, max_norm, eps, norm, scratch, size, None)

    for kw in (dict(second=(None, 2 * P, 10, 0, 0)), dict(second=(P, None, 10, 0, 0)), dict(second=(P + 1, 2 * P, 10, 0, 0)),
               dict(second=(P, 2 * P + 2, 10, 0, 0)), dict(second=(P, 2 * P, -1, 0, 0)), dict(second=(P, 2 * P, 10, 3, 3)),
               dict(second=(P, 2 * P, 10, 0, 2)), dict(second=(P, 2 * P, 10, 1, 2)), dict(second=(P, P, 10, 1, 0)), dict(count=-1),
               dict(max_norm=-1.0), dict(max_norm=float("nan")), dict(eps=-1.0), dict(norm=None), dict(norm=P + 2), dict(table=False)):
        assert call(**kw) == gem.E_INVALID, kw
    for kw in (dict(scratch=None), dict(scratch=P + 16), dict(size=size - 8)):
        assert call(**kw) == gem.E_WORKSPACE, kw


def test_tensors_on_the_host_are_refused():
    x = torch.randn(4, 8)
    with pytest.raises(ValueError):
        gem.layer_norm(x)
    with pytest.raises(ValueError):
        gem.layer_norm_backward(x, x, x[:, 0], x[:, 0])
    with pytest.raises(ValueError):
        gem.label_cross_entropy(x, torch.zeros(4, dtype=torch.int32))
    with pytest.raises(ValueError):
        gem.clip_grad_norm([x], 1.0)
    with pytest.raises(ValueError):
        gem.grad_norm([x])


def test_record_layout():
    assert C.sizeof(training.Tensor) == 32
