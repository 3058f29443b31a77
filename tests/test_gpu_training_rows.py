"""Row kernels of the training operators where a group, a block or a cluster has many rows, and where matrices begin off
16 bytes or rows are not a width apart (bounds: training_reference.py)."""
import pytest
import torch

import paper_2609_36074_b200 as gem
import training_reference as ref

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
NAN = float("nan")
# rows enough that every block or cluster takes at least nine of them: more than the stages of its ring and more than twice
# the parts of its messages' buffer
MANY = [(5600, 4000), (5600, 4001), (1500, 8200), (1500, 8199), (750, 16400), (750, 16385), (400, 32768), (400, 40000), (400, 40001)]


def lying(n, d, dtype, ld, first, around=NAN):
    """(memory, n x d view of it): rows ld apart from element `first` on, `around` everywhere else."""
    flat = torch.full((first + (n - 1) * ld + d + 16,), around, dtype=dtype, device="cuda")
    return flat, flat.as_strided((n, d), (ld, 1), first)


def filled(n, d, dtype, ld, first, seed, scale=1.0, offset=0.0):
    flat, m = lying(n, d, dtype, ld, first)
    gen = torch.Generator(device="cuda").manual_seed(seed)
    if ld >= d:
        m.copy_(torch.randn(n, d, generator=gen, device="cuda") * scale + offset)
    else:                                             # overlapping or repeated rows: all of their memory
        span = (n - 1) * ld + d
        flat[first:first + span] = torch.randn(span, generator=gen, device="cuda") * scale + offset
    return m


def kept(flat, n, d, ld, first, around=7.0):
    outside = torch.ones(flat.numel(), dtype=torch.bool, device="cuda")
    outside.as_strided((n, d), (ld, 1), first).fill_(False)
    return bool((flat[outside] == around).all())


def check_norm(x, dy, w, b, out=None, grads=(True, True, True)):
    want, bound = ref.norm(x, w, b, 1e-5)
    got = gem.layer_norm(x, w, b, out=out)
    for g, v, e, name in zip(got, want, bound, ("y", "mean", "rstd")):
        ref.assert_within(g, v, e, name)
    _, mean, rstd = got
    want, bound = ref.norm_grad(dy, x, mean, rstd, w, w.dtype)
    got = gem.layer_norm_backward(dy, x, mean, rstd, w, *grads)
    for g, v, e, name in zip(got, want, bound, ("dx", "dw", "db")):
        if g is not None:
            ref.assert_within(g, v, e, name)


def check_loss(z, labels, mean=True, **kw):
    want, bound = ref.cross_entropy(z, labels, mean)
    got = gem.label_cross_entropy(z, labels, mean=mean, **kw)
    for g, v, e, name in zip(got, want, bound, ("loss", "row_loss", "dlogits")):
        if g is not None:
            ref.assert_within(g, v, e, name)


def weights(d, seed, dtype=F32):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return ((1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(dtype), (0.2 * torch.randn(d, generator=gen, device="cuda")).to(dtype))


def some_labels(n, k, seed):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    labels = torch.randint(0, k, (n,), generator=gen, device="cuda", dtype=torch.int32)
    labels[torch.rand(n, generator=gen, device="cuda") < 0.2] = -1
    return labels


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("shape", MANY, ids=lambda s: f"{s[0]}x{s[1]}")
def test_many_rows_a_block_or_cluster(shape, dtype):
    n, d = shape
    x, dy = filled(n, d, dtype, d, 0, 1, 1.0, 0.3), filled(n, d, dtype, d, 0, 2, 0.1)
    check_norm(x, dy, *weights(d, 3))
    labels = some_labels(n, d, 5)
    z = filled(n, d, dtype, d, 0, 4, 3.0)
    check_loss(z, labels)
    want, bound = ref.cross_entropy(z, labels, True)
    gem.label_cross_entropy(z, labels, dlogits=z)
    ref.assert_within(z, want[2], bound[2], "over the logits")


# widths of a vector, a warp, a block and a cluster
@pytest.mark.parametrize("dtype", [F32, BF16], ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("first,more", [(1, 0), (3, 0), (5, 8), (7, 1), (2, 13)])
@pytest.mark.parametrize("shape", [(70, 3), (700, 33), (300, 250), (200, 777), (90, 2050), (700, 4100), (300, 9000), (120, 25003), (60, 33001)],
                         ids=lambda s: f"{s[0]}x{s[1]}")
def test_matrices_that_begin_off_16_bytes(shape, first, more, dtype):
    n, d = shape
    ld = d + more
    x, dy = filled(n, d, dtype, ld, first, 1, 1.0, 0.3), filled(n, d, dtype, ld, first, 2, 0.1)
    w, b = weights(d, 3)
    flat, out = lying(n, d, dtype, ld, first, 7.0)
    check_norm(x, dy, w, b, out=out, grads=(False, True, True))
    assert kept(flat, n, d, ld, first)
    z, labels = filled(n, d, dtype, ld, first, 4, 3.0), some_labels(n, d, 5)
    check_loss(z, labels, need_grad=False)
    flat, dz = lying(n, d, dtype, ld, first, 7.0)
    check_loss(z, labels, dlogits=dz)
    assert kept(flat, n, d, ld, first)
    want, bound = ref.cross_entropy(z, labels, True)
    gem.label_cross_entropy(z, labels, dlogits=z)
    ref.assert_within(z, want[2], bound[2], "over the logits")
    if more:
        assert z.as_strided((n - 1, more), (ld, 1), first + d).isnan().all()


@pytest.mark.parametrize("dtype", [F32, BF16], ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("n,d,ld,first", [(500, 768, 0, 0), (500, 768, 0, 1), (500, 769, 0, 0), (40, 9001, 0, 3), (300, 64, 0, 0), (300, 64, 4, 1),
                                          (300, 700, 1, 0), (300, 700, 8, 3), (60, 5000, 2500, 0), (60, 5000, 2501, 2), (9, 40001, 0, 0),
                                          (9, 70000, 35000, 0)])
def test_rows_that_repeat_or_overlap(n, d, ld, first, dtype):
    x, dy = filled(n, d, dtype, ld, first, 1, 1.0, 0.3), filled(n, d, dtype, ld, first, 2, 0.1)
    w, b = weights(d, 3)
    check_norm(x, dy, w, b)
    check_norm(x, dy, w, b, grads=(False, True, True))
    check_norm(x.contiguous(), dy, w, b)
    check_loss(x, some_labels(n, d, 5))
    check_loss(x, some_labels(n, d, 5), need_grad=False)
