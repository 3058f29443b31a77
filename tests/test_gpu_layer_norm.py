"""Layer norm and its gradient against the definition in 64 bits (bounds: training_reference.py)."""
import pytest
import torch

import paper_2609_36074_b200 as gem
import training_reference as ref

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SHAPES = [(1, 1), (3, 2), (5, 7), (2, 31), (4, 32), (9, 33), (7, 100), (1, 768), (24, 768), (300, 768), (65, 1000), (33, 1001),
          (9, 1024), (17, 1026), (6, 2048), (5, 2049), (3, 4096), (130, 4100), (3, 8191), (2, 16384), (2, 16400), (2, 20000),
          (1, 32768), (2, 40001), (1, 70000)]
TYPES = [(F32, F32), (F16, F16), (F16, F32), (BF16, BF16), (BF16, F32)]


def matrix(n, d, dtype, gen, pad=0, first=0, scale=1.0, offset=0.0):
    """n x d with rows d + pad apart, beginning `first` elements into its memory."""
    flat = torch.empty(n * (d + pad) + first, dtype=dtype, device="cuda")
    m = flat[first:].view(n, d + pad)[:, :d]
    m.copy_(torch.randn(n, d, generator=gen, device="cuda") * scale + offset)
    return m


def inputs(n, d, dtype, wdtype, pad=0, first=0, offset=0.3, seed=0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 7 * n + d)
    x = matrix(n, d, dtype, gen, pad, first, 1.0, offset)
    dy = matrix(n, d, dtype, gen, pad, first, 0.1)
    w = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(wdtype)
    b = (0.2 * torch.randn(d, generator=gen, device="cuda")).to(wdtype)
    return x, dy, w, b


def check(x, dy, w, b, eps=1e-5):
    want, bound = ref.norm(x, w, b, eps)
    got = gem.layer_norm(x, w, b, eps=eps)
    assert got[0].dtype == x.dtype and got[1].dtype == got[2].dtype == F32
    for g, v, e, name in zip(got, want, bound, ("y", "mean", "rstd")):
        ref.assert_within(g, v, e, name)
    _, mean, rstd = got
    wdt = F32 if w is None else w.dtype
    want, bound = ref.norm_grad(dy, x, mean, rstd, w, wdt)
    got = gem.layer_norm_backward(dy, x, mean, rstd, w, need_dweight=True, need_dbias=True)
    assert got[0].dtype == x.dtype and got[1].dtype == got[2].dtype == wdt
    for g, v, e, name in zip(got, want, bound, ("dx", "dw", "db")):
        ref.assert_within(g, v, e, name)


@pytest.mark.parametrize("types", TYPES, ids=lambda t: "-".join(str(x)[6:] for x in t))
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}")
def test_shapes(shape, types):
    check(*inputs(*shape, *types))


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("shape", [(37, 768), (37, 1000), (3, 4096), (2, 20000)], ids=lambda s: f"{s[0]}x{s[1]}")
@pytest.mark.parametrize("pad,first", [(8, 0), (3, 0), (0, 1), (2, 2), (4, 4), (16, 8), (1, 5)])
def test_strides_and_alignment(shape, dtype, pad, first):
    check(*inputs(*shape, dtype, dtype, pad, first))


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 147, 149, 1000, 5000, 40000])
@pytest.mark.parametrize("d", [40, 768, 1001])
def test_row_counts(n, d):
    check(*inputs(n, d, BF16, F32))


@pytest.mark.parametrize("d", [64, 768, 5000])
def test_without_weight_and_bias(d):
    x, dy, w, b = inputs(11, d, F32, F32)
    check(x, dy, None, None)
    want, bound = ref.norm(x, None, b, 1e-5)
    ref.assert_within(gem.layer_norm(x, None, b)[0], want[0], bound[0], "bias alone")
    want, bound = ref.norm(x, w, None, 1e-5)
    ref.assert_within(gem.layer_norm(x, w)[0], want[0], bound[0], "weight alone")


@pytest.mark.parametrize("n,d", [(40, 768), (3, 5000), (2, 40001)])
def test_parts_of_the_gradient(n, d):
    x, dy, w, b = inputs(n, d, F32, F32)
    _, mean, rstd = gem.layer_norm(x, w, b)
    whole = gem.layer_norm_backward(dy, x, mean, rstd, w)
    for need in [(1, 0, 0), (0, 1, 0), (0, 0, 1), (1, 1, 0), (0, 1, 1), (1, 0, 1)]:
        part = gem.layer_norm_backward(dy, x, mean, rstd, w, *map(bool, need))
        for p, q, k in zip(part, whole, need):
            assert (p is None) == (not k)
            if k:
                want, bound = ref.norm_grad(dy, x, mean, rstd, w, F32)
                i = [a is p for a in part].index(True)
                ref.assert_within(p, want[i], bound[i])


@pytest.mark.parametrize("d", [64, 768, 1001, 6000, 40001])
def test_an_offset_far_above_the_spread(d):
    x, dy, w, b = inputs(9, d, F32, F32, offset=1000.0)
    check(x, dy, w, b)


@pytest.mark.parametrize("d", [1, 64, 768, 4096])
def test_rows_of_one_value(d):
    x = torch.full((5, d), 3.0, device="cuda")
    b = torch.linspace(-1, 1, d, device="cuda") if d > 1 else torch.ones(1, device="cuda")
    y, mean, rstd = gem.layer_norm(x, torch.ones(d, device="cuda"), b, eps=1e-5)
    assert (mean - 3.0).abs().max() <= 1e-5
    assert (rstd * (1e-5 ** 0.5) - 1).abs().max() <= 1e-3
    assert (y - b).abs().max() <= 2e-3          # (3 - mean) rstd: the mean's rounding times 316


@pytest.mark.parametrize("d", [100, 768, 1001, 5000, 40001])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_bad_row_stays_alone(d, bad):
    x, dy, w, b = inputs(12, d, F32, F32)
    clean = gem.layer_norm(x, w, b)
    x2 = x.clone()
    x2[5, d // 2] = bad
    y, mean, rstd = gem.layer_norm(x2, w, b)
    rows = [i for i in range(12) if i != 5]
    assert torch.equal(y[rows], clean[0][rows]) and torch.equal(mean[rows], clean[1][rows])
    assert y[5].isnan().all()
    dx = gem.layer_norm_backward(dy, x2, mean, rstd, w)[0]
    want = gem.layer_norm_backward(dy, x, clean[1], clean[2], w)[0]
    assert torch.equal(dx[rows], want[rows]) and dx[5].isnan().all()


@pytest.mark.parametrize("d", [6, 100, 768])
def test_gradient_against_differences(d):
    n, eps, step = 3, 1e-5, 1e-4
    x, dy, w, b = inputs(n, d, F32, F32)
    _, mean, rstd = gem.layer_norm(x, w, b, eps=eps)
    dx, dw, db = gem.layer_norm_backward(dy, x, mean, rstd, w)

    def loss(x, w, b):
        return (ref.norm(x, w, b, eps)[0][0] * dy.double()).sum()

    gen = torch.Generator(device="cuda").manual_seed(3)
    for which, grad in enumerate((dx, dw, db)):
        for _ in range(4):
            args = [x.double(), w.double(), b.double()]
            way = torch.randn(args[which].shape, generator=gen, device="cuda", dtype=torch.float64)
            lo, hi = list(args), list(args)
            lo[which], hi[which] = args[which] - step * way, args[which] + step * way
            diff = (loss(*hi) - loss(*lo)) / (2 * step)
            # central differences: step^2 times the third derivative, here below 1e-5 of the terms
            assert (diff - (grad.double() * way).sum()).abs() <= 2e-5 * (grad.double() * way).abs().sum() + 1e-7


def test_leading_dimensions_and_repeated_rows():
    x, dy, w, b = inputs(24, 96, F32, F32)
    y, mean, rstd = gem.layer_norm(x.view(2, 3, 4, 96), w, b)
    flat = gem.layer_norm(x, w, b)
    assert y.shape == (2, 3, 4, 96) and mean.shape == (2, 3, 4)
    assert torch.equal(y.view(24, 96), flat[0])
    dx = gem.layer_norm_backward(dy.view(2, 3, 4, 96), x.view(2, 3, 4, 96), mean, rstd, w)
    want = gem.layer_norm_backward(dy, x, flat[1], flat[2], w)
    assert torch.equal(dx[0].view(24, 96), want[0]) and torch.equal(dx[1], want[1])
    # a gradient that is one row broadcast over all of them
    one = dy[:1].expand(24, 96)
    got = gem.layer_norm_backward(one, x, flat[1], flat[2], w)
    want = gem.layer_norm_backward(one.contiguous(), x, flat[1], flat[2], w)
    for g, v in zip(got, want):
        assert torch.allclose(g, v, rtol=1e-5, atol=1e-6)


def test_no_rows():
    x = torch.empty(0, 768, device="cuda")
    w = torch.ones(768, device="cuda")
    y, mean, rstd = gem.layer_norm(x, w, w)
    assert y.shape == (0, 768) and mean.shape == (0,)
    dx, dw, db = gem.layer_norm_backward(x, x, mean, rstd, w)
    assert dx.shape == (0, 768) and (dw == 0).all() and (db == 0).all()


def test_output_given():
    x, dy, w, b = inputs(20, 100, BF16, F32)
    want, bound = ref.norm(x, w, b, 1e-5)
    whole = torch.full((20, 120), 7.0, dtype=BF16, device="cuda")
    y = gem.layer_norm(x, w, b, out=whole[:, 10:110])[0]
    ref.assert_within(y, want[0], bound[0])
    assert (whole[:, :10] == 7).all() and (whole[:, 110:] == 7).all()


@pytest.mark.parametrize("d", [64, 777])
def test_offsets_beyond_32_bits(d):
    n, ld = 2100, 2 ** 20 + 8
    flat = torch.empty((n - 1) * ld + d, dtype=BF16, device="cuda")
    x = flat.as_strided((n, d), (ld, 1))
    gen = torch.Generator(device="cuda").manual_seed(1)
    x.copy_(torch.randn(n, d, generator=gen, device="cuda"))
    w = torch.ones(d, device="cuda")
    check(x, x, w, w)


def test_same_bits_each_time_and_on_a_side_stream_and_in_a_graph():
    for n, d, dtype in ((5000, 768, BF16), (70, 5000, F32), (24, 768, F32), (4000, 1001, F16), (3, 40001, F32)):
        x, dy, w, b = inputs(n, d, dtype, F32)

        def both(stream=None):
            y, mean, rstd = gem.layer_norm(x, w, b, stream=stream)
            return (y, mean, rstd) + gem.layer_norm_backward(dy, x, mean, rstd, w, stream=stream)

        first = both()
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        second = both(side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            third = both()
        graph.replay()
        torch.cuda.synchronize()
        for a, p, q in zip(first, second, third):
            assert torch.equal(a, p) and torch.equal(a, q)


def test_refusals():
    x = torch.randn(4, 64, device="cuda")
    w, s = torch.ones(64, device="cuda"), torch.ones(4, device="cuda")
    for call in (lambda: gem.layer_norm(x.double()), lambda: gem.layer_norm(x.cpu()), lambda: gem.layer_norm(x.t()),
                 lambda: gem.layer_norm(x, w[:63]), lambda: gem.layer_norm(x, w.half()), lambda: gem.layer_norm(x, w, w.half()),
                 lambda: gem.layer_norm(x, w, w, eps=-1.0), lambda: gem.layer_norm(x, w, w, eps=float("nan")),
                 lambda: gem.layer_norm(x, out=torch.empty(4, 63, device="cuda")),
                 lambda: gem.layer_norm(x, torch.ones(128, device="cuda")[::2]),
                 lambda: gem.layer_norm(torch.empty(3, 0, device="cuda")), lambda: gem.layer_norm(s[0]),
                 lambda: gem.layer_norm(torch.randn(4, 6, 64, device="cuda").transpose(0, 1)),
                 lambda: gem.layer_norm_backward(x[:3], x, s, s, w), lambda: gem.layer_norm_backward(x.half(), x, s, s, w),
                 lambda: gem.layer_norm_backward(x, x, s[:3], s, w), lambda: gem.layer_norm_backward(x, x, s, s.half(), w)):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError):
        gem.layer_norm(x, out=x)                     # the output may not be the input
