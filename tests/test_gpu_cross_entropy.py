"""Cross entropy on cluster labels, loss and gradient, against the definition in 64 bits."""
import pytest
import torch

import paper_2609_36074_b200 as gem
import training_reference as ref

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SHAPES = [(1, 1), (2, 2), (3, 3), (5, 31), (4, 32), (9, 33), (16, 100), (1, 1000), (300, 1000), (65, 1001), (9, 2048), (5, 2049),
          (33, 4096), (3, 8190), (7, 8193), (2, 32768), (3, 32770), (2, 50000), (1, 131073)]


def inputs(n, k, dtype, pad=0, first=0, out=0.2, seed=0, spread=3.0):
    gen = torch.Generator(device="cuda").manual_seed(seed + 5 * n + k)
    flat = torch.empty(n * (k + pad) + first, dtype=dtype, device="cuda")
    z = flat[first:].view(n, k + pad)[:, :k]
    z.copy_(torch.randn(n, k, generator=gen, device="cuda") * spread)
    labels = torch.randint(0, k, (n,), generator=gen, device="cuda", dtype=torch.int32)
    labels[torch.rand(n, generator=gen, device="cuda") < out] = -1
    return z, labels


def check(z, labels, mean=True, **kw):
    want, bound = ref.cross_entropy(z, labels, mean)
    got = gem.label_cross_entropy(z, labels, mean=mean, **kw)
    assert got[0].dtype == got[1].dtype == F32 and got[0].shape == () and got[2].dtype == z.dtype
    for g, v, e, name in zip(got, want, bound, ("loss", "row_loss", "dlogits")):
        ref.assert_within(g, v, e, name)
    return got


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: f"{s[0]}x{s[1]}")
def test_shapes(shape, dtype):
    z, labels = inputs(*shape, dtype)
    check(z, labels, True)
    check(z, labels, False)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=lambda t: str(t)[6:])
@pytest.mark.parametrize("shape", [(37, 1000), (37, 1001), (3, 4096), (2, 40000)], ids=lambda s: f"{s[0]}x{s[1]}")
@pytest.mark.parametrize("pad,first", [(8, 0), (3, 0), (0, 1), (2, 2), (4, 4), (16, 8), (1, 5)])
def test_strides_and_alignment(shape, dtype, pad, first):
    check(*inputs(*shape, dtype, pad, first))


@pytest.mark.parametrize("n", [1, 2, 31, 32, 33, 147, 149, 1000, 5000, 40000, 70001])
@pytest.mark.parametrize("k", [8, 100, 1001])
def test_row_counts(n, k):
    check(*inputs(n, k, BF16))


@pytest.mark.parametrize("shape", [(40, 100), (21, 1000), (21, 1001), (4, 9000), (3, 60001)], ids=lambda s: f"{s[0]}x{s[1]}")
@pytest.mark.parametrize("dtype", [F32, BF16], ids=lambda t: str(t)[6:])
def test_gradient_written_over_the_logits(shape, dtype):
    z, labels = inputs(*shape, dtype)
    want = check(z, labels)
    got = gem.label_cross_entropy(z, labels, dlogits=z)
    assert got[2] is z and all(torch.equal(g, v) for g, v in zip(got, want))


def test_loss_alone_and_output_given():
    z, labels = inputs(50, 100, BF16)
    want = check(z, labels)
    got = gem.label_cross_entropy(z, labels, need_grad=False)
    assert got[2] is None and torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    whole = torch.full((50, 130), 7.0, dtype=BF16, device="cuda")
    gem.label_cross_entropy(z, labels, dlogits=whole[:, 5:105])
    want, bound = ref.cross_entropy(z, labels, True)
    ref.assert_within(whole[:, 5:105], want[2], bound[2])
    assert (whole[:, :5] == 7).all() and (whole[:, 105:] == 7).all()


@pytest.mark.parametrize("k", [7, 100, 1001, 5000, 40001])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=lambda t: str(t)[6:])
def test_masked_clusters(k, dtype):
    z, labels = inputs(8, k, dtype, out=0.0)
    lowest = torch.finfo(dtype).min
    at = torch.arange(8, device="cuda")
    keep = z[at, labels.long()].clone()
    z[0, : k // 2] = -float("inf")                 # some clusters masked by -inf
    z[1, 1:] = -float("inf")                       # all but one
    z[2, : k // 2] = lowest                        # the type's lowest value instead
    z[3, :] = lowest                               # nothing but it: all alike
    z[at, labels.long()] = torch.where(at == 3, z[at, labels.long()], keep)
    labels[1] = 0
    z[1, 1:] = -float("inf")
    z[1, 0] = 2.0
    check(z, labels)
    row, dz = gem.label_cross_entropy(z, labels, mean=False)[1:]
    assert row[1] == 0 and (dz[1] == 0).all()
    want = torch.log(torch.tensor(float(k), dtype=torch.float64))
    assert abs(row[3].item() - want.item()) <= 1e-5 * max(1.0, want.item())


@pytest.mark.parametrize("k", [7, 100, 1001, 5000, 40001])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=lambda t: str(t)[6:])
def test_rows_without_an_answer(k, dtype):
    z, labels = inputs(9, k, dtype, out=0.0)
    clean = gem.label_cross_entropy(z, labels, mean=False)
    inf, nan = float("inf"), float("nan")
    z2, l2 = z.clone(), labels.clone()
    z2[0] = -inf                                   # nothing left
    z2[1, labels[1].long()] = -inf                 # the label's own cluster masked
    z2[2, k // 2] = nan
    z2[3, k // 2] = inf
    z2[4] = nan                                    # does not count, whatever it holds
    l2[4] = -100
    l2[5] = k                                      # no such cluster
    l2[6] = 2 ** 31 - 1
    loss, row, dz = gem.label_cross_entropy(z2, l2, mean=False)
    assert row[0] == inf and (dz[0] == 0).all()
    assert row[1] == inf and dz[1].isfinite().all() and dz[1, labels[1].long()] == -1
    for i in (2, 3, 5, 6):
        assert row[i].isnan() and dz[i].isnan().all(), i
    assert row[4] == 0 and (dz[4] == 0).all()
    assert torch.equal(row[7:], clean[1][7:]) and torch.equal(dz[7:], clean[2][7:])
    assert loss.isnan()


@pytest.mark.parametrize("n,k", [(1, 10), (40, 1000), (3, 50000)])
def test_no_row_counts(n, k):
    z, _ = inputs(n, k, F32)
    labels = torch.full((n,), -1, dtype=torch.int32, device="cuda")
    for mean in (True, False):
        loss, row, dz = gem.label_cross_entropy(z, labels, mean=mean)
        assert loss == 0 and (row == 0).all() and (dz == 0).all()


def test_no_rows():
    loss, row, dz = gem.label_cross_entropy(torch.empty(0, 10, device="cuda"), torch.empty(0, dtype=torch.int32, device="cuda"))
    assert loss == 0 and row.shape == (0,) and dz.shape == (0, 10)


@pytest.mark.parametrize("scale", [1e3, 1e30])
def test_logits_far_apart(scale):
    z, labels = inputs(30, 257, F32, spread=scale)
    check(z, labels)


@pytest.mark.parametrize("k", [5, 100, 1500])
def test_gradient_against_differences(k):
    z, labels = inputs(6, k, F32)
    loss, _, dz = gem.label_cross_entropy(z, labels)
    gen = torch.Generator(device="cuda").manual_seed(3)
    step = 1e-4
    for _ in range(6):
        way = torch.randn(z.shape, generator=gen, device="cuda", dtype=torch.float64)
        f = [ref.cross_entropy(z.double() + s * step * way, labels, True)[0][0] for s in (1, -1)]
        got = (dz.double() * way).sum()
        assert ((f[0] - f[1]) / (2 * step) - got).abs() <= 2e-5 * (dz.double() * way).abs().sum() + 1e-7


def test_leading_dimensions():
    z, labels = inputs(24, 100, F32)
    want = gem.label_cross_entropy(z, labels)
    got = gem.label_cross_entropy(z.view(4, 6, 100), labels.view(4, 6))
    assert got[1].shape == (4, 6) and got[2].shape == (4, 6, 100)
    assert torch.equal(got[2].view(24, 100), want[2]) and torch.equal(got[0], want[0])


@pytest.mark.parametrize("k", [64, 777])
def test_offsets_beyond_32_bits(k):
    n, ld = 2100, 2 ** 20 + 8
    z = torch.empty((n - 1) * ld + k, dtype=BF16, device="cuda").as_strided((n, k), (ld, 1))
    gen = torch.Generator(device="cuda").manual_seed(1)
    z.copy_(torch.randn(n, k, generator=gen, device="cuda"))
    labels = torch.randint(0, k, (n,), generator=gen, device="cuda", dtype=torch.int32)
    want, bound = ref.cross_entropy(z, labels, True)
    check(z, labels)
    gem.label_cross_entropy(z, labels, dlogits=z)
    ref.assert_within(z, want[2], bound[2])


def test_same_bits_each_time_and_on_a_side_stream_and_in_a_graph():
    for n, k, dtype in ((5000, 1000, BF16), (16, 100, F32), (3000, 1001, F16), (40, 20000, F32), (3, 60000, F32)):
        z, labels = inputs(n, k, dtype)
        first = gem.label_cross_entropy(z, labels)
        side = torch.cuda.Stream()
        side.wait_stream(torch.cuda.current_stream())
        second = gem.label_cross_entropy(z, labels, stream=side)
        torch.cuda.current_stream().wait_stream(side)
        torch.cuda.synchronize()
        graph = torch.cuda.CUDAGraph()
        with torch.cuda.graph(graph):
            third = gem.label_cross_entropy(z, labels)
        for _ in range(2):
            graph.replay()
        torch.cuda.synchronize()
        for a, p, q in zip(first, second, third):
            assert torch.equal(a, p) and torch.equal(a, q)


def test_refusals():
    z = torch.randn(4, 64, device="cuda")
    y = torch.zeros(4, dtype=torch.int32, device="cuda")
    for call in (lambda: gem.label_cross_entropy(z.double(), y), lambda: gem.label_cross_entropy(z, y.long()),
                 lambda: gem.label_cross_entropy(z, y[:3]), lambda: gem.label_cross_entropy(z.t(), y),
                 lambda: gem.label_cross_entropy(z, y.cpu()), lambda: gem.label_cross_entropy(z.cpu(), y),
                 lambda: gem.label_cross_entropy(z, y, dlogits=z.half()), lambda: gem.label_cross_entropy(z, y, dlogits=z[:3]),
                 lambda: gem.label_cross_entropy(z[:, :0], y),
                 lambda: gem.label_cross_entropy(z, torch.zeros(8, dtype=torch.int32, device="cuda")[::2])):
        with pytest.raises(ValueError):
            call()
    with pytest.raises(RuntimeError):
        gem.label_cross_entropy(z, y, dlogits=torch.empty(1, 64, device="cuda").expand(4, 64))
