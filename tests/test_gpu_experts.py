"""The experts' products, and the weighted sums of their rows, against their definitions in 64 bits."""
import pytest
import torch

import expert_reference as ref
import paper_2609_36074_b200 as gem
from training_reference import assert_within

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
NAMES = {F32: "f32", F16: "f16", BF16: "bf16"}


def name(t):
    return NAMES.get(t, str(t))


def matrix(n, d, dtype, seed, pad=0, first=0, scale=1.0):
    """n rows of d values, `pad` elements between rows, the first `first` elements into its memory."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((n * (d + pad) + first + 8,), float("nan"), dtype=dtype, device="cuda")
    m = flat[first:first + n * (d + pad)].view(n, d + pad)[:, :d]
    m.copy_(torch.randn(n, d, generator=gen, device="cuda") * scale)
    return m


def weights(experts, d_in, d_out, dtype, seed, turned=False):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    w = torch.randn(experts, d_in, d_out, generator=gen, device="cuda") * d_in ** -0.5
    return w.transpose(1, 2).contiguous().to(dtype).transpose(1, 2) if turned else w.to(dtype)


def split(places, experts, seed, uneven=False):
    """Offsets of a random division of the places, some experts without any."""
    gen = torch.Generator().manual_seed(seed)
    share = torch.rand(experts, generator=gen) ** (4 if uneven else 1)
    share[torch.rand(experts, generator=gen) < (0.4 if uneven else 0.1)] = 0.0
    share = share / share.sum().clamp(min=1e-9)
    ends = (share.cumsum(0) * places).round().long().clamp(max=places)
    return torch.cat([torch.zeros(1, dtype=torch.int64), ends]).int().cuda()


def check(places, experts, d_in, d_out, dtype, turned=False, gather=0, pad=0, first=0, seed=0, uneven=False, offset=None):
    offset = split(places, experts, seed + 5, uneven) if offset is None else offset
    row = None
    if gather:
        gen = torch.Generator(device="cuda").manual_seed(seed + 7)
        row = torch.randint(-1, gather, (places,), generator=gen, device="cuda", dtype=torch.int32)
    x = matrix(gather or places, d_in, dtype, seed + 1, pad, first)
    w = weights(experts, d_in, d_out, dtype, seed + 2, turned)
    dy = matrix(places, d_out, dtype, seed + 3, pad, first, 0.1)
    y = gem.expert_product(x, w, offset, row)
    want, bound = ref.product(x, w, offset, row)
    assert_within(y, want, bound, "y")
    used = ref.ranges(offset, places)[-1][1]
    assert (y[used:] == 0).all()
    dx, dw = gem.expert_product_backward(dy, x, w, offset, row)
    (wx, bx), (ww, bw) = ref.product_grad(dy, x, w, offset, row)
    assert dw.shape == w.shape and dw.stride() == w.stride()
    assert_within(dx, wx, bx, "dx")
    assert_within(dw, ww, bw, "dw")
    assert (dx[used:] == 0).all()
    return x, w, dy, offset, row, y, dx, dw


SHAPES = [(1, 1, 8, 8), (1, 4, 64, 64), (5, 3, 64, 72), (129, 2, 768, 128), (300, 5, 200, 264), (513, 7, 1000, 136), (1000, 3, 72, 1024), (2100, 11, 256, 520)]


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=name)
@pytest.mark.parametrize("turned", [False, True], ids=["plain", "turned"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_aligned(shape, turned, dtype):
    check(*shape, dtype, turned, seed=sum(shape))


@pytest.mark.parametrize("dtype", [F32, BF16], ids=name)
@pytest.mark.parametrize("turned", [False, True], ids=["plain", "turned"])
@pytest.mark.parametrize("shape", SHAPES, ids=lambda s: "x".join(map(str, s)))
def test_gathered(shape, turned, dtype):
    check(*shape, dtype, turned, gather=max(1, shape[0] // 3), seed=sum(shape))


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=name)
@pytest.mark.parametrize("gather", [0, 40], ids=["as they are", "gathered"])
@pytest.mark.parametrize("turned", [False, True], ids=["plain", "turned"])
@pytest.mark.parametrize("shape", [(1, 1, 1, 1), (3, 2, 5, 7), (130, 3, 33, 65), (257, 4, 1001, 131), (700, 5, 129, 515)], ids=lambda s: "x".join(map(str, s)))
def test_odd_widths(shape, turned, gather, dtype):
    check(*shape, dtype, turned, gather, seed=sum(shape))


@pytest.mark.parametrize("pad,first", [(8, 0), (3, 0), (0, 1), (16, 8), (1, 5), (8, 4)])
@pytest.mark.parametrize("gather", [0, 50], ids=["as they are", "gathered"])
def test_strides_and_alignment(pad, first, gather):
    check(200, 3, 136, 72, BF16, False, gather, pad, first)
    check(200, 3, 136, 72, F32, True, gather, pad, first)


@pytest.mark.parametrize("turned", [False, True], ids=["plain", "turned"])
@pytest.mark.parametrize("places,experts,d_in,d_out", [(20000, 8, 256, 512), (9000, 64, 128, 264), (5000, 2, 512, 1160), (30000, 300, 64, 64), (4000, 512, 64, 128)])
def test_many_tiles(places, experts, d_in, d_out, turned):
    check(places, experts, d_in, d_out, BF16, turned, gather=places // 2, uneven=True)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=name)
@pytest.mark.parametrize("gather", [0, 1500], ids=["as they are", "gathered"])
@pytest.mark.parametrize("turned", [False, True], ids=["plain", "turned"])
@pytest.mark.parametrize("places,experts,d_in,d_out", [(6000, 6, 520, 1160), (9000, 16, 768, 328), (4097, 2, 1544, 2056)])
def test_large_tiles(places, experts, d_in, d_out, turned, gather, dtype):
    check(places, experts, d_in, d_out, dtype, turned, gather, uneven=True, seed=places + turned)


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=name)
@pytest.mark.parametrize("gather", [0, 900], ids=["as they are", "gathered"])
@pytest.mark.parametrize("places,experts,d_in,d_out", [(20000, 2, 64, 64), (9001, 1, 33, 200), (4096, 3, 256, 40), (70000, 4, 100, 130), (600, 1, 16, 16), (3000, 5, 130, 72)])
def test_long_sums_in_parts(places, experts, d_in, d_out, gather, dtype):
    check(places, experts, d_in, d_out, dtype, False, gather, seed=places)
    check(places, experts, d_in, d_out, dtype, True, gather, uneven=True, seed=places + 1)


@pytest.mark.parametrize("gather", [0, 4000], ids=["as they are", "gathered"])
@pytest.mark.parametrize("experts", [1, 3, 40])
def test_many_tiles_a_block(experts, gather):
    """Dozens of tiles for each block, full ones and almost empty ones after one another."""
    check(40000, experts, 392, 648, BF16, gather=gather, uneven=True, seed=experts)
    offset = torch.arange(experts + 1, dtype=torch.int32, device="cuda") * (40000 // experts)
    offset[1:-1:2] += 1 - 40000 // experts                       # every other expert has one row
    check(40000, experts, 136, 1032, F16, True, gather, offset=offset)


@pytest.mark.parametrize("d_in", [64, 65])
def test_wild_offsets(d_in):
    for o in ([0, 0, 0, 0], [0, 100, 100, 100], [5, 20, 60, 90], [0, 50, 30, 100], [-7, 40, 400, 100], [100, 100, 100, 100], [0, 1, 2, 3]):
        check(100, 3, d_in, 72, F16, offset=torch.tensor(o, dtype=torch.int32, device="cuda"))


@pytest.mark.parametrize("d", [64, 67])
def test_infinities_stay_with_their_rows(d):
    """A NaN or an infinity of one expert (or of an unused row) reaches no other expert's results."""
    offset = torch.tensor([0, 70, 70, 200, 250], dtype=torch.int32, device="cuda")
    x, w, dy = matrix(260, d, BF16, 1), weights(4, d, 72, BF16, 2), matrix(260, 72, BF16, 3)
    clean = gem.expert_product(x, w, offset), *gem.expert_product_backward(dy, x, w, offset)
    x[70:200], dy[70:200], w[2] = float("inf"), float("nan"), float("nan")
    x[250:], dy[250:], w[1] = float("nan"), float("inf"), float("inf")
    y, (dx, dw) = gem.expert_product(x, w, offset), gem.expert_product_backward(dy, x, w, offset)
    for got, want in ((y, clean[0]), (dx, clean[1])):
        assert torch.equal(got[:70], want[:70]) and torch.equal(got[200:], want[200:]) and torch.isnan(got[70:200]).all()
    assert torch.equal(dw[[0, 1, 3]], clean[2][[0, 1, 3]]) and torch.isnan(dw[2]).all()


@pytest.mark.parametrize("d_in,d_out", [(64, 64), (65, 66)])
def test_nothing_to_do(d_in, d_out):
    w = weights(3, d_in, d_out, BF16, 1)
    offset = torch.zeros(4, dtype=torch.int32, device="cuda")
    x, dy = torch.empty(0, d_in, dtype=BF16, device="cuda"), torch.empty(0, d_out, dtype=BF16, device="cuda")
    assert gem.expert_product(x, w, offset).shape == (0, d_out)
    dx, dw = gem.expert_product_backward(dy, x, w, offset)
    assert dx.shape == (0, d_in) and (dw == 0).all()
    # places without rows of x behind them
    row = torch.full((5,), -1, dtype=torch.int32, device="cuda")
    offset = torch.tensor([0, 2, 2, 5], dtype=torch.int32, device="cuda")
    assert (gem.expert_product(x, w, offset, row) == 0).all()
    assert (gem.expert_product_backward(matrix(5, d_out, BF16, 2), x, w, offset, row)[1] == 0).all()


def test_float32_of_any_size():
    """Columns from the smallest to the largest numbers: what is split into three parts is exact there too."""
    x, w = matrix(90, 64, F32, 1), weights(2, 64, 72, F32, 2)
    x *= torch.exp2(torch.arange(90, device="cuda") * 2.0 - 100)[:, None]
    offset = torch.tensor([0, 40, 90], dtype=torch.int32, device="cuda")
    y = gem.expert_product(x, w, offset)
    assert_within(y, *ref.product(x, w, offset))
    one = torch.eye(64, device="cuda").expand(2, 64, 64).contiguous()
    big = torch.tensor([3.4028235e38, -3.4028235e38, 3.39e38, 1.5 * 2.0 ** -120], dtype=torch.float64).float().cuda().repeat(90, 16)
    got = gem.expert_product(big, one, offset)
    assert ((got.double() - big.double()).abs() <= 4 * 2.0 ** -24 * big.double().abs()).all()
    x[7, 3] = float("inf")
    y = gem.expert_product(x, w, offset)
    assert not torch.isfinite(y[7]).any() and torch.isfinite(torch.cat([y[:7], y[8:]])).all()


def test_outputs_given_and_parts_of_wider_ones():
    offset = split(300, 4, 1)
    x, w = matrix(300, 128, BF16, 1), weights(4, 128, 100, BF16, 2)
    for dtype in (BF16, F32):
        x, w = x.to(dtype), w.to(dtype)
        outputs_given(x, w, offset, dtype)


def outputs_given(x, w, offset, dtype):
    want = gem.expert_product(x, w, offset)
    for left, wide in ((8, 128), (5, 131)):
        whole = torch.full((300, wide), 7.0, dtype=dtype, device="cuda")
        out = whole[:, left:left + 100]
        assert gem.expert_product(x, w, offset, out=out) is out
        assert torch.equal(out, want) and (whole[:, :left] == 7).all() and (whole[:, left + 100:] == 7).all()


def test_parts_of_the_gradient_and_its_repetition():
    x, w, dy, offset, row, y, dx, dw = check(900, 6, 136, 200, BF16, gather=200)
    assert torch.equal(gem.expert_product_backward(dy, x, w, offset, row, need_dw=False)[0], dx)
    assert torch.equal(gem.expert_product_backward(dy, x, w, offset, row, need_dx=False)[1], dw)
    assert gem.expert_product_backward(dy, x, w, offset, row, need_dx=False, need_dw=False) == (None, None)
    for _ in range(3):
        assert torch.equal(gem.expert_product(x, w, offset, row), y)
        again = gem.expert_product_backward(dy, x, w, offset, row)
        assert torch.equal(again[0], dx) and torch.equal(again[1], dw)


def test_weights_shared_by_all_experts():
    w = weights(1, 64, 72, BF16, 2).expand(3, 64, 72)
    offset = split(100, 3, 1)
    x = matrix(100, 64, BF16, 1)
    assert_within(gem.expert_product(x, w, offset), *ref.product(x, w, offset))


def test_one_row_for_all():
    x = matrix(1, 72, BF16, 1).expand(50, 72)
    w, offset = weights(2, 72, 64, BF16, 2), split(50, 2, 3)
    assert_within(gem.expert_product(x, w, offset), *ref.product(x, w, offset))


def test_streams_and_graphs():
    x, w, dy, offset, row, y, dx, dw = check(700, 5, 256, 128, BF16, gather=300)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gem.expert_product(x, w, offset, row, stream=side)
    side.synchronize()
    assert torch.equal(got, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = gem.expert_product(x, w, offset, row), *gem.expert_product_backward(dy, x, w, offset, row)
    x.mul_(2)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(outs[0], gem.expert_product(x, w, offset, row)) and torch.equal(outs[1], dx)


def slots(n, k, places, seed, left_out=0.2):
    """Places of n x k slots, each at most once, -1 for some, and the used places first."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    out = torch.rand(n * k, generator=gen, device="cuda") < left_out
    used = int((~out).sum())
    place = torch.full((n * k,), -1, dtype=torch.int32, device="cuda")
    place[~out] = torch.randperm(used, generator=gen, device="cuda").int()
    return place.view(n, k), used


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=name)
@pytest.mark.parametrize("weighted", [True, False])
@pytest.mark.parametrize("n,k,d,pad,first", [(1, 1, 1, 0, 0), (1, 8, 768, 0, 0), (7, 2, 33, 0, 0), (40, 4, 1000, 0, 0), (33, 9, 257, 3, 1), (2000, 3, 96, 8, 8), (3, 32, 4099, 0, 0),
                                             (1500, 2, 1024, 0, 4)])
def test_combine(n, k, d, pad, first, weighted, dtype):
    place, used = slots(n, k, n * k, n + d)
    offset = torch.tensor([0, used // 2, used], dtype=torch.int32, device="cuda")
    y, dout = matrix(n * k, d, dtype, 1, pad, first), matrix(n, d, dtype, 2, pad, first)
    weight = torch.rand(n, k, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)) - 0.3 if weighted else None
    assert_within(gem.combine(y, place, weight), *ref.combine(y, place, weight), "out")
    dy, dw = gem.combine_backward(dout, y, place, weight, offset)
    (wy, by), (ww, bw) = ref.combine_grad(dout, y, place, weight)
    assert_within(dy, wy, by, "dy")
    assert_within(dw, ww, bw, "dweight")
    assert (dy[used:] == 0).all()
    assert torch.equal(gem.combine_backward(dout, y, place, weight, offset, need_dy=False)[1], dw)
    assert torch.equal(gem.combine_backward(dout, y, place, weight, offset, need_dweight=False)[0], dy)


def test_combine_where_nothing_is():
    y = matrix(4, 72, BF16, 1)
    place = torch.full((3, 2), -1, dtype=torch.int32, device="cuda")
    place[1, 0], place[2, 1] = 9, 2
    weight = torch.ones(3, 2, device="cuda")
    weight[0, 1] = float("nan")
    out = gem.combine(y, place, weight)
    assert torch.isnan(out[0]).all() and (out[1] == 0).all() and torch.equal(out[2], y[2])
    none = torch.empty(0, 2, dtype=torch.int32, device="cuda")
    assert gem.combine(y, none).shape == (0, 72)
    offset = torch.tensor([0, 0], dtype=torch.int32, device="cuda")
    dy, dw = gem.combine_backward(torch.empty(0, 72, dtype=BF16, device="cuda"), y, none, None, offset)
    assert (dy == 0).all() and dw.shape == (0, 2)


def test_the_sum_over_a_rows_places():
    """The gradient of a gathered row is combine without weights."""
    gen = torch.Generator(device="cuda").manual_seed(0)
    r = gem.route(torch.randn(300, 8, generator=gen, device="cuda"), 3)
    dplace = matrix(900, 96, BF16, 4)
    want = torch.zeros(300, 96, dtype=torch.float64, device="cuda").index_add_(0, r.row.long(), dplace.double())
    bound = 5 * 2.0 ** -24 * torch.zeros_like(want).index_add_(0, r.row.long(), dplace.double().abs()) + 2.0 ** -8 * want.abs() + 1e-30
    assert_within(gem.combine(dplace, r.place), want, bound)
