"""Routing rows to experts, and its gradient, against the definition in 64 bits."""
import math

import pytest
import torch

import expert_reference as ref
import paper_2609_36074_b200 as gem
from training_reference import assert_within

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
INF, NAN = math.inf, math.nan


def name(t):
    return {F32: "f32", F16: "f16", BF16: "bf16"}.get(t, str(t))


def logits(n, e, dtype=F32, seed=0, pad=0, spread=1.5):
    gen = torch.Generator(device="cuda").manual_seed(seed + 3 * n + e)
    whole = torch.full((n, e + pad), NAN, dtype=dtype, device="cuda")
    z = whole[:, :e]
    z.copy_(torch.randn(n, e, generator=gen, device="cuda") * spread)
    return z


def biases(e, seed=0):
    return torch.randn(e, generator=torch.Generator(device="cuda").manual_seed(seed + e), device="cuda") * 0.05


def check(z, k, score="softmax", bias=None, groups=1, kept=None, best=1, renorm=True, scale=1.0):
    got = gem.route(z, k, score, bias, groups, kept, best, renorm, scale)
    want = ref.route(z, k, score, bias, groups, kept, best, renorm, scale)
    assert torch.equal(got.expert, want[0])
    for g, v, what in zip(got[2:], want[2:5], ("offset", "row", "place")):
        assert torch.equal(g, v), what
    nan = torch.isnan(want[1])
    assert torch.equal(torch.isnan(got.weight), nan)
    assert_within(got.weight[~nan], want[1][~nan], want[5][~nan], "weight")
    v = torch.randn(got.weight.shape, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    if not nan.any():
        grad, bound = ref.route_grad(v, z, got.expert, score, renorm, scale)
        assert_within(gem.route_backward(v, z, got.expert, score, renorm, scale), grad, bound, "dlogits")
    return got


@pytest.mark.parametrize("renorm", [True, False], ids=["renormalized", "as they are"])
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=name)
@pytest.mark.parametrize("n,e,k", [(1, 1, 1), (1, 8, 2), (3, 2, 2), (64, 31, 4), (65, 32, 32), (100, 33, 5), (700, 64, 4), (300, 65, 7), (300, 128, 8), (90, 129, 6), (50, 256, 8),
                                   (40, 257, 3), (70, 512, 8)])
def test_choice(n, e, k, dtype, score, renorm):
    z = logits(n, e, dtype)
    check(z, k, score, renorm=renorm, scale=2.5)
    check(z, k, score, biases(e), renorm=renorm)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [True, False], ids=["biased", "plain"])
@pytest.mark.parametrize("best", [1, 2])
@pytest.mark.parametrize("e,groups,kept,k", [(8, 2, 1, 3), (64, 8, 3, 6), (96, 32, 5, 9), (30, 6, 2, 10), (256, 4, 2, 8), (32, 32, 4, 4), (512, 16, 4, 8)])
def test_groups(e, groups, kept, k, best, biased, score):
    for dtype in (F32, BF16):
        check(logits(200, e, dtype), k, score, biases(e) if biased else None, groups, kept, best)


@pytest.mark.parametrize("n", [1, 2, 15, 16, 17, 63, 64, 65, 1000, 4737, 30001])
def test_row_counts(n):
    check(logits(n, 64), 4)
    check(logits(n, 20, BF16, pad=3), 2, "sigmoid", biases(20))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [True, False], ids=["biased", "plain"])
def test_ties_go_to_the_lowest_index(score, biased):
    z = logits(500, 96, BF16, spread=0.02).float().mul(64).round().div(64)         # a handful of values
    bias = torch.zeros(96, device="cuda") if biased else None
    got = check(z, 8, score, bias)
    check(z, 6, score, bias, 8, 3, 2)
    check(z, 6, score, bias, 8, 3, 1)
    assert (torch.zeros(9, 40, device="cuda") == 0).all()
    same = check(torch.zeros(9, 40, device="cuda"), 5, score, None)
    assert torch.equal(same.expert, torch.arange(5, device="cuda", dtype=torch.int32).expand(9, 5))
    assert got.expert.shape == (500, 8)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_scores_that_32_bits_do_not_tell_apart(score):
    """Biases set so that the scores of half the experts are a few 2^-30 from one another."""
    z = logits(400, 64, F32, spread=1.0)
    z[1:] = z[0]
    gen = torch.Generator(device="cuda").manual_seed(5)
    z[:, ::2] += torch.randn(400, 32, generator=gen, device="cuda") * 1e-7
    d = z[0].double()
    s = torch.softmax(d, 0) if score == "softmax" else torch.sigmoid(d)
    bias = (0.75 - s).float()
    check(z, 8, score, bias)
    check(z, 8, score, bias, 8, 4, 2)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("k,equals", [(1, 2), (2, 3), (4, 5), (7, 9), (9, 12)])
@pytest.mark.parametrize("e", [16, 40, 300])
def test_equals_at_the_border_before_a_larger_one(e, k, equals, score):
    """More equals than are chosen, and behind them one that 32 bits do not tell from them and that 64 bits do."""
    low = 14.0 if score == "sigmoid" else -17.0          # scores of about 1 and 0, apart by some 2^-26
    step = 0.125
    z = torch.full((60, e), -30.0, device="cuda")
    for i in range(60):
        z[i, :equals] = low
        z[i, equals + i % (e - equals)] = low + (step if i % 3 else -step)
        z[i, equals + (i + 1) % (e - equals)] = low + (2 * step if i % 5 else 0.0)
    bias = torch.full((e,), 0.125, device="cuda")
    if score == "softmax":
        z[:, e - 1], bias[e - 1] = 0.0, -0.5             # the largest score, chosen by none
    for dtype in (F32, F16, BF16):
        check(z.to(dtype), k, score, bias)
        check(z.to(dtype), k, score, bias, 4, 4, 2)
    near = z.clone()                                     # logits apart in their last bits, without a bias
    near[:, :equals] = 1.0
    for i in range(60):
        near[i, equals + i % (e - equals)] = 1.0 + (2.0 ** -22 if i % 3 else -(2.0 ** -22))
    check(near, k, score)


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_rows_of_one_score(score):
    for e, k in ((16, 1), (40, 7), (300, 9)):
        z = torch.full((500, e), 0.25, device="cuda")
        got = check(z, k, score, torch.full((e,), 0.125, device="cuda"))
        assert torch.equal(got.expert, torch.arange(k, device="cuda", dtype=torch.int32).expand(500, k))


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("e", [12, 40, 128, 300])
def test_biases_of_any_size(e, score):
    """Biases beyond the scores, beyond the keys' range, of both signs, and experts put out of reach."""
    z = logits(120, e)
    for scale in (0.5, 3.0, 40.0, 1e6):
        check(z, min(6, e), score, biases(e, 3) * 20 * scale)
    out = biases(e, 4)
    out[::3] = -1e9
    check(z, 4, score, out)
    check(z, e // 2 + 1 if e < 60 else 9, score, out)
    out[1], out[2] = INF, -INF
    check(z, 4, score, out)
    out[:] = 0.25
    check(z, 4, score, out, 4, 2, 2)


def test_a_bias_that_is_not_a_number():
    z, bias = logits(20, 16), biases(16)
    bias[3] = NAN
    r = gem.route(z, 2, "sigmoid", bias)
    assert (r.expert == -1).all() and torch.isnan(r.weight).all() and r.offset.sum() == 0


def test_two_streams_at_once():
    """Two plans and two products at a time, each on a stream of its own."""
    z = [logits(3000, 32, seed=i) for i in range(2)]
    x = torch.randn(3000, 96, device="cuda").bfloat16()
    w = torch.randn(32, 96, 64, device="cuda").bfloat16()
    want = [gem.route(v, 4) for v in z]
    y = [gem.expert_product(x, w, r.offset, r.row) for r in want]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in z]
    for _ in range(10):
        got = []
        for v, s in zip(z, streams):
            with torch.cuda.stream(s):
                r = gem.route(v, 4)
                got.append((r, gem.expert_product(x, w, r.offset, r.row)))
        torch.cuda.synchronize()
        for (r, p), a, b in zip(got, want, y):
            assert all(torch.equal(u, v) for u, v in zip(r, a)) and torch.equal(p, b)


def test_saturated_scores():
    z = logits(300, 32, F32, spread=30.0)
    check(z, 4, "sigmoid", biases(32))
    check(z, 4, "softmax", biases(32))
    check(z, 4, "sigmoid")
    check(z, 4, "softmax")


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("biased", [True, False], ids=["biased", "plain"])
@pytest.mark.parametrize("groups,kept,best", [(1, 1, 1), (4, 2, 2), (4, 2, 1)])
def test_experts_left_out(groups, kept, best, biased, score):
    z = logits(200, 16)
    gen = torch.Generator(device="cuda").manual_seed(2)
    z[torch.rand(z.shape, generator=gen, device="cuda") < 0.6] = -INF
    z[3] = z[77] = -INF
    z[9, 1:] = -INF
    z[10] = torch.finfo(F32).min
    z[11, ::2] = torch.finfo(F32).min
    bias = biases(16) if biased else None
    got = check(z, 5, score, bias, groups, kept, best)
    check(z, 5, score, bias, groups, kept, best, renorm=False)
    assert (got.expert[3] == -1).all() and (got.weight[3] == 0).all() and (got.place[3] == -1).all()
    assert (got.expert[9] >= 0).sum() == (z[9, 0] > -INF)
    if biased:
        bias[4] = -INF
        assert not (gem.route(z, 5, score, bias, groups, kept, best).expert == 4).any()


@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_rows_that_are_not_numbers(score):
    z = logits(100, 20)
    z[5, 7], z[6, 0], z[50, 19] = NAN, INF, -INF
    got = check(z, 4, score)
    assert (got.expert[5] == -1).all() and torch.isnan(got.weight[5]).all()
    if score == "softmax":
        assert (got.expert[6] == -1).all() and torch.isnan(got.weight[6]).all()
    else:
        assert got.expert[6, 0] == 0
    v = torch.ones(100, 4, device="cuda")
    chosen = torch.arange(4, device="cuda", dtype=torch.int32).expand(100, 4).contiguous()
    d = gem.route_backward(v, z, chosen + 5, score, renormalize=score == "sigmoid")
    assert torch.isnan(d[5]).any() and torch.isfinite(d[7:]).all() and torch.isfinite(d[:5]).all()


def test_gradient_of_slots_that_are_not_there():
    z = logits(50, 12)
    r = gem.route(z, 3)
    e = r.expert.clone()
    e[4, 1] = -1
    e[5] = -1
    e[6, 0] = 40                                  # no such expert
    v = torch.randn(50, 3, device="cuda")
    v[4, 1] = v[5, 0] = v[6, 0] = NAN
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            d = gem.route_backward(v, z, e, score, renorm)
            clean = torch.where((e < 0) | (e >= 12), -1, e)
            grad, bound = ref.route_grad(v.nan_to_num(0.0), z, clean, score, renorm, 1.0)
            assert_within(d, grad, bound, f"{score} {renorm}")
            assert (d[5] == 0).all()


@pytest.mark.parametrize("e,k", [(8, 2), (40, 4), (300, 6), (20, 9)])
def test_gradient_of_an_expert_named_twice_is_the_sum(e, k):
    z = logits(60, e)
    gen = torch.Generator(device="cuda").manual_seed(k)
    twice = torch.randint(0, max(2, k - 1), (60, k), generator=gen, device="cuda", dtype=torch.int32)
    v = torch.randn(60, k, generator=gen, device="cuda")
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            grad, bound = ref.route_grad(v, z, twice, score, renorm, 1.0)
            assert_within(gem.route_backward(v, z, twice, score, renorm), grad, bound, f"{score} {renorm}")


def test_gradient_against_differences():
    z = logits(6, 10, F32).double()
    r = gem.route(z.float(), 3, "softmax")
    v = torch.randn(6, 3, device="cuda", dtype=torch.float64, generator=torch.Generator(device="cuda").manual_seed(1))
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            def loss(x):
                s = torch.softmax(x, 1) if score == "softmax" else torch.sigmoid(x)
                w = s.gather(1, r.expert.long())
                return ((w / w.sum(1, keepdim=True) if renorm else w) * v).sum()
            d = gem.route_backward(v.float(), z.float(), r.expert, score, renorm)
            h = 1e-5
            for i in range(6):
                for j in range(0, 10, 3):
                    a, b = z.clone(), z.clone()
                    a[i, j] += h
                    b[i, j] -= h
                    # the difference is off by h^2 times the third derivative (at most 6 |v|), the rest is 32-bit rounding
                    assert abs(((loss(a) - loss(b)) / (2 * h)).item() - d[i, j].item()) <= 6 * h * h * v[i].abs().sum().item() + 1e-5


@pytest.mark.parametrize("dtype", [F32, BF16], ids=name)
def test_gradients_next_to_the_smallest_numbers(dtype):
    z = torch.linspace(-95.0, 0.0, 64, device="cuda").to(dtype).expand(20, 64).contiguous()
    chosen = torch.tensor([[0, 5, 9, 63]], dtype=torch.int32, device="cuda").expand(20, 4).contiguous()
    v = logits(20, 4, F32, 3) * 40
    for score in ("softmax", "sigmoid"):
        for renorm in (True, False):
            grad, bound = ref.route_grad(v, z, chosen, score, renorm, 1.0)
            assert_within(gem.route_backward(v, z, chosen, score, renorm), grad, bound, f"{score} {renorm}")


def test_nothing_to_route_and_large_plans():
    r = gem.route(torch.empty(0, 8, device="cuda"), 2)
    assert r.offset.tolist() == [0] * 9 and r.row.numel() == 0
    assert gem.route_backward(torch.empty(0, 2, device="cuda"), torch.empty(0, 8, device="cuda"), r.expert).shape == (0, 8)
    check(logits(70000, 8, BF16), 3)
    check(logits(20000, 512, BF16), 16)


def test_repetition_streams_and_graphs():
    z, bias = logits(5000, 64), biases(64)
    want = check(z, 6, "sigmoid", bias, 8, 3, 2)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gem.route(z, 6, "sigmoid", bias, 8, 3, 2, stream=side)
    side.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        outs = gem.route(z, 6, "sigmoid", bias, 8, 3, 2)
        d = gem.route_backward(outs.weight, z, outs.expert, "sigmoid")
    z.copy_(logits(5000, 64, seed=9))
    graph.replay()
    torch.cuda.synchronize()
    again = gem.route(z, 6, "sigmoid", bias, 8, 3, 2)
    assert all(torch.equal(a, b) for a, b in zip(outs, again))
    assert torch.equal(d, gem.route_backward(again.weight, z, again.expert, "sigmoid"))
