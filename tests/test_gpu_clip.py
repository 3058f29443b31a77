"""The norm over many tensors, and clipping, against the definition in 64 bits."""
import math

import pytest
import torch

import paper_2609_36074_b200 as gem
import training_reference as ref

pytestmark = pytest.mark.gpu

F32, F16, BF16 = torch.float32, torch.float16, torch.bfloat16
SIZES = [(1,), (5,), (768,), (100, 768), (1000,), (0,), (8191,), (8192,), (8193,), (3, 5, 7), (), (65537,), (300, 1001)]


def tensors(sizes, kinds, seed=0, scale=0.01):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    return [(torch.randn(s, generator=gen, device="cuda") * scale).to(kinds[i % len(kinds)]) for i, s in enumerate(sizes)]


def check(grads, max_norm, out=None, eps=1e-6):
    keep = [g.clone() for g in grads]
    want, c = ref.clip(keep, max_norm, eps)
    norm = gem.clip_grad_norm(grads, max_norm, out=out, eps=eps)
    assert norm.dtype == F32 and norm.shape == ()
    assert abs(norm.item() - want.item()) <= ref.CLIP_NORM * want.item() + 1e-45
    if out is not None:
        assert all(torch.equal(g, k) for g, k in zip(grads, keep))
    for g, o in zip(keep, grads if out is None else out):
        v = g.double() * c
        ref.assert_within(o, v, v.abs() * ref.CLIP_SCALE + ref.store(v, o.dtype))


@pytest.mark.parametrize("kinds", [(F32,), (F16,), (BF16,), (F32, BF16, F16)], ids=lambda k: "-".join(str(t)[6:] for t in k))
@pytest.mark.parametrize("max_norm", [0.0, 0.05, 1e4])
@pytest.mark.parametrize("out", ["in place", "same", "float32"])
def test_types_and_sizes(kinds, max_norm, out):
    grads = tensors(SIZES, kinds)
    to = None if out == "in place" else [torch.empty_like(g, dtype=F32 if out == "float32" else g.dtype) for g in grads]
    check(grads, max_norm, to)


@pytest.mark.parametrize("size", [1, 2, 7, 8, 9, 255, 256, 2047, 8192, 8200, 16385, 1 << 20, (1 << 22) + 3])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=lambda t: str(t)[6:])
def test_one_tensor(size, dtype):
    check(tensors([(size,)], (dtype,)), 0.5)


@pytest.mark.parametrize("first,to", [(1, 1), (1, 0), (0, 1), (3, 2), (4, 4), (8, 0), (2, 6)])
@pytest.mark.parametrize("kind,okind", [(F32, F32), (BF16, BF16), (BF16, F32), (F16, F32)], ids=str)
def test_alignment(first, to, kind, okind):
    gen = torch.Generator(device="cuda").manual_seed(first)
    n = 20011
    g = torch.randn(n + first, generator=gen, device="cuda").to(kind)[first:]
    whole = torch.full((n + to + 9,), 7.0, device="cuda", dtype=okind)
    check([g], 0.5, [whole[to: to + n]])
    assert (whole[:to] == 7).all() and (whole[to + n:] == 7).all()
    check([g], 0.5)


@pytest.mark.parametrize("count", [1, 63, 64, 65, 999, 1000, 1001, 2503])
def test_many_tensors(count):
    gen = torch.Generator().manual_seed(count)
    sizes = [(int(torch.randint(0, 300, (1,), generator=gen)),) for _ in range(count)]
    sizes[-1] = (20000,)
    check(tensors(sizes, (F32, BF16)), 0.1)


def test_nothing_is_written_when_nothing_is_clipped():
    grads = tensors(SIZES, (F32, BF16))
    keep = [g.clone() for g in grads]
    gem.clip_grad_norm(grads, 1e6)
    assert all(torch.equal(g, k) for g, k in zip(grads, keep))


def test_norm_alone():
    grads = tensors(SIZES, (F32, BF16, F16))
    keep = [g.clone() for g in grads]
    want = ref.clip(grads, 1.0, 0.0)[0].item()
    assert abs(gem.grad_norm(grads).item() - want) <= ref.CLIP_NORM * want
    assert all(torch.equal(g, k) for g, k in zip(grads, keep))


@pytest.mark.parametrize("value", [1e-30, 1e-25, 1e-19, 1e19, 1e25, 1e30])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=lambda t: str(t)[6:])
def test_squares_beyond_the_range_of_32_bits(value, dtype):
    grads = [torch.full((1000,), value, device="cuda").to(dtype), torch.zeros(300, device="cuda", dtype=dtype)]
    want = math.sqrt(1000) * grads[0][0].double().item()
    assert abs(gem.grad_norm(grads).item() - want) <= ref.CLIP_NORM * want
    check(grads, want / 2, eps=0.0)


def test_a_small_share_beside_a_large_one():
    grads = [torch.full((4096,), 1e-18, device="cuda"), torch.full((8,), 1e-15, device="cuda")]
    check(grads, 1e-16, eps=0.0)


def test_zeros():
    grads = [torch.zeros(5000, device="cuda"), torch.zeros(3, device="cuda", dtype=BF16)]
    for max_norm, eps in ((1.0, 1e-6), (1.0, 0.0), (0.0, 0.0)):
        assert gem.clip_grad_norm(grads, max_norm, eps=eps) == 0
        assert all((g == 0).all() for g in grads)


@pytest.mark.parametrize("dtype", [F32, BF16], ids=lambda t: str(t)[6:])
def test_nan_and_infinity(dtype):
    for bad in (float("nan"), float("inf"), -float("inf")):
        grads = tensors([(1000,), (9000,)], (dtype,))
        grads[0][10] = bad
        norm = gem.clip_grad_norm(grads, 1.0)
        if bad != bad:
            assert norm.isnan() and all(g.isnan().all() for g in grads)
        else:
            assert norm == float("inf") and (grads[1] == 0).all() and grads[0][10].isnan()
            assert (torch.cat([grads[0][:10], grads[0][11:]]) == 0).all()


def test_orders_of_dimensions():
    gen = torch.Generator(device="cuda").manual_seed(0)
    g = torch.randn(40, 30, 5, generator=gen, device="cuda").permute(2, 0, 1)
    check([g], 0.5)
    check([g], 0.5, [torch.empty_like(g)])
    check([g], 0.5, [torch.empty_strided(g.shape, g.stride(), device="cuda")])


def test_offsets_beyond_32_bits():
    n = 2 ** 31 + 77
    g = torch.ones(n, dtype=BF16, device="cuda")
    g[-1] = 3.0
    norm = gem.clip_grad_norm([g], math.sqrt(n + 8) / 2, eps=0.0)
    assert abs(norm.item() - math.sqrt(n + 8)) <= ref.CLIP_NORM * math.sqrt(n)
    assert g[-1] == 1.5 and (g[-100:-1] == 0.5).all() and (g[::1048573] == 0.5).all()
    assert g.sum(dtype=torch.float64).item() == (n - 1) * 0.5 + 1.5


def test_same_bits_each_time_and_on_a_side_stream_and_in_a_graph():
    grads = tensors(SIZES, (F32, BF16))
    out = [[torch.empty_like(g) for g in grads] for _ in range(3)]
    norms = [gem.clip_grad_norm(grads, 0.1, out=out[0])]
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    norms.append(gem.clip_grad_norm(grads, 0.1, out=out[1], stream=side))
    torch.cuda.current_stream().wait_stream(side)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        norms.append(gem.clip_grad_norm(grads, 0.1, out=out[2]))
    graph.replay()
    torch.cuda.synchronize()
    for k in (1, 2):
        assert torch.equal(norms[0], norms[k]) and all(torch.equal(a, b) for a, b in zip(out[0], out[k]))


def test_refusals():
    g = torch.randn(4, 64, device="cuda")
    for call in (lambda: gem.clip_grad_norm([], 1.0), lambda: gem.clip_grad_norm([g.double()], 1.0),
                 lambda: gem.clip_grad_norm([g[:, :10]], 1.0), lambda: gem.clip_grad_norm([g.cpu()], 1.0),
                 lambda: gem.clip_grad_norm([g, g.cpu()], 1.0), lambda: gem.clip_grad_norm([g], -1.0),
                 lambda: gem.clip_grad_norm([g], float("nan")), lambda: gem.clip_grad_norm([g], 1.0, eps=-1.0),
                 lambda: gem.clip_grad_norm([g], 1.0, out=[]), lambda: gem.clip_grad_norm([g], 1.0, out=[g.half()]),
                 lambda: gem.clip_grad_norm([g], 1.0, out=[g[:3]]), lambda: gem.clip_grad_norm([g.expand(2, 4, 64)], 1.0),
                 lambda: gem.clip_grad_norm([g.t()], 1.0, out=[torch.empty(64, 4, device="cuda")]),
                 lambda: gem.grad_norm([g.double()])):
        with pytest.raises(ValueError):
            call()
