"""Activations with 8-bit checkpoints, there and back, against their definitions in 64 bits."""
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


def matrix(n, d, dtype, seed, pad=0, first=0, scale=1.0):
    gen = torch.Generator(device="cuda").manual_seed(seed)
    flat = torch.full((n * (d + pad) + first + 8,), NAN, dtype=dtype, device="cuda")
    m = flat[first:first + n * (d + pad)].view(n, d + pad)[:, :d]
    m.copy_(torch.randn(n, d, generator=gen, device="cuda") * scale * torch.exp(torch.randn(d, generator=gen, device="cuda")))
    return m


def check(z, kind, gated, dy):
    y, saved = gem.activation(z, kind, gated)
    d = dy.shape[1]
    assert_within(y, *ref.activation(z, kind, gated), "y")
    halves = [z[:, :d], z[:, d:]] if gated else [z]
    v = torch.cat([ref.restored(h) for h in halves], 1)
    dz, again = gem.activation_backward(dy, saved, kind, gated, need_y=True)
    assert dz.shape == z.shape and again.shape == dy.shape
    assert_within(dz, *ref.activation_grad(dy, v, kind, gated, z.dtype), "dz")
    assert_within(again, *ref.activation(v.to(z.dtype), kind, gated), "y again")
    dz, again = gem.activation_backward(dy, z, kind, gated, need_y=True)                # from z itself
    assert_within(dz, *ref.activation_grad(dy, z.double(), kind, gated, z.dtype), "dz of z")
    assert torch.equal(again, y)
    return y, saved


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=name)
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("kind", ["silu", "gelu", "tanh", "identity"])
@pytest.mark.parametrize("n,d", [(1, 1), (3, 8), (5, 31), (4, 32), (7, 33), (9, 100), (2, 1000), (33, 264), (3, 2048), (2, 4099), (1500, 40)])
def test_shapes(n, d, kind, gated, dtype):
    check(matrix(n, 2 * d if gated else d, dtype, n + d), kind, gated, matrix(n, d, dtype, 1))


@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
@pytest.mark.parametrize("dtype", [F32, BF16], ids=name)
@pytest.mark.parametrize("pad,first", [(8, 0), (3, 0), (0, 1), (16, 8), (1, 5), (4, 4)])
def test_strides_and_alignment(pad, first, dtype, gated):
    check(matrix(20, 2 * 104 if gated else 104, dtype, 3, pad, first), "silu", gated, matrix(20, 104, dtype, 4, pad, first))


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=name)
@pytest.mark.parametrize("n,d", [(1, 1), (4, 31), (3, 32), (6, 97), (50, 768), (2000, 64), (1, 5000)])
def test_restored(n, d, dtype):
    x = matrix(n, d, dtype, n)
    saved = gem.checkpoint(x)
    assert saved.q.dtype == torch.int8 and saved.q.shape == (n, -(-d // 32) * 32) and saved.scale.shape == (n, -(-d // 32))
    assert (saved.q[:, d:] == 0).all()
    got = gem.restore(saved)
    assert got.dtype == dtype and torch.equal(got.double(), ref.restored(x))
    top = torch.nn.functional.pad(x.double().abs(), (0, -d % 32)).view(n, -1, 32).amax(2, keepdim=True).expand(-1, -1, 32).reshape(n, -1)[:, :d]
    assert ((got.double() - x.double()).abs() <= top / 127.0).all()          # half of 2^e, and 63.75 2^e <= top
    assert torch.equal(gem.restore(gem.checkpoint(got)), got)                 # what 8 bits hold they hold again


def test_borders_of_the_scale():
    """Largest magnitudes at and next to 127.5 2^e, halves of a step, and the ends of the range."""
    v = torch.zeros(40, 32, device="cuda")
    tops = [127.5, 127.49999, 127.50001, 127.0, 128.0, 64.0, 63.75, 63.7499, 255.0, 254.99998, 2.0 ** -126, 2.0 ** -149, 2.0 ** -120, 127.5 * 2.0 ** -127, 127.0 * 2.0 ** -127, torch.finfo(F32).max,
            3.4e38, 2.0 ** 127, 1.0, 0.0]
    for i, t in enumerate(tops):
        v[i, 0], v[20 + i, 31] = t, -t
        v[i, 1:20] = torch.linspace(-1, 1, 19, device="cuda") * t
        v[20 + i, :20] = (torch.arange(20, device="cuda") - 10 + 0.5) * (t / 127)
    v[18, 5:9] = torch.tensor([0.5, 1.5, 2.5, -0.5], device="cuda") / 64
    got = gem.restore(gem.checkpoint(v))
    assert torch.equal(got.double(), ref.restored(v))


@pytest.mark.parametrize("dtype", [F32, F16, BF16], ids=name)
def test_what_is_not_a_number(dtype):
    x = matrix(6, 96, dtype, 1)
    x[1, 40], x[2, 0], x[3, 95], x[4, 33] = NAN, INF, -INF, torch.finfo(dtype).max
    saved = gem.checkpoint(x)
    got, want = gem.restore(saved), ref.restored(x)
    assert torch.equal(torch.isnan(got), torch.isnan(want)) and torch.isnan(got).sum() == 96
    assert torch.equal(got.double().nan_to_num(0.0), want.nan_to_num(0.0))
    assert saved.scale[1, 1] == saved.scale[2, 0] == saved.scale[3, 2] == 255
    y, _ = gem.activation(x, "tanh")
    assert torch.isnan(y[1, 40]) and y[2, 0] == 1 and y[3, 95] == -1 and y[4, 33] == 1


@pytest.mark.parametrize("kind", ["silu", "gelu", "tanh"])
def test_far_from_zero(kind):
    z = torch.tensor([[-1e4, -200.0, -88.0, -40.0, -14.0, -13.0, -6.0, -1e-30, 0.0, -0.0, 1e-30, 6.0, 13.0, 40.0, 88.0, 200.0, 1e4]], device="cuda")
    for dtype in (F32, BF16, F16):
        x = z.to(dtype)
        dy = torch.ones_like(x)
        assert_within(gem.activation(x, kind, checkpoint=False)[0], *ref.activation(x, kind, False), "y")
        dz, _ = gem.activation_backward(dy, x, kind)
        assert_within(dz, *ref.activation_grad(dy, x.double(), kind, False, dtype), "dz")


@pytest.mark.parametrize("kind", ["silu", "gelu", "tanh"])
@pytest.mark.parametrize("gated", [False, True], ids=["plain", "gated"])
def test_gradient_against_differences(kind, gated):
    z = matrix(4, 24, F32, 7).clamp(-5, 5)
    dy = matrix(4, 12 if gated else 24, F32, 8)
    dz, _ = gem.activation_backward(dy, z, kind, gated)

    def loss(v):
        if gated:
            return (ref.act(v[:, :12], kind, F32)[0] * v[:, 12:] * dy.double()).sum()
        return (ref.act(v, kind, F32)[0] * dy.double()).sum()

    h = 1e-4
    for i, j in ((0, 0), (1, 5), (2, 11), (3, 23), (0, 17)):
        a, b = z.double().clone(), z.double().clone()
        a[i, j] += h
        b[i, j] -= h
        # h^2 times a third derivative of at most 2, and 32-bit rounding
        scale = dy.abs().max().item() * max(1.0, z.abs().max().item())
        assert abs(((loss(a) - loss(b)) / (2 * h)).item() - dz[i, j].item()) <= (2 * h * h + 1e-5) * scale


def test_parts_leading_dimensions_and_outputs_given():
    z = matrix(12, 64, BF16, 2).view(3, 4, 64)
    dy = matrix(12, 32, BF16, 3).view(3, 4, 32)
    y, saved = gem.activation(z, "silu", True)
    flat, kept = gem.activation(z.view(12, 64), "silu", True)
    assert y.shape == (3, 4, 32) and torch.equal(y.view(12, 32), flat) and torch.equal(saved.q, kept.q)
    dz, _ = gem.activation_backward(dy, saved, "silu", True)
    assert dz.shape == z.shape
    assert gem.activation(z, "silu", True, checkpoint=False)[1] is None and gem.activation(z, "silu", True, need_y=False)[0] is None
    assert torch.equal(gem.activation(z, "silu", True, need_y=False)[1].q, saved.q)
    alone = gem.activation_backward(None, saved, "silu", True, need_y=True)
    assert alone[0] is None and torch.equal(alone[1], gem.activation_backward(dy, saved, "silu", True, need_y=True)[1])
    assert gem.activation_backward(None, saved, "silu", True) == (None, None)
    whole = torch.full((12, 40), 7.0, dtype=BF16, device="cuda")
    out = whole[:, 3:35]
    assert gem.activation(z.view(12, 64), "silu", True, out=out)[0] is out
    assert torch.equal(out, flat) and (whole[:, :3] == 7).all() and (whole[:, 35:] == 7).all()
    empty = torch.empty(0, 64, dtype=BF16, device="cuda")
    y, saved = gem.activation(empty, "gelu")
    assert y.shape == (0, 64) and gem.activation_backward(y, saved, "gelu", need_y=True)[1].shape == (0, 64) and gem.restore(gem.checkpoint(empty)).shape == (0, 64)


def test_layer_norms_gradient_from_8_bits():
    """The saved input of a layer norm held in 8 bits: its gradient is the one at the restored input."""
    x, dy = matrix(50, 96, F32, 1), matrix(50, 96, F32, 2)
    saved = gem.checkpoint(x)
    _, mean, rstd = gem.layer_norm(x)
    got = gem.layer_norm_backward(dy, gem.restore(saved), mean, rstd)[0]
    assert torch.equal(got, gem.layer_norm_backward(dy, ref.restored(x).float(), mean, rstd)[0])


def test_streams_and_graphs():
    z, dy = matrix(300, 512, BF16, 1), matrix(300, 256, BF16, 2)
    want = gem.activation(z, "silu", True)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    got = gem.activation(z, "silu", True, stream=side)
    side.synchronize()
    assert torch.equal(got[0], want[0]) and torch.equal(got[1].q, want[1].q)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, saved = gem.activation(z, "silu", True)
        dz, again = gem.activation_backward(dy, saved, "silu", True, need_y=True)
    z.mul_(-0.5)
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(y, gem.activation(z, "silu", True)[0])
    assert torch.equal(dz, gem.activation_backward(dy, gem.activation(z, "silu", True)[1], "silu", True)[0])
