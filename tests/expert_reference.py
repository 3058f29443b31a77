"""The expert layer's definitions in 64 bits, and how far a kernel that works in 32 bits may be from them.

U = 2^-24 is the rounding of one FP32 operation, STEP half a step of the type that a result is stored in.  The bounds add up
what each operation may be off by, element by element; the tensor cores' sums are taken to lose a whole step of 2^-23 of the
terms' magnitudes at each term, whatever their order."""
import math

import torch

from training_reference import U, store

INF = math.inf


def route(z, k, score="softmax", bias=None, groups=1, kept=None, best=1, renorm=True, scale=1.0):
    """(expert, weight, offset, row, place, bound of the weights)"""
    n, e = z.shape
    kept = groups if kept is None else kept
    z = z.double()
    bad = torch.isnan(z).any(1) | ((z == INF).any(1) if score == "softmax" else False)
    z = z.masked_fill(bad[:, None], -INF)
    none = z == -INF
    top = z.max(1, keepdim=True).values
    if score == "softmax":
        x = (z - top.clamp(min=-1e300)).exp()
        s = x / x.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        s = 1 / (1 + (-z).exp())
    c = z if bias is None else torch.where(none, z, s + bias.double())
    if groups > 1:
        by = c if bias is not None or best == 1 else torch.where(none, z, s)
        v = by.view(n, groups, -1).sort(dim=2, descending=True).values[:, :, :best]
        v = v[:, :, 0] + v[:, :, 1:].masked_fill(v[:, :, 1:] == -INF, 0).sum(2)
        at = v.sort(dim=1, descending=True, stable=True).indices[:, :kept]
        stays = torch.zeros(n, groups, dtype=torch.bool, device=z.device).scatter_(1, at, True)
        c = torch.where(stays[:, :, None], c.reshape(n, groups, -1), -INF).reshape(n, e)
    got = c.sort(dim=1, descending=True, stable=True)
    has = got.values[:, :k] != -INF
    expert = torch.where(has, got.indices[:, :k], -1)
    at = expert.clamp(min=0)
    zc = torch.where(has, z.gather(1, at), -INF)
    if renorm:
        log = zc if score == "softmax" else torch.where(has, torch.nn.functional.logsigmoid(zc), -INF)
        first = log.max(1, keepdim=True).values.clamp(min=-1e300)
        x = (log - first).exp()
        w = x / x.sum(1, keepdim=True).clamp(min=1e-300)
        # exp to 2 units and its argument's rounding (of the logs themselves too), a sum of k, a quotient, the scale
        far = (first - log).clamp(max=200.0) + (0 if score == "softmax" else log.abs().clamp(max=200.0) + 2)
        rel = (far + far.max(1, keepdim=True).values + 24) * 2 * U
    else:
        w = torch.where(has, s.gather(1, at), 0.0)
        far = (top - zc).clamp(max=200.0) if score == "softmax" else zc.abs().clamp(max=200.0)
        rel = (far.nan_to_num(0.0, 0.0, 0.0) + 40) * 2 * U
    w = torch.where(has, w, 0.0) * scale
    rel = torch.where(has, rel, 0.0)
    w = torch.where(bad[:, None], math.nan, w)
    return (expert.int(), w, *plan(expert, e), rel * w.abs().nan_to_num(0.0) + 2.0 ** -126)


def plan(expert, experts):
    """(offset, row, place) by counting."""
    n, k = expert.shape
    flat = expert.reshape(-1).tolist()
    lists = [[i for i, e in enumerate(flat) if e == x] for x in range(experts)] if n * k <= 4096 else None
    if lists is None:
        e = expert.reshape(-1).long()
        key = torch.where(e < 0, experts, e)
        order = key.sort(stable=True).indices
        count = torch.bincount(key, minlength=experts + 1)[:experts]
    else:
        order = torch.tensor([i for x in lists for i in x], dtype=torch.int64, device=expert.device)
        count = torch.tensor([len(x) for x in lists], device=expert.device)
    offset = torch.cat([count.new_zeros(1), count.cumsum(0)])
    used = int(offset[-1])
    place = torch.full((n * k,), -1, dtype=torch.int64, device=expert.device)
    place[order[:used]] = torch.arange(used, device=expert.device)
    row = torch.full((n * k,), -1, dtype=torch.int64, device=expert.device)
    row[:used] = order[:used] // k
    return offset.int(), row.int(), place.int().view(n, k)


def route_grad(dweight, z, expert, score, renorm, scale):
    """(dlogits, bound)"""
    dtype, z = z.dtype, z.double()
    has, at = expert >= 0, expert.clamp(min=0).long()
    live = has.any(1, keepdim=True)
    x = z.masked_fill(~live & (z == -INF).all(1, keepdim=True), 0.0).requires_grad_(True)
    if score == "softmax":
        s = torch.softmax(x, 1)
        log = torch.log_softmax(x, 1)
    else:
        s, log = torch.sigmoid(x), torch.nn.functional.logsigmoid(x)
    chosen = torch.where(has, log.gather(1, at), -INF)
    if renorm:
        if score == "softmax":
            chosen = torch.where(has, x.gather(1, at), -INF)
        w = torch.softmax(torch.where(live, chosen, 0.0), 1)
    else:
        w = torch.where(has, s.gather(1, at), 0.0)
    v = torch.where(has, dweight.double() * scale, 0.0)
    loss = (torch.where(has, w, 0.0) * v).sum()
    grad = torch.autograd.grad(loss, x)[0].nan_to_num(0.0)
    # every share is p (v - t) r with p off by its exponential and its sum, t by a sum of k products
    spread = (z.masked_fill(z == -INF, 0).abs().amax(1, keepdim=True) * 2).clamp(max=200.0)
    rel = (2 * spread + 80) * 2 * U                      # (the 64-bit values' own rounding is far below)
    p = torch.where(has, w, 0.0).detach()
    share = p * (v.abs() + (p * v.abs()).sum(1, keepdim=True))
    bound = torch.zeros_like(grad).scatter_add_(1, at, torch.where(has, share, 0.0))
    if score == "softmax" and not renorm:
        bound = bound + s.detach().nan_to_num(0.0) * (p * v.abs()).sum(1, keepdim=True)
    return grad, bound * rel + store(grad, dtype) + 2.0 ** -126


def ranges(offset, places):
    """The experts' (first, end), wild offsets cut to what is possible."""
    reached, out = 0, []
    for v in [0] + offset.tolist()[1:]:
        reached = max(reached, min(max(v, 0), places))
        out.append(reached)
    return list(zip(out[:-1], out[1:]))


def rows_of(x, row, a, b):
    if row is None:
        return x[a:b].double()
    r = row[a:b].long()
    there = (r >= 0) & (r < x.shape[0])
    return torch.where(there[:, None], x[r.clamp(0, max(0, x.shape[0] - 1))].double(), 0.0) if x.shape[0] else torch.zeros(b - a, x.shape[1], dtype=torch.float64, device=x.device)


def off_by_sum(terms, magnitude):
    return (terms + 32) * 2 * U * magnitude


def product(x, w, offset, row=None):
    """(y, bound)"""
    places = x.shape[0] if row is None else row.shape[0]
    y = torch.zeros(places, w.shape[2], dtype=torch.float64, device=x.device)
    mag = torch.zeros_like(y)
    for e, (a, b) in enumerate(ranges(offset, places)):
        v, m = rows_of(x, row, a, b), w[e].double()
        y[a:b], mag[a:b] = v @ m, v.abs() @ m.abs()
    return y, off_by_sum(x.shape[1], mag) + store(y, x.dtype)


def product_grad(dy, x, w, offset, row=None):
    """((dx, bound), (dw, bound))"""
    places = dy.shape[0]
    dx = torch.zeros(places, w.shape[1], dtype=torch.float64, device=x.device)
    dw = torch.zeros(w.shape, dtype=torch.float64, device=x.device)
    mx, bw = torch.zeros_like(dx), torch.zeros_like(dw)
    for e, (a, b) in enumerate(ranges(offset, places)):
        v, g, m = rows_of(x, row, a, b), dy[a:b].double(), w[e].double()
        dx[a:b], mx[a:b] = g @ m.t(), g.abs() @ m.abs().t()
        dw[e], bw[e] = v.t() @ g, off_by_sum(b - a, v.abs().t() @ g.abs())
    return (dx, off_by_sum(w.shape[2], mx) + store(dx, x.dtype)), (dw, bw + store(dw, w.dtype))


def combine(y, place, weight=None):
    n, k = place.shape
    has = (place >= 0) & (place < y.shape[0])
    v = y.double()[place.clamp(0, y.shape[0] - 1).long()]
    w = torch.ones(n, k, dtype=torch.float64, device=y.device) if weight is None else weight.double()
    t = torch.where(has[:, :, None], w[:, :, None] * v, 0.0)
    out = t.sum(1)
    return out, (k + 2) * U * t.abs().sum(1) + store(out, y.dtype)


def combine_grad(dout, y, place, weight):
    """((dy, bound), (dweight, bound))"""
    n, k = place.shape
    has, at = place >= 0, place.clamp(min=0).long()
    w = torch.ones(n, k, dtype=torch.float64, device=y.device) if weight is None else weight.double()
    g, d = dout.double(), y.shape[1]
    t = y.double()[at] * g[:, None, :]
    dw = torch.where(has, t.sum(2), 0.0)
    dy = torch.zeros(y.shape, dtype=torch.float64, device=y.device)
    dy[at[has]] = (w[:, :, None] * g[:, None, :])[has]
    # a lane adds d / 32 products and seven more of its last vector, then 5 steps of a warp and 8 of a block
    return (dy, 2 * U * dy.abs() + store(dy, y.dtype)), (dw, torch.where(has, (d / 32 + 24) * U * t.abs().sum(2), 0.0) + 2.0 ** -126)


def restored(z):
    """What the 8 bits of each 32 columns stand for, by whole numbers: z as m 2^-149 m whole."""
    n, d = z.shape
    v = torch.nn.functional.pad(z.float(), (0, -d % 32)).view(n, -1, 32).double()
    top = v.abs().amax(2, keepdim=True)
    e = torch.full_like(top, -127.0)
    for _ in range(256):                                 # the smallest e: step by step
        e = torch.where(top >= 127.5 * torch.exp2(e), e + 1, e)
    e = e.clamp(max=9.0 if z.dtype == torch.float16 else 121.0)
    q = torch.round(v * torch.exp2(-e)).clamp(-127, 127)
    q = torch.where(torch.isfinite(top), q * torch.exp2(e), math.nan)
    return q.view(n, -1)[:, :d]


def act(z, kind, dtype):
    """(value, slope, their bounds) at 64-bit z."""
    e = (6 + z.abs().clamp(max=200.0)) * (2 * U if dtype == torch.float32 else 8 * U)       # of the exponential, relative
    if kind == "silu":
        p = torch.sigmoid(z)
        y, s = z * p, p * (1 + z * (1 - p))
        return y, s, (e + 8 * U) * y.abs(), (e + 8 * U) * (p + 2 * (z * p).abs())
    if kind == "gelu":
        p, phi = 0.5 * torch.erfc(-z * math.sqrt(0.5)), (-0.5 * z * z).exp() / math.sqrt(2 * math.pi)
        rel = (16 + 2 * z * z) * 2 * U                   # erfc to 6 units, and its argument's rounding times 1 + z^2
        ef = (8 + z * z) * (2 * U if dtype == torch.float32 else 8 * U)
        return z * p, p + z * phi, rel * (z * p).abs() + 2.0 ** -126, rel * p + ef * (z * phi).abs() + 2.0 ** -126
    if kind == "tanh":
        y = torch.tanh(z)
        return y, 1 - y * y, 6 * U * y.abs(), 16 * U * torch.ones_like(y)
    return z, torch.ones_like(z), 0 * z, 0 * z


def activation(z, kind, gated):
    """(y, bound)"""
    if gated:
        g, u = z.double().chunk(2, 1)
        y, _, by, _ = act(g, kind, z.dtype)
        return y * u, (by + 2 * U * y.abs()) * u.abs() + store(y * u, z.dtype)
    y, _, by, _ = act(z.double(), kind, z.dtype)
    return y, by + store(y, z.dtype)


def activation_grad(dy, v, kind, gated, dtype):
    """(dz, bound) at the 64-bit values v of z."""
    d = dy.double()
    if gated:
        g, u = v.chunk(2, 1)
        y, s, by, bs = act(g, kind, dtype)
        dz = torch.cat([d * u * s, d * y], 1)
        b = torch.cat([(d * u).abs() * (bs + 3 * U * s.abs()), d.abs() * (by + 2 * U * y.abs())], 1)
    else:
        _, s, _, bs = act(v, kind, dtype)
        dz, b = d * s, d.abs() * (bs + 2 * U * s.abs())
    return dz, b + store(dz, dtype)
