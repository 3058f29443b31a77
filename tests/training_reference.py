"""The training operators' definitions in 64 bits, and how far a kernel that works in 32 bits may be from them.

u = 2^-24 is the rounding of one FP32 operation.  A sum of m terms in FP32, taken in any tree with at most `seq(m)`
additions in a row, is off by at most seq(m) u times the sum of the terms' magnitudes; seq(m) = 32 + m / 64 covers a
block of 64 or more partial sums and their joining.  Every other operation adds one u of its result, and the store in
`dtype` half a step of that type.  The bounds below add these up, element by element."""
import torch

U = 2.0 ** -24
STEP = {torch.float32: 2.0 ** -24, torch.float16: 2.0 ** -11, torch.bfloat16: 2.0 ** -8,     # half a step, relative
        torch.float64: 2.0 ** -53}
TINY = {torch.float32: 2.0 ** -126, torch.float16: 2.0 ** -24, torch.bfloat16: 2.0 ** -126,  # where steps stop shrinking
        torch.float64: 0.0}


def seq(m):
    return 32 + m / 64


def store(v, dtype):
    return v.abs() * STEP[dtype] * 1.01 + TINY[dtype]


def assert_within(got, want, bound, what=""):
    g = got.double()
    assert g.shape == want.shape, (what, g.shape, want.shape)
    off = (g - want).abs()
    bad = ~(off <= bound)
    if bad.any():
        i = int(torch.where(bad, off / bound.clamp(min=1e-300), torch.zeros_like(off)).nan_to_num(1e300).flatten().argmax())
        raise AssertionError(f"{what}: {int(bad.sum())} of {bad.numel()} beyond the bound; worst at {i}: got "
                             f"{g.flatten()[i].item()} want {want.flatten()[i].item()} bound {bound.flatten()[i].item()}")


def norm(x, w, b, eps):
    """(y, mean, rstd) and their bounds (y's for the type of x)."""
    v, d = x.double(), x.shape[-1]
    mean = v.mean(-1)
    c = v - mean[..., None]
    rstd = 1.0 / (c.square().mean(-1) + eps).sqrt()
    h = c * rstd[..., None]
    wd = torch.ones(d, dtype=torch.float64, device=x.device) if w is None else w.double()
    bd = torch.zeros(d, dtype=torch.float64, device=x.device) if b is None else b.double()
    y = h * wd + bd
    m1 = v.abs().mean(-1)
    e_mean = (seq(d) + 4) * U * m1
    # the variance's terms (x - mu)^2: each off by 2 |x - mu| (e_mean + u |x - mu|), then the sum's own rounding
    e_c = e_mean[..., None] + U * c.abs()
    e_var = (2 * c.abs() * e_c + e_c.square()).mean(-1) + (seq(d) + 4) * U * c.square().mean(-1)
    e_rstd = 0.5 * rstd ** 3 * e_var * 1.1 + 4 * U * rstd
    e_h = rstd[..., None] * e_c + c.abs() * e_rstd[..., None] + e_c * e_rstd[..., None] + 2 * U * h.abs()
    e_y = e_h * wd.abs() + 2 * U * (h * wd).abs() + 2 * U * y.abs()
    return (y, mean, rstd), (e_y + store(y, x.dtype), e_mean + U * mean.abs(), e_rstd)


def norm_grad(dy, x, mean, rstd, w, wdtype):
    """(dx, dw, db) and their bounds, with the mean and rstd that the forward pass stored as inputs."""
    d, n = x.shape[-1], x.shape[0]
    g0, r = dy.double(), rstd.double()[:, None]
    c = x.double() - mean.double()[:, None]
    h = c * r
    wd = torch.ones(d, dtype=torch.float64, device=x.device) if w is None else w.double()
    g = g0 * wd
    c1, c2 = g.mean(-1, keepdim=True), (g * h).mean(-1, keepdim=True)
    dx = r * (g - c1 - h * c2)
    e1 = (seq(d) + 6) * U * g.abs().mean(-1, keepdim=True)
    e2 = (seq(d) + 10) * U * (g * h).abs().mean(-1, keepdim=True)
    e_dx = r * (4 * U * g.abs() + e1 + h.abs() * e2 + 6 * U * (h * c2).abs() + 4 * U * c1.abs()) + 2 * U * dx.abs()
    dw, db = (g0 * h).sum(0), g0.sum(0)
    e_dw = (seq(n) + 6) * U * (g0 * h).abs().sum(0)
    e_db = (seq(n) + 6) * U * g0.abs().sum(0)
    return (dx, dw, db), (e_dx + store(dx, x.dtype), e_dw + store(dw, wdtype), e_db + store(db, wdtype))


def cross_entropy(z, labels, mean):
    """(loss, row_loss, dz) and their bounds; rows of finite logits and -inf, with a finite logit at the label."""
    v, k = z.double(), z.shape[-1]
    y = labels.long()
    kept = y >= 0
    s = 1.0 / max(1, int(kept.sum())) if mean else 1.0
    m = v.max(-1, keepdim=True).values
    t = v - m
    e = t.exp()
    total = e.sum(-1, keepdim=True)
    p = e / total
    at = y.clamp(min=0)[:, None]
    tl = t.gather(1, at)
    row = torch.where(kept, (total.log() - tl)[:, 0], torch.zeros_like(tl[:, 0]))
    one = torch.zeros_like(p).scatter_(1, at, 1.0)
    dz = (p - one) * kept[:, None] * s
    # exp's argument is off by 3 u |t| (the difference, and the change of base), exp by 4 u; then the sum's rounding
    depth = torch.where(t.isinf(), torch.zeros_like(t), t.abs())
    e_rel = U * (3 * depth + 4)
    e_total = (p * e_rel).sum(-1, keepdim=True) + (seq(k) + 4) * U
    e_p = p * (e_rel + e_total + 6 * U)
    e_dz = (e_p + 2 * U * dz.abs() / s) * s + U * 2 * dz.abs() + 2.0 ** -126
    e_row = (e_total + 4 * U * (total.log().abs() + tl.abs() + 1))[:, 0] * kept
    loss = row.sum() * s
    e_loss = e_row.sum() * s + 4 * U * loss.abs() + 2.0 ** -126
    return (loss, row, dz), (e_loss, e_row + 2.0 ** -126, e_dz * kept[:, None] + store(dz, z.dtype))


def clip(grads, max_norm, eps):
    """(norm, c) in 64 bits."""
    n = torch.stack([g.double().square().sum() for g in grads]).sum().sqrt()
    return n, min(1.0, max_norm / (float(n) + eps))


#: squares are summed in FP32 over at most 32 values, then in FP64; the root halves it, c adds two roundings
CLIP_NORM = 24 * U
CLIP_SCALE = 30 * U
