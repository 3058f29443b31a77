"""Cases of the training operators: layer norm (forward, backward), cross entropy on cluster labels, gradient clipping.

Each case is one call that a program makes which trains an encoder on the labels that the clustering
gave its features.  `run` does it either in plain torch operations in 32 bits (own = False) or through
this package's entry points (own = True); `exact` does it in 64 bits.
"""
import math

import torch

own = False

EPS = 1e-5          # layer norm
CLIP_EPS = 1e-6     # added to the norm before the division
TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}

# Widths: 768 features and 1000 clusters are the embedding workload of this repository's benchmark, 64 and
# 100 its many-cluster workload; the other sizes are generic.
LISTED = [
    # one vector is embedded when a query arrives: nothing but latency
    {"name": "norm one query", "op": "norm", "n": 1, "d": 768, "type": "f32", "wtype": "f32", "pad": 0},
    # odd width, so that rows begin at any address of their type
    {"name": "norm odd width", "op": "norm", "n": 4099, "d": 1001, "type": "f16", "wtype": "f16", "pad": 0},
    # a pass of the encoder's last norm over a shard of the embedding workload
    {"name": "norm embedding shard", "op": "norm", "n": 262144, "d": 768, "type": "bf16", "wtype": "f32", "pad": 0},
    # the smallest training step: a few rows
    {"name": "norm grad few rows", "op": "norm_grad", "n": 24, "d": 768, "type": "f32", "wtype": "f32", "pad": 0},
    # an ordinary batch whose rows are a slice of wider ones
    {"name": "norm grad sliced batch", "op": "norm_grad", "n": 32768, "d": 1000, "type": "bf16", "wtype": "f32", "pad": 24},
    # a large batch, all in bf16
    {"name": "norm grad embedding batch", "op": "norm_grad", "n": 262144, "d": 768, "type": "bf16", "wtype": "bf16", "pad": 0},
    # a wide hidden layer: few rows, and the weight's gradient is as wide
    {"name": "norm grad wide", "op": "norm_grad", "n": 1021, "d": 16384, "type": "f32", "wtype": "f32", "pad": 0},
    # a few rows against the many-cluster workload's 100 labels
    {"name": "labels few rows", "op": "labels", "n": 16, "k": 100, "type": "f32", "left_out": 0.0, "pad": 0},
    # a batch against 1000 clusters, some rows masked out of the loss
    {"name": "labels batch", "op": "labels", "n": 131072, "k": 1000, "type": "bf16", "left_out": 0.08, "pad": 0},
    # a fine clustering: rows that no warp holds in its registers
    {"name": "labels fine clustering", "op": "labels", "n": 2053, "k": 32768, "type": "f16", "left_out": 0.02, "pad": 0},
    # a small head's gradients: two linear layers and a norm
    {"name": "clip head", "op": "clip", "layers": 1, "width": 256, "type": "f32", "out": "f32", "max_norm": 0.5},
    # an encoder's gradients, weights' and norms' in bf16, clipped into the optimizer's 32-bit buffers
    {"name": "clip encoder", "op": "clip", "layers": 10, "width": 1024, "type": "bf16", "out": "f32", "max_norm": 1.0},
]
MOST = 1.2e9        # bytes of the largest listed case; drawn ones stay below


def listed():
    return [dict(c) for c in LISTED]


def spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["norm", "norm", "norm_grad", "norm_grad", "norm_grad", "labels", "labels", "labels", "clip", "clip"])
    kind = rng.choice(["f32", "f16", "bf16"])
    if op == "clip":
        width = spread(rng, 48, 1024)
        while True:
            layers = spread(rng, 1, 10)
            case = {"op": op, "layers": layers, "width": width, "type": kind, "out": rng.choice([kind, "f32"]),
                    "max_norm": rng.choice([0.1, 1.0, 1e4])}
            if work(case)["bytes"] <= MOST:
                return case
    pad = rng.choice([0, 0, 0, 8, 13])
    while True:
        n = spread(rng, 1, 262144)
        wide = spread(rng, 2, 32768) if op == "labels" else spread(rng, 16, 16384)
        if op == "labels":
            case = {"op": op, "n": n, "k": wide, "type": kind, "left_out": rng.choice([0.0, 0.08, 0.3]), "pad": pad}
        else:
            case = {"op": op, "n": n, "d": wide, "type": kind, "wtype": rng.choice(["f32", kind]), "pad": pad}
        if work(case)["bytes"] <= MOST:
            return case


def shapes(case):
    """The parameters of an encoder of `layers` blocks: two products with their biases and one norm each."""
    w, f = case["width"], 4 * case["width"] + 1     # one odd width among them
    block = [(f, w), (f,), (w, f), (w,), (w,), (w,)]
    return block * case["layers"] + [(100, w)]


def work(case):
    op = case["op"]
    if op == "clip":
        e = sum(math.prod(s) for s in shapes(case))
        return {"bytes": e * (SIZE[case["type"]] + SIZE[case["out"]]) + 4, "flops": 3 * e}
    n, s = case["n"], SIZE[case["type"]]
    if op == "norm":
        d, ws = case["d"], SIZE[case["wtype"]]
        return {"bytes": 2 * n * d * s + 2 * d * ws + 8 * n, "flops": 7 * n * d}
    if op == "norm_grad":
        d, ws = case["d"], SIZE[case["wtype"]]
        return {"bytes": 3 * n * d * s + 3 * d * ws + 8 * n, "flops": 13 * n * d}
    k = case["k"]
    return {"bytes": 2 * n * k * s + 8 * n + 4, "flops": 6 * n * k}


def rows(gen, n, wide, pad, kind, scale=1.0, shift=None):
    """n rows of `wide` values; with pad, a slice of rows that are `pad` longer."""
    x = torch.randn(n, wide + pad, generator=gen, device="cuda")
    x = x.mul_(scale)[:, :wide]
    if shift is not None:
        x += shift
    if pad == 0:
        return x.to(TYPES[kind])
    whole = torch.empty(n, wide + pad, device="cuda", dtype=TYPES[kind])
    whole[:, :wide] = x
    return whole[:, :wide]


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op = case["op"]
    if op == "clip":
        made = [(torch.randn(s, generator=gen, device="cuda") * (0.02 / math.sqrt(s[-1]))).to(TYPES[case["type"]])
                for s in shapes(case)]
        return {"op": op, "grads": made, "max_norm": case["max_norm"],
                "out": [torch.empty(g.shape, device="cuda", dtype=TYPES[case["out"]]) for g in made]}
    n = case["n"]
    if op == "labels":
        # logits of a part-trained head: spread out, the right cluster ahead in most rows; a few clusters own many rows
        k = case["k"]
        z = torch.randn(n, k, generator=gen, device="cuda").mul_(2.0)
        u = torch.rand(n, generator=gen, device="cuda")
        labels = (u * u * k).to(torch.int64).clamp_(max=k - 1)
        ahead = torch.rand(n, generator=gen, device="cuda") * 8.0
        z.scatter_add_(1, labels[:, None], ahead[:, None])
        out = torch.rand(n, generator=gen, device="cuda") < case["left_out"]
        labels = torch.where(out, torch.full_like(labels, -1), labels).to(torch.int32)
        whole = torch.empty(n, k + case["pad"], device="cuda", dtype=TYPES[case["type"]])
        whole[:, :k] = z
        return {"op": op, "logits": whole[:, :k], "labels": labels}
    # features: each column with its own offset, and a few columns far above the others
    d = case["d"]
    shift = torch.randn(d, generator=gen, device="cuda") * 0.5
    shift[:: max(1, d // 4)] += 6.0
    x = rows(gen, n, d, case["pad"], case["type"], 1.0, shift)
    w = (1.0 + 0.1 * torch.randn(d, generator=gen, device="cuda")).to(TYPES[case["wtype"]])
    b = (0.1 * torch.randn(d, generator=gen, device="cuda")).to(TYPES[case["wtype"]])
    if op == "norm":
        return {"op": op, "x": x, "weight": w, "bias": b}
    dy = rows(gen, n, d, case["pad"], case["type"], 0.05)
    _, mean, rstd = plain_norm(x, w, b)
    return {"op": op, "dy": dy, "x": x, "mean": mean, "rstd": rstd, "weight": w}


def plain_norm(x, weight, bias):
    v = x.float()
    mean = v.mean(1)
    c = v - mean[:, None]
    rstd = 1.0 / (c.square().mean(1) + EPS).sqrt()
    y = c * rstd[:, None] * weight.float() + bias.float()
    return y.to(x.dtype), mean, rstd


def plain_norm_grad(dy, x, mean, rstd, weight):
    g = dy.float()
    h = (x.float() - mean[:, None]) * rstd[:, None]
    gw = g * weight.float()
    dx = rstd[:, None] * (gw - gw.mean(1, keepdim=True) - h * (gw * h).mean(1, keepdim=True))
    return dx.to(x.dtype), (g * h).sum(0).to(weight.dtype), g.sum(0).to(weight.dtype)


def plain_labels(logits, labels):
    z = logits.float()
    kept = labels >= 0
    at = labels.clamp(min=0).long()[:, None]
    s = z - z.max(1, keepdim=True).values
    e = s.exp()
    total = e.sum(1, keepdim=True)
    row = torch.where(kept, (total.log() - s.gather(1, at))[:, 0], torch.zeros_like(total[:, 0]))
    scale = 1.0 / kept.sum().clamp(min=1).float()
    dz = e / total
    dz.scatter_add_(1, at, torch.full_like(total, -1.0))
    dz = dz * (scale * kept.float())[:, None]
    return row.sum() * scale, row, dz.to(logits.dtype)


def plain_clip(grads, out, max_norm):
    norm = torch.stack([g.float().square().sum() for g in grads]).sum().sqrt()
    c = (max_norm / (norm + CLIP_EPS)).clamp(max=1.0)
    return norm, [(g.float() * c).to(o.dtype) for g, o in zip(grads, out)]


def run(state):
    op = state["op"]
    if op == "norm":
        x, w, b = state["x"], state["weight"], state["bias"]
        if own:
            import paper_2609_36074_b200 as gem
            return gem.layer_norm(x, w, b, eps=EPS)
        return plain_norm(x, w, b)
    if op == "norm_grad":
        dy, x, mean, rstd, w = (state[k] for k in ("dy", "x", "mean", "rstd", "weight"))
        if own:
            import paper_2609_36074_b200 as gem
            return gem.layer_norm_backward(dy, x, mean, rstd, w)
        return plain_norm_grad(dy, x, mean, rstd, w)
    if op == "labels":
        z, labels = state["logits"], state["labels"]
        if own:
            import paper_2609_36074_b200 as gem
            return gem.label_cross_entropy(z, labels)
        return plain_labels(z, labels)
    grads, out, most = state["grads"], state["out"], state["max_norm"]
    if own:
        import paper_2609_36074_b200 as gem
        return gem.clip_grad_norm(grads, most, out=out, eps=CLIP_EPS), out
    return plain_clip(grads, out, most)


def exact(case, seed):
    """The definitions in 64 bits, taken over blocks of rows so that the largest case fits."""
    s = prepare(case, seed)
    op = s["op"]
    if op == "clip":
        big = torch.cat([g.reshape(-1).double() for g in s["grads"]])
        norm = torch.linalg.vector_norm(big)
        del big
        ratio = float(s["max_norm"]) / (float(norm) + CLIP_EPS)
        return norm, [g.double() * min(1.0, ratio) for g in s["grads"]]
    step = max(1, 2 ** 25 // max(case.get("d", 1), case.get("k", 1)))
    spans = [slice(i, i + step) for i in range(0, case["n"], step)]
    if op == "norm":
        parts = []
        for a in spans:
            v = s["x"][a].double()
            var, mean = torch.var_mean(v, dim=1, unbiased=False)
            r = torch.rsqrt(var + EPS)
            y = torch.addcmul(s["bias"].double(), (v - mean[:, None]) * r[:, None], s["weight"].double())
            parts.append((y, mean, r))
        return tuple(torch.cat(p) for p in zip(*parts))
    if op == "norm_grad":
        w, d = s["weight"].double(), case["d"]
        dx, dw, db = [], torch.zeros_like(w), torch.zeros_like(w)
        for a in spans:
            g, r = s["dy"][a].double(), s["rstd"][a].double()[:, None]
            h = (s["x"][a].double() - s["mean"][a].double()[:, None]) * r
            dw += torch.einsum("nd,nd->d", g, h)
            db += torch.einsum("nd->d", g)
            c1 = torch.einsum("nd,d->n", g, w) / d
            c2 = torch.einsum("nd,nd,d->n", g, h, w) / d
            dx.append((g * w - c1[:, None] - h * c2[:, None]) * r)
        return torch.cat(dx), dw, db
    z, y = s["logits"], s["labels"].long()
    kept = y >= 0
    scale = 1.0 / max(1, int(kept.sum()))
    row, dz = [], []
    for a in spans:
        logp = torch.log_softmax(z[a].double(), 1)
        one = torch.nn.functional.one_hot(y[a].clamp(min=0), case["k"]).double()
        row.append(torch.where(kept[a], -(logp * one).sum(1), 0.0))
        dz.append((logp.exp() - one) * kept[a][:, None] * scale)
    row = torch.cat(row)
    return row.sum() * scale, row, torch.cat(dz)
