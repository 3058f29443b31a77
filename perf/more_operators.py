"""Cases of an expert layer's operators: routing rows to experts, the experts' products, the weighted sum of their outputs, and
activations whose inputs are kept in 8 bits for the backward pass.

Each case is one call (or a call and its gradient) that a program makes which trains an encoder with expert layers.  `run`
does it either in plain torch operations (own = False) or through this package's entry points (own = True); `exact` does it in
64 bits.
"""
import math

import torch

own = False

TYPES = {"f32": torch.float32, "f16": torch.float16, "bf16": torch.bfloat16}
SIZE = {"f32": 4, "f16": 2, "bf16": 2}

# Widths: 768 features are the embedding workload of this repository's benchmark; the other sizes are generic.
LISTED = [
    # one query is embedded: nothing but latency
    {"name": "route one row", "op": "route", "n": 1, "experts": 8, "k": 2, "score": "softmax", "bias": False, "groups": 1, "kept": 1,
     "best": 1, "renorm": True, "type": "f32", "left_out": 0.0},
    # a training batch: sigmoid scores, a bias that balances the load, experts in groups
    {"name": "route batch in groups", "op": "route", "n": 65536, "experts": 128, "k": 6, "score": "sigmoid", "bias": True, "groups": 8,
     "kept": 4, "best": 2, "renorm": True, "type": "f32", "left_out": 0.02},
    # the router's gradient, whole softmax
    {"name": "route grad batch", "op": "route_grad", "n": 131072, "experts": 64, "k": 4, "score": "softmax", "bias": False, "groups": 1,
     "kept": 1, "best": 1, "renorm": False, "type": "bf16", "left_out": 0.0},
    # a few queries: every expert's weights are read for a handful of rows
    {"name": "product few rows", "op": "product", "n": 16, "experts": 8, "k": 2, "din": 768, "dout": 1024, "type": "bf16", "gather": True,
     "turned": False, "left_out": 0.0},
    # odd widths, so that rows begin at any address of their type
    {"name": "product odd widths", "op": "product", "n": 3001, "experts": 12, "k": 1, "din": 1001, "dout": 515, "type": "f16", "gather": False,
     "turned": True, "left_out": 0.1},
    # the first product of a training batch
    {"name": "product batch", "op": "product", "n": 32768, "experts": 32, "k": 4, "din": 768, "dout": 2048, "type": "bf16", "gather": True,
     "turned": False, "left_out": 0.0},
    # both gradients of the second product of a training batch
    {"name": "product grad batch", "op": "product_grad", "n": 32768, "experts": 32, "k": 4, "din": 2048, "dout": 768, "type": "bf16",
     "gather": False, "turned": False, "left_out": 0.0},
    # the second product's rows back to their tokens
    {"name": "combine batch", "op": "combine", "n": 32768, "k": 4, "experts": 32, "d": 768, "type": "bf16", "left_out": 0.0},
    # and the gradient of that
    {"name": "combine grad batch", "op": "combine_grad", "n": 32768, "k": 4, "experts": 32, "d": 768, "type": "bf16", "left_out": 0.02},
    # a few rows through an activation and back
    {"name": "activation few rows", "op": "activation", "n": 24, "d": 1000, "kind": "gelu", "gated": False, "type": "f32"},
    # gated units of a training batch, there and back from the 8 bits
    {"name": "activation gated batch", "op": "activation", "n": 65536, "d": 2048, "kind": "silu", "gated": True, "type": "bf16"},
    # features kept in 8 bits and restored
    {"name": "checkpoint features", "op": "checkpoint", "n": 262144, "d": 768, "type": "f32"},
]
MOST_BYTES, MOST_FLOPS = 1.8e9, 8.3e11        # of the largest listed cases; drawn ones stay below


def listed():
    return [dict(c) for c in LISTED]


def spread(rng, lo, hi):
    """A whole number between lo and hi, even over the logarithm."""
    return max(lo, min(hi, round(math.exp(rng.uniform(math.log(lo), math.log(hi + 1))))))


def draw(rng):
    op = rng.choice(["route", "route", "route_grad", "product", "product", "product", "product_grad", "product_grad", "combine",
                     "combine_grad", "activation", "activation", "checkpoint"])
    while True:
        case = drawn(rng, op)
        w = work(case)
        if w["bytes"] <= MOST_BYTES and w["flops"] <= MOST_FLOPS:
            return case


def drawn(rng, op):
    if op in ("route", "route_grad"):
        groups = rng.choice([1, 1, 2, 4, 8])
        experts = groups * spread(rng, 4, 256 // groups)
        kept = 1 if groups == 1 else rng.randint(groups // 2, groups)
        k = rng.randint(1, min(8, kept * (experts // groups)))
        return {"op": op, "n": spread(rng, 1, 131072), "experts": experts, "k": k, "score": rng.choice(["softmax", "sigmoid"]),
                "bias": rng.random() < 0.5, "groups": groups, "kept": kept, "best": 1 if groups == 1 else rng.choice([1, 2]),
                "renorm": rng.random() < 0.6, "type": rng.choice(["f32", "f16", "bf16"]), "left_out": rng.choice([0.0, 0.0, 0.1])}
    if op in ("product", "product_grad"):
        experts = spread(rng, 2, 64)
        grain = rng.choice([1, 8, 64])
        return {"op": op, "n": spread(rng, 1, 65536), "experts": experts, "k": rng.randint(1, min(4, experts)),
                "din": grain * spread(rng, -(-32 // grain), 2048 // grain), "dout": grain * spread(rng, -(-32 // grain), 2048 // grain),
                "type": rng.choice(["f16", "bf16"]), "gather": rng.random() < 0.5, "turned": rng.random() < 0.3,
                "left_out": rng.choice([0.0, 0.0, 0.1])}
    if op in ("combine", "combine_grad"):
        return {"op": op, "n": spread(rng, 1, 65536), "k": rng.randint(1, 8), "experts": spread(rng, 8, 64), "d": spread(rng, 16, 4096),
                "type": rng.choice(["f32", "f16", "bf16"]), "left_out": rng.choice([0.0, 0.0, 0.1])}
    if op == "activation":
        return {"op": op, "n": spread(rng, 1, 131072), "d": spread(rng, 16, 4096), "kind": rng.choice(["silu", "gelu", "tanh"]),
                "gated": rng.random() < 0.5, "type": rng.choice(["f32", "f16", "bf16"])}
    return {"op": op, "n": spread(rng, 1, 262144), "d": spread(rng, 16, 4096), "type": rng.choice(["f32", "f16", "bf16"])}


def work(case):
    op, n = case["op"], case["n"]
    if op in ("route", "route_grad"):
        e, k, s = case["experts"], case["k"], SIZE[case["type"]]
        if op == "route":
            return {"bytes": n * e * s + 16 * n * k + 8 * e, "flops": 8 * n * e}
        return {"bytes": 2 * n * e * s + 8 * n * k, "flops": 10 * n * e}
    if op in ("product", "product_grad"):
        m, i, o = n * case["k"], case["din"], case["dout"]
        x, w, y = (n if case["gather"] else m) * i, min(case["experts"], m) * i * o, m * o
        if op == "product":
            return {"bytes": 2 * (x + w + y) + 4 * m, "flops": 2 * m * i * o}
        return {"bytes": 2 * (x + y + w + m * i + case["experts"] * i * o) + 4 * m, "flops": 4 * m * i * o}
    s, d = SIZE[case["type"]], case["d"]
    if op == "combine":
        return {"bytes": n * (case["k"] + 1) * d * s + 8 * n * case["k"], "flops": 2 * n * case["k"] * d}
    if op == "combine_grad":
        return {"bytes": n * (2 * case["k"] + 1) * d * s + 12 * n * case["k"], "flops": 3 * n * case["k"] * d}
    if op == "activation":
        wide = 2 * d if case["gated"] else d
        # z and dy are read, y, the gradient and y again are written; the 8 bits and their scales are written and read
        return {"bytes": n * (2 * wide * s + 3 * d * s + 2 * wide + wide // 16), "flops": 25 * n * wide}
    return {"bytes": n * d * 2 * s + n * d * 2 + n * (d // 16), "flops": 4 * n * d}


def some_logits(case, gen):
    """Logits of a part-trained router: some experts are more popular than others; rows left out have none to go to."""
    n, e = case["n"], case["experts"]
    z = torch.randn(n, e, generator=gen, device="cuda") + 0.25 * torch.randn(e, generator=gen, device="cuda")
    out = torch.rand(n, generator=gen, device="cuda") < case["left_out"]
    return z.masked_fill(out[:, None], -math.inf)


def plan(expert, experts):
    """(offset, row, place) of a choice of experts (n x k, -1 for none): the places sorted by expert, rows in order."""
    n, k = expert.shape
    e = expert.reshape(-1).long()
    key = torch.where(e < 0, torch.full_like(e, experts), e)
    order = torch.sort(key, stable=True).indices
    offset = torch.searchsorted(key[order].contiguous(), torch.arange(experts + 1, device=e.device))
    at = torch.arange(n * k, device=e.device)
    used = at < offset[-1]
    place = torch.empty_like(at).index_copy_(0, order, torch.where(used, at, torch.full_like(at, -1)))
    row = torch.where(used, order // k, torch.full_like(at, -1))
    return offset.int(), row.int(), place.int().view(n, k)


def some_plan(case, gen):
    z = some_logits(case, gen)
    top = z.topk(case["k"], dim=1)
    expert = torch.where(top.values == -math.inf, torch.full_like(top.indices, -1), top.indices).int()
    return plan(expert, case["experts"])


def prepare(case, seed):
    gen = torch.Generator(device="cuda").manual_seed(int(seed))
    op, n = case["op"], case["n"]

    def normal(*shape, scale=1.0, kind=None):
        return (torch.randn(*shape, generator=gen, device="cuda") * scale).to(TYPES[kind or case["type"]])

    s = {"op": op, "case": case}
    if op in ("route", "route_grad"):
        s["logits"] = some_logits(case, gen).to(TYPES[case["type"]])
        s["bias"] = normal(case["experts"], scale=0.05, kind="f32") if case["bias"] else None
        if op == "route_grad":
            top = s["logits"].float().topk(case["k"], dim=1)
            s["expert"] = torch.where(top.values == -math.inf, torch.full_like(top.indices, -1), top.indices).int()
            s["dweight"] = normal(n, case["k"], kind="f32")
        return s
    if op in ("product", "product_grad"):
        e, i, o = case["experts"], case["din"], case["dout"]
        s["offset"], row, _ = some_plan(case, gen)
        s["row"] = row if case["gather"] else None
        s["x"] = normal(n if case["gather"] else n * case["k"], i)
        w = normal(e, o, i, scale=i ** -0.5) if case["turned"] else normal(e, i, o, scale=i ** -0.5)
        s["w"] = w.transpose(1, 2) if case["turned"] else w
        if op == "product_grad":
            s["dy"] = normal(n * case["k"], o, scale=0.05)
        # the widest expert's rows: the plain form takes the experts' products as one batch of that height
        s["most"] = int((s["offset"][1:] - s["offset"][:-1]).max())
        return s
    if op in ("combine", "combine_grad"):
        k = case["k"]
        s["offset"], _, s["place"] = some_plan(case, gen)
        s["weight"] = torch.rand(n, k, generator=gen, device="cuda")
        s["weight"] /= s["weight"].sum(1, keepdim=True)
        s["y"] = normal(n * k, case["d"])
        if op == "combine_grad":
            s["dout"] = normal(n, case["d"], scale=0.05)
        return s
    wide = 2 * case["d"] if op == "activation" and case["gated"] else case["d"]
    # each column has its own spread, and a few are far above the others
    spreads = torch.exp(0.5 * torch.randn(wide, generator=gen, device="cuda"))
    spreads[:: max(1, wide // 4)] *= 6.0
    s["z"] = (torch.randn(n, wide, generator=gen, device="cuda") * spreads).to(TYPES[case["type"]])
    if op == "activation":
        s["dy"] = normal(n, case["d"], scale=0.05)
    return s


def plain_route(s):
    """The choice is made in 64 bits: scores that are next to one another decide it."""
    c = s["case"]
    n, e, k, groups = c["n"], c["experts"], c["k"], c["groups"]
    z = s["logits"].double()
    none = z == -math.inf
    if c["score"] == "softmax":
        x = (z - z.max(1, keepdim=True).values.clamp(min=-1e300)).exp()
        score = x / x.sum(1, keepdim=True).clamp(min=1e-300)
    else:
        score = 1.0 / (1.0 + (-z).exp())
    key = z if s["bias"] is None else torch.where(none, z, score + s["bias"].double())
    if groups > 1:
        by = (key if c["best"] == 1 else torch.where(none, z, score) if s["bias"] is None else key).view(n, groups, e // groups)
        best = by.sort(dim=2, descending=True).values[:, :, :c["best"]]
        best = best[:, :, 0] + torch.where(best[:, :, 1:] == -math.inf, 0.0, best[:, :, 1:]).sum(2)
        at = best.sort(dim=1, descending=True, stable=True).indices[:, :c["kept"]]
        stays = torch.zeros(n, groups, dtype=torch.bool, device=z.device).scatter_(1, at, True)
        key = torch.where(stays[:, :, None], key.view(n, groups, -1), -math.inf).view(n, e)
    top = key.sort(dim=1, descending=True, stable=True)
    chosen, has = top.indices[:, :k], top.values[:, :k] != -math.inf
    w = torch.where(has, score.gather(1, chosen), 0.0)
    if c["renorm"]:
        total = w.sum(1, keepdim=True)
        w = torch.where(total > 0, w / total, 0.0)
    expert = torch.where(has, chosen, -1).int()
    return (expert, (w * SCALE).float(), *plan(expert, e))


SCALE = 1.5          # of the routing weights


def plain_route_grad(s):
    c = s["case"]
    z, has = s["logits"].float(), s["expert"] >= 0
    at = s["expert"].clamp(min=0).long()
    if c["score"] == "softmax":
        x = (z - z.max(1, keepdim=True).values.clamp(min=-3e38)).exp()
        score = x / x.sum(1, keepdim=True).clamp(min=1e-37)
    else:
        score = 1.0 / (1.0 + (-z).exp())
    picked = torch.where(has, score.gather(1, at), 0.0)
    g = torch.where(has, s["dweight"], 0.0) * SCALE
    if c["renorm"]:
        total = picked.sum(1, keepdim=True).clamp(min=1e-37)
        g = (g - (picked * g).sum(1, keepdim=True) / total) / total
    g = torch.where(has, g, 0.0)
    dscore = torch.zeros_like(z).scatter_add_(1, at, g)
    if c["score"] == "softmax":
        dz = score * (dscore - (score * dscore).sum(1, keepdim=True))
    else:
        dz = score * (1.0 - score) * dscore
    return dz.to(s["logits"].dtype)


def padded(s):
    """For a batch with every expert's rows side by side: (place of each of its rows, which of them there are)."""
    first, count = s["offset"][:-1].long(), (s["offset"][1:] - s["offset"][:-1]).long()
    at = torch.arange(s["most"], device=first.device)
    there = at[None, :] < count[:, None]
    return torch.where(there, first[:, None] + at[None, :], 0), there


def as_batch(v, at, there):
    return torch.where(there[:, :, None], v.float()[at], 0.0)


def from_batch(v, at, there, rows):
    """The batch's rows at their places, zeros at places without an expert."""
    out = torch.zeros(rows + 1, v.shape[2], device=v.device)
    out.index_copy_(0, torch.where(there, at, rows).reshape(-1), v.reshape(-1, v.shape[2]))
    return out[:rows]


def plain_product(s):
    at, there = padded(s)
    rows = s["case"]["n"] * s["case"]["k"]
    source = at if s["row"] is None else s["row"].clamp(min=0).long()[at]
    y = torch.bmm(as_batch(s["x"], source, there), s["w"].float())
    return from_batch(y, at, there, rows).to(s["x"].dtype)


def plain_product_grad(s):
    at, there = padded(s)
    rows = s["case"]["n"] * s["case"]["k"]
    source = at if s["row"] is None else s["row"].clamp(min=0).long()[at]
    dy = as_batch(s["dy"], at, there)
    dx = from_batch(torch.bmm(dy, s["w"].float().transpose(1, 2)), at, there, rows).to(s["x"].dtype)
    return dx, torch.bmm(as_batch(s["x"], source, there).transpose(1, 2), dy).to(s["w"].dtype)


def plain_combine(s):
    has = s["place"] >= 0
    y = s["y"].float()[s["place"].clamp(min=0).long()]
    return (torch.where(has, s["weight"], 0.0)[:, :, None] * y).sum(1).to(s["y"].dtype)


def plain_combine_grad(s):
    has, at = s["place"] >= 0, s["place"].clamp(min=0).long()
    dout = s["dout"].float()
    dweight = torch.where(has, (s["y"].float()[at] * dout[:, None, :]).sum(2), 0.0)
    rows = s["y"].shape[0]
    dy = torch.zeros(rows + 1, dout.shape[1], device=dout.device)
    v = s["weight"][:, :, None] * dout[:, None, :]
    dy.index_copy_(0, torch.where(has, s["place"].long(), rows).reshape(-1), v.reshape(-1, dout.shape[1]))
    return dy[:rows].to(s["y"].dtype), dweight


def plain_restored(z):
    """What the 8 bits of each 32 columns stand for: q 2^e, q = z 2^-e rounded to a whole number, e the smallest of -127 and above
    with the largest magnitude below 127.5 2^e."""
    n, d = z.shape
    v = torch.nn.functional.pad(z.float(), (0, -d % 32)).view(n, -1, 32)
    top = v.abs().amax(2, keepdim=True)
    e = torch.frexp(top / 127.5).exponent                    # top / 127.5 = f 2^e, f in [0.5, 1): the quotient is below 2^e
    e = torch.where(top < 127.5 * torch.ldexp(torch.ones_like(top), e - 1), e - 1, e)
    e = torch.where(top < 127.5 * torch.ldexp(torch.ones_like(top), e), e, e + 1).clamp(min=-127)
    return torch.ldexp(torch.round(torch.ldexp(v, -e)), e).view(n, -1)[:, :d]


def plain_act(z, kind):
    """(value, slope)"""
    if kind == "silu":
        p = 1.0 / (1.0 + (-z).exp())
        return z * p, p * (1.0 + z * (1.0 - p))
    if kind == "gelu":
        p = 0.5 * torch.erfc(z * -math.sqrt(0.5))
        return z * p, p + z * (-0.5 * z * z).exp() * (1.0 / math.sqrt(2.0 * math.pi))
    t = torch.tanh(z)
    return t, 1.0 - t * t


def plain_activation(s):
    c, z, dy = s["case"], s["z"], s["dy"].float()
    if c["gated"]:
        g, u = z.float().chunk(2, 1)
        y = plain_act(g, c["kind"])[0] * u
        g, u = (plain_restored(t) for t in z.chunk(2, 1))
        a, slope = plain_act(g, c["kind"])
        dz, again = torch.cat([dy * u * slope, dy * a], 1), a * u
    else:
        y = plain_act(z.float(), c["kind"])[0]
        again, slope = plain_act(plain_restored(z), c["kind"])
        dz = dy * slope
    return y.to(z.dtype), dz.to(z.dtype), again.to(z.dtype)


def run(state):
    s, op, c = state, state["op"], state["case"]
    if own:
        import paper_2609_36074_b200 as gem
        if op == "route":
            return tuple(gem.route(s["logits"], c["k"], c["score"], bias=s["bias"], groups=c["groups"], kept_groups=c["kept"],
                                   group_best=c["best"], renormalize=c["renorm"], scale=SCALE))
        if op == "route_grad":
            return gem.route_backward(s["dweight"], s["logits"], s["expert"], c["score"], renormalize=c["renorm"], scale=SCALE)
        if op == "product":
            return gem.expert_product(s["x"], s["w"], s["offset"], s["row"])
        if op == "product_grad":
            return gem.expert_product_backward(s["dy"], s["x"], s["w"], s["offset"], s["row"])
        if op == "combine":
            return gem.combine(s["y"], s["place"], s["weight"])
        if op == "combine_grad":
            return gem.combine_backward(s["dout"], s["y"], s["place"], s["weight"], s["offset"])
        if op == "activation":
            y, saved = gem.activation(s["z"], c["kind"], gated=c["gated"])
            return (y, *gem.activation_backward(s["dy"], saved, c["kind"], gated=c["gated"], need_y=True))
        return gem.restore(gem.checkpoint(s["z"]))
    if op == "route":
        return plain_route(s)
    if op == "route_grad":
        return plain_route_grad(s)
    if op == "product":
        return plain_product(s)
    if op == "product_grad":
        return plain_product_grad(s)
    if op == "combine":
        return plain_combine(s)
    if op == "combine_grad":
        return plain_combine_grad(s)
    if op == "activation":
        return plain_activation(s)
    return plain_restored(s["z"]).to(s["z"].dtype)


def exact_restored(z):
    """The same by powers of two in 64 bits, rounding the logarithm down and mending it."""
    n, d = z.shape
    v = torch.nn.functional.pad(z.double(), (0, -d % 32)).view(n, -1, 32)
    top = v.abs().amax(2, keepdim=True)
    e = torch.floor(torch.log2((top / 127.5).clamp(min=2.0 ** -128)))
    e = torch.where(top >= 127.5 * torch.exp2(e), e + 1, e)
    e = torch.where(top < 127.5 * torch.exp2(e - 1), e - 1, e).clamp(min=-127)
    return (torch.round(v / torch.exp2(e)) * torch.exp2(e)).view(n, -1)[:, :d]


def exact_act(z, kind):
    z = z.detach().requires_grad_(True)
    if kind == "silu":
        y = torch.nn.functional.silu(z)
    elif kind == "gelu":
        y = z * torch.special.ndtr(z)
    else:
        y = torch.tanh(z)
    return y.detach(), torch.autograd.grad(y.sum(), z)[0]


def exact(case, seed):
    """The definitions in 64 bits, the products expert by expert."""
    s = prepare(case, seed)
    op, n = case["op"], case["n"]
    if op == "route":
        z, k = s["logits"].double(), case["k"]
        expert = plain_route(s)[0]
        has, at = expert >= 0, expert.clamp(min=0).long()
        log = torch.log_softmax(z, 1) if case["score"] == "softmax" else torch.nn.functional.logsigmoid(z)
        picked = torch.where(has, log.gather(1, at), -math.inf)
        w = torch.softmax(picked, 1) if case["renorm"] else picked.exp()
        return None, torch.where(has, w, 0.0) * SCALE, None, None, None
    if op == "route_grad":
        z = s["logits"].double()
        dead = (z == -math.inf).all(1)
        z = z.masked_fill(dead[:, None], 0.0).requires_grad_(True)
        has, at = s["expert"] >= 0, s["expert"].clamp(min=0).long()
        score = torch.softmax(z, 1) if case["score"] == "softmax" else torch.sigmoid(z)
        w = score.gather(1, at)
        if case["renorm"]:
            w = w / w.sum(1, keepdim=True)
        return torch.autograd.grad((torch.where(has, w, 0.0) * s["dweight"].double()).sum() * SCALE, z)[0]
    if op in ("product", "product_grad"):
        m, i, o = n * case["k"], case["din"], case["dout"]
        first = s["offset"].tolist()
        if op == "product":
            y = torch.zeros(m, o, dtype=torch.float64, device="cuda")
        else:
            dx = torch.zeros(m, i, dtype=torch.float64, device="cuda")
            dw = torch.zeros(case["experts"], i, o, dtype=torch.float64, device="cuda")
        for e in range(case["experts"]):
            a = slice(first[e], first[e + 1])
            x = (s["x"][a] if s["row"] is None else s["x"][s["row"][a].long()]).double()
            if op == "product":
                y[a] = x @ s["w"][e].double()
            else:
                dy = s["dy"][a].double()
                dx[a] = dy @ s["w"][e].double().t()
                dw[e] = x.t() @ dy
        return y if op == "product" else (dx, dw)
    if op in ("combine", "combine_grad"):
        step = max(1, 2 ** 26 // (case["k"] * case["d"]))
        has, at = s["place"] >= 0, s["place"].clamp(min=0).long()
        out, dweight, dy = [], [], torch.zeros(s["y"].shape[0], case["d"], dtype=torch.float64, device="cuda")
        for i in range(0, n, step):
            a = slice(i, i + step)
            y, w, h = s["y"][at[a]].double(), s["weight"][a].double(), has[a]
            if op == "combine":
                out.append(torch.einsum("nk,nkd->nd", w * h, y))
            else:
                g = s["dout"][a].double()
                dweight.append(torch.einsum("nkd,nd->nk", y, g) * h)
                dy[at[a][h]] = (w[:, :, None] * g[:, None, :])[h]
        return torch.cat(out) if op == "combine" else (dy, torch.cat(dweight))
    z, d = s["z"], case["d"]
    parts = []
    step = max(1, 2 ** 25 // z.shape[1])
    for i in range(0, n, step):
        a = slice(i, i + step)
        if op == "checkpoint":
            parts.append((exact_restored(z[a]),))
            continue
        dy = s["dy"][a].double()
        if case["gated"]:
            y = exact_act(z[a, :d].double(), case["kind"])[0] * z[a, d:].double()
            g, u = exact_restored(z[a, :d]), exact_restored(z[a, d:])
            v, slope = exact_act(g, case["kind"])
            parts.append((y, torch.cat([dy * u * slope, dy * v], 1), v * u))
        else:
            y = exact_act(z[a].double(), case["kind"])[0]
            v, slope = exact_act(exact_restored(z[a]), case["kind"])
            parts.append((y, dy * slope, v))
    got = tuple(torch.cat(p) for p in zip(*parts))
    return got[0] if op == "checkpoint" else got
