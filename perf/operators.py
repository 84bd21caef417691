"""Cases of the operators on the tokens of a window: route counts, the router with its balance loss, the rotation of queries and keys in
packed rows and the attention inside their samples, with their gradients.

``own`` says which side ``run`` computes: the plain form (elementary torch operations in 32 bits, angles in 64) or the calls of this
framework's entry points.  Sizes of experts, layers and choices per token are those of the framework's windows; samples' lengths are
lognormal as theirs; head counts and widths are generic.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32,
         "u8": torch.uint8, "i16": torch.int16, "i32": torch.int32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4, "u8": 1, "i16": 2, "i32": 4}
COEF = 0.01
EPS = 1e-6


def listed():
    return [
        # the record of a small window: a few short samples, four layers, kept layer after layer by a trainer
        {"name": "counts small", "op": "counts", "tokens": 5003, "samples": 16, "layers": 4, "experts": 16, "k": 2, "type": "i32", "order": "layer"},
        # the record of a step's window, kept in bytes per token as a serving engine hands it over
        {"name": "counts step", "op": "counts", "tokens": 900001, "samples": 640, "layers": 32, "experts": 128, "k": 8, "type": "u8", "order": "token"},
        # one decoding step of a few sequences
        {"name": "route decode", "op": "route", "tokens": 16, "groups": 1, "experts": 256, "k": 8, "type": "bf16", "score": "sigmoid", "replay": False},
        # a cell of 32768 tokens, loss for each sample, routes chosen
        {"name": "route samples", "op": "route", "tokens": 32768, "groups": 41, "experts": 64, "k": 4, "type": "f32", "score": "softmax", "replay": False},
        # the largest cell of the widest window, the loss over the whole of it
        {"name": "route wide", "op": "route", "tokens": 131072, "groups": 1, "experts": 256, "k": 8, "type": "bf16", "score": "sigmoid", "replay": False},
        # its backward pass, routes replayed as reinforcement learning does, loss for each sample
        {"name": "route grad wide", "op": "route_grad", "tokens": 131072, "groups": 33, "experts": 256, "k": 8, "type": "bf16", "score": "softmax", "replay": True},
        # decoding: one token of each sequence, far into its context
        {"name": "rotate decode", "op": "rotate", "tokens": 64, "samples": 64, "q": 32, "k": 8, "dim": 128, "rotary": 128, "layout": "half", "norm": True, "type": "bf16", "far": 400000},
        # a packed row in training
        {"name": "rotate row", "op": "rotate", "tokens": 32768, "samples": 29, "q": 32, "k": 8, "dim": 128, "rotary": 128, "layout": "half", "norm": True, "type": "bf16", "far": 0},
        # the backward pass of a row, a part of each head rotated, neighbours paired
        {"name": "rotate grad row", "op": "rotate_grad", "tokens": 16411, "samples": 37, "q": 32, "k": 8, "dim": 128, "rotary": 64, "layout": "interleaved", "norm": True, "type": "bf16", "far": 0},
        # a row of many short samples
        {"name": "attend ragged", "op": "attend", "tokens": 4096, "samples": 23, "q": 16, "k": 16, "dim": 64, "causal": True, "type": "f16"},
        # a row of a few long ones, four query heads to a key head
        {"name": "attend long", "op": "attend", "tokens": 12289, "samples": 2, "q": 16, "k": 4, "dim": 128, "causal": True, "type": "bf16"},
        # the backward pass
        {"name": "attend grad", "op": "attend_grad", "tokens": 8192, "samples": 3, "q": 16, "k": 4, "dim": 128, "causal": True, "type": "bf16"},
    ]


def spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(high)))))


def draw(rng):
    op = rng.choice(["counts", "route", "route_grad", "rotate", "rotate_grad", "attend", "attend_grad"])
    if op in ("attend", "attend_grad"):
        q, k = rng.choice([(16, 4), (16, 16), (8, 2), (12, 4), (5, 1)])
        return {"op": op, "tokens": spread(rng, 1, 12289 if op == "attend" else 8192), "samples": rng.choice([1, 1, 2, 5, 17, 60]), "q": q, "k": k,
                "dim": rng.choice([64, 128]), "causal": rng.random() < 0.8, "type": rng.choice(["bf16", "f16"])}
    if op == "counts":
        experts, k = rng.choice([(16, 2), (64, 4), (128, 8), (256, 8)])
        layers = rng.choice([4, 16, 23, 32, 48])
        tokens = spread(rng, 50, 200000000 // (layers * k))
        return {"op": op, "tokens": tokens, "samples": min(tokens, spread(rng, 1, 700)), "layers": layers, "experts": experts, "k": k,
                "type": rng.choice(["u8", "i16", "i32"]) if layers * k * tokens < 50000000 else "u8", "order": rng.choice(["token", "layer"])}
    if op in ("route", "route_grad"):
        experts, k = rng.choice([(16, 2), (60, 4), (64, 4), (128, 8), (160, 6), (256, 8)])
        kind = rng.choice(["bf16", "f16", "f32"])
        tokens = spread(rng, 1, 65536 if kind == "f32" else 131072)
        return {"op": op, "tokens": tokens, "groups": min(tokens, spread(rng, 1, 300)), "experts": experts, "k": k, "type": kind,
                "score": rng.choice(["softmax", "sigmoid"]), "replay": rng.random() < 0.5}
    q, k = rng.choice([(32, 8), (16, 2), (8, 8), (40, 8), (5, 1)])
    dim = rng.choice([64, 80, 96, 128, 192, 256])
    kind = rng.choice(["bf16", "f16", "f32"])
    most = 32768 * 40 * 128 * 2 // ((q + k) * dim * SIZE[kind] * (2 if op == "rotate_grad" else 1))
    tokens = spread(rng, 1, min(65536, most))
    return {"op": op, "tokens": tokens, "samples": min(tokens, spread(rng, 1, 300)), "q": q, "k": k, "dim": dim,
            "rotary": rng.choice([dim, dim // 2]), "layout": rng.choice(["half", "interleaved"]), "norm": rng.random() < 0.7, "type": kind,
            "far": rng.choice([0, 0, 100000, 1000000])}


def cut(gen, tokens, parts):
    """Starts [parts + 1] of samples with lognormal lengths, each of one token at least, that fill `tokens`."""
    weight = torch.exp(torch.randn(parts, generator=gen, device="cuda", dtype=torch.float64) * 1.1)
    inner = torch.floor(torch.cumsum(weight, 0) / weight.sum() * (tokens - parts)).long().clamp(max=tokens - parts)
    start = torch.zeros(parts + 1, dtype=torch.int64, device="cuda")
    start[1:] = inner + torch.arange(1, parts + 1, device="cuda")
    start[parts] = tokens
    return start


def sample_starts(case):
    """Starts of a row's samples, the same for every seed: lengths of a lognormal law, none of no token where the tokens suffice."""
    rng = random.Random(case["tokens"])
    weight = [math.exp(rng.gauss(0.0, 0.8)) for _ in range(case["samples"])]
    spare, start, done = max(0, case["tokens"] - case["samples"]), [0], 0.0
    for i, w in enumerate(weight):
        done += w
        start.append(min(case["tokens"], int(spare * done / sum(weight)) + i + 1))
    start[-1] = case["tokens"]
    return start


def popularity(gen, rows, experts):
    """Skewed shares of experts, another for each row: a few of them take most tokens."""
    return torch.randn(rows, experts, generator=gen, device="cuda") * 1.5


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    T = case["tokens"]
    st = {"case": case}
    if case["op"] == "counts":
        L, E, k = case["layers"], case["experts"], case["k"]
        st["start"] = cut(gen, T, case["samples"])
        shape = (T, L, k) if case["order"] == "token" else (L, T, k)
        cdf = torch.cumsum(torch.softmax(popularity(gen, L, E), 1), 1)
        routes = torch.empty(shape, dtype=TYPES[case["type"]], device="cuda")
        for l in range(L):
            ids = torch.searchsorted(cdf[l], torch.rand(T * k, generator=gen, device="cuda")).clamp(max=E - 1).view(T, k)
            if case["order"] == "token":
                routes[:, l] = ids.to(routes.dtype)
            else:
                routes[l] = ids.to(routes.dtype)
        st["routes"] = routes if case["order"] == "token" else routes.transpose(0, 1)
        return st
    if case["op"] in ("route", "route_grad"):
        E, k = case["experts"], case["k"]
        st["start"] = cut(gen, T, case["groups"])
        x = torch.randn(T, E, generator=gen, device="cuda") + popularity(gen, 1, E)
        st["logits"] = x.to(TYPES[case["type"]])
        other = x + 0.1 * torch.randn(T, E, generator=gen, device="cuda")         # the pass that recorded the routes
        st["routes"] = torch.topk(other, k, dim=1).indices.to(torch.int32).contiguous()
        if case["op"] == "route_grad":
            st["gates_grad"] = torch.randn(T, k, generator=gen, device="cuda")
            st["loss_grad"] = torch.full((1,), float(T), device="cuda")            # a loss summed over tokens
            group = torch.searchsorted(st["start"], torch.arange(T, device="cuda"), right=True) - 1
            st["counts"] = torch.bincount((group[:, None] * E + st["routes"]).reshape(-1), minlength=case["groups"] * E).view(-1, E).to(torch.int32)
        return st
    d = case["dim"]
    kind = TYPES[case["type"]]
    if case["op"] in ("attend", "attend_grad"):
        st["start"] = torch.tensor(sample_starts(case), device="cuda")
        for name, heads in (("q", case["q"]), ("k", case["k"]), ("v", case["k"])):
            st[name] = torch.randn(T, heads, d, generator=gen, device="cuda").to(kind)
        if case["op"] == "attend_grad":
            st["grad"] = torch.randn(T, case["q"], d, generator=gen, device="cuda").to(kind)
            st["out"], st["lse"] = plain_attend(st)
        return st
    r = case["rotary"]
    st["start"] = cut(gen, T, case["samples"])
    st["first"] = torch.randint(0, case["far"], (case["samples"],), generator=gen, device="cuda") if case["far"] else None
    scale = torch.exp(torch.randn(T, 1, 1, generator=gen, device="cuda") * 0.5)
    st["q"] = (torch.randn(T, case["q"], d, generator=gen, device="cuda") * scale).to(kind)
    st["k"] = (torch.randn(T, case["k"], d, generator=gen, device="cuda") * scale).to(kind)
    st["inv_freq"] = 500000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
    norm = case["norm"]
    st["q_weight"] = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(kind) if norm else None
    st["k_weight"] = (1 + 0.2 * torch.randn(d, generator=gen, device="cuda")).to(kind) if norm else None
    if case["op"] == "rotate_grad":
        st["q_grad"] = torch.randn(T, case["q"], d, generator=gen, device="cuda").to(kind)
        st["k_grad"] = torch.randn(T, case["k"], d, generator=gen, device="cuda").to(kind)
    return st


# ---- plain forms ------------------------------------------------------------------------
def owner(start, tokens):
    return torch.searchsorted(start, torch.arange(tokens, device="cuda"), right=True) - 1


def plain_counts(st):
    c = st["case"]
    L, E, N = c["layers"], c["experts"], c["samples"]
    row = owner(st["start"], c["tokens"])[:, None] * L + torch.arange(L, device="cuda")
    at = row[:, :, None] * E + st["routes"]
    return torch.bincount(at.reshape(-1), minlength=N * L * E).view(N, L, E).to(torch.int32)


def plain_scores(x, score):
    s = torch.exp(x - x.amax(1, keepdim=True)) if score == "softmax" else 1 / (1 + torch.exp(-x))
    total = s.sum(1, keepdim=True)
    return (s / total if score == "softmax" else s), s / total, total


def plain_route(st):
    c = st["case"]
    E, G, k, T = c["experts"], c["groups"], c["k"], c["tokens"]
    x = st["logits"].float()
    routes = st["routes"] if c["replay"] else torch.sort(x, dim=1, descending=True, stable=True).indices[:, :k].to(torch.int32)
    s, p, _ = plain_scores(x, c["score"])
    chosen = s.gather(1, routes.long())
    gates = chosen / chosen.sum(1, keepdim=True)
    group = owner(st["start"], T)
    counts = torch.bincount((group[:, None] * E + routes).reshape(-1), minlength=G * E).view(G, E)
    sums = torch.zeros(G, E, device="cuda").index_add_(0, group, p)
    size = (st["start"][1:] - st["start"][:-1]).double()
    loss = (COEF / G * (E / (k * size * size)) * (counts.double() * sums.double()).sum(1)).sum().float().view(1)
    return routes, gates, counts.to(torch.int32), loss


def plain_route_grad(st):
    c = st["case"]
    E, G, k, T = c["experts"], c["groups"], c["k"], c["tokens"]
    s, p, total = plain_scores(st["logits"].float(), c["score"])
    size = (st["start"][1:] - st["start"][:-1]).float()
    b = (st["loss_grad"] * (COEF / G) * E / k / size / size)[:, None] * st["counts"].float()
    b = b[owner(st["start"], T)]
    at = st["routes"].long()
    chosen = s.gather(1, at)
    z = chosen.sum(1, keepdim=True)
    gates = chosen / z
    part = (st["gates_grad"] - (gates * st["gates_grad"]).sum(1, keepdim=True)) / z
    ds = (b - (p * b).sum(1, keepdim=True)) / (1 if c["score"] == "softmax" else total)
    ds = ds.scatter_add(1, at, part)
    return (ds * (s if c["score"] == "softmax" else s * (1 - s))).to(st["logits"].dtype)


def plain_angles(st):
    c = st["case"]
    row = owner(st["start"], c["tokens"])
    position = torch.arange(c["tokens"], device="cuda") - st["start"][row]
    if st["first"] is not None:
        position = position + st["first"][row]
    angle = position.double()[:, None] * st["inv_freq"]
    return torch.cos(angle).float()[:, None], torch.sin(angle).float()[:, None]


def plain_turn(y, cos, sin, c):
    r = c["rotary"]
    head, rest = y[..., :r], y[..., r:]
    if c["layout"] == "half":
        a, b = head[..., : r // 2], head[..., r // 2:]
        head = torch.cat([a * cos - b * sin, a * sin + b * cos], -1)
    else:
        a, b = head[..., 0::2], head[..., 1::2]
        head = torch.stack([a * cos - b * sin, a * sin + b * cos], -1).flatten(-2)
    return torch.cat([head, rest], -1)


def plain_rotate(st):
    c = st["case"]
    cos, sin = plain_angles(st)

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
        return plain_turn(y, cos, sin, c).to(x.dtype)

    return one(st["q"], st["q_weight"]), one(st["k"], st["k_weight"])


def plain_rotate_grad(st):
    c = st["case"]
    cos, sin = plain_angles(st)

    def one(dy, x, w):
        u = plain_turn(dy.float(), cos, -sin, c)
        if w is None:
            return u.to(x.dtype), None
        y = x.float()
        r = torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS)
        hat = y * r
        wu = u * w.float()
        return (r * (wu - hat * (wu * hat).mean(-1, keepdim=True))).to(x.dtype), (u * hat).sum((0, 1))

    dq, dwq = one(st["q_grad"], st["q"], st["q_weight"])
    dk, dwk = one(st["k_grad"], st["k"], st["k_weight"])
    return dq, dk, dwq, dwk


def plain_weights(st):
    """Attention weights [heads, T, T] inside the samples, the log of each row's sum, and keys' and values' heads for each query head."""
    c = st["case"]
    T, share = c["tokens"], c["q"] // c["k"]
    q = st["q"].float().transpose(0, 1)
    k, v = (st[n].float().transpose(0, 1).repeat_interleave(share, 0) for n in ("k", "v"))
    sample = owner(st["start"], T)
    seen = sample[:, None] == sample
    if c["causal"]:
        seen &= torch.ones(T, T, dtype=torch.bool, device="cuda").tril_()
    s = torch.matmul(q, k.transpose(1, 2)).mul_(c["dim"] ** -0.5).masked_fill_(~seen, -math.inf)
    top = s.amax(2, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(2, keepdim=True)
    return p.div_(total), (top + torch.log(total)).squeeze(2), q, k, v


def plain_attend(st):
    p, lse, _, _, v = plain_weights(st)
    return torch.matmul(p, v).transpose(0, 1).to(st["q"].dtype).contiguous(), lse.transpose(0, 1).contiguous()


def plain_attend_grad(st):
    c = st["case"]
    p, _, q, k, v = plain_weights(st)
    do = st["grad"].float().transpose(0, 1)
    dv = torch.matmul(p.transpose(1, 2), do)
    ds = torch.matmul(do, v.transpose(1, 2)).sub_((do * torch.matmul(p, v)).sum(2, keepdim=True)).mul_(p)
    dq = torch.matmul(ds, k) * c["dim"] ** -0.5
    dk = torch.matmul(ds.transpose(1, 2), q) * c["dim"] ** -0.5

    def shared(x):
        return x.view(c["k"], -1, c["tokens"], c["dim"]).sum(1).transpose(0, 1)

    return tuple(x.to(st["q"].dtype).contiguous() for x in (dq.transpose(0, 1), shared(dk), shared(dv)))


PLAIN = {"attend": plain_attend, "attend_grad": plain_attend_grad, "counts": plain_counts, "route": plain_route, "route_grad": plain_route_grad, "rotate": plain_rotate, "rotate_grad": plain_rotate_grad}


def run(state):
    c = state["case"]
    if not own:
        return PLAIN[c["op"]](state)
    import paper_2608_12146_b200.binding as rp

    if c["op"] == "counts":
        return rp.rp_count_routes(state["routes"], state["start"], c["experts"])
    if c["op"] == "route":
        return rp.rp_route(state["logits"], c["k"], state["start"], score=c["score"], normalise=True, loss_coef=COEF,
                           replay=state["routes"] if c["replay"] else None)
    if c["op"] == "route_grad":
        return rp.rp_route_grad(state["logits"], state["routes"], state["start"], state["counts"], gates_grad=state["gates_grad"],
                                loss_grad=state["loss_grad"], score=c["score"], normalise=True, loss_coef=COEF)
    if c["op"] == "attend":
        return rp.rp_attend(state["q"], state["k"], state["v"], state["start"], causal=c["causal"])
    if c["op"] == "attend_grad":
        return rp.rp_attend_grad(state["grad"], state["q"], state["k"], state["v"], state["out"], state["lse"], state["start"], causal=c["causal"])
    if c["op"] == "rotate":
        return rp.rp_rotate(state["q"], state["k"], state["inv_freq"], state["start"], first_position=state["first"],
                            q_weight=state["q_weight"], k_weight=state["k_weight"], eps=EPS, layout=c["layout"])
    return rp.rp_rotate_grad(state["q_grad"], state["k_grad"], state["q"], state["k"], state["inv_freq"], state["start"],
                             first_position=state["first"], q_weight=state["q_weight"], k_weight=state["k_weight"], eps=EPS, layout=c["layout"])


def work(case):
    T, size = case["tokens"], SIZE[case["type"]]
    if case["op"] == "counts":
        picks = T * case["layers"] * case["k"]
        return {"bytes": picks * size + case["samples"] * (case["layers"] * case["experts"] * 4 + 8), "flops": picks}
    if case["op"] in ("route", "route_grad"):
        E, k, G = case["experts"], case["k"], case["groups"]
        if case["op"] == "route":
            return {"bytes": T * E * size + T * k * 8 + G * (E * 4 + 8), "flops": T * E * 5}
        return {"bytes": 2 * T * E * size + T * k * 8 + G * (E * 4 + 8), "flops": T * E * 8}
    if case["op"] in ("attend", "attend_grad"):
        start = sample_starts(case)
        pairs = sum((hi - lo) * ((hi - lo + 1) / 2 if case["causal"] else hi - lo) for lo, hi in zip(start, start[1:]))
        q, kv, lse = T * case["q"] * case["dim"] * size, T * case["k"] * case["dim"] * size, T * case["q"] * 4
        if case["op"] == "attend":
            return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * pairs * case["q"] * case["dim"]}
        return {"bytes": 4 * q + 4 * kv + lse, "flops": 10 * pairs * case["q"] * case["dim"]}
    heads = T * (case["q"] + case["k"]) * case["dim"]
    n = 2 if case["op"] == "rotate" else 3
    return {"bytes": n * heads * size + case["samples"] * 8, "flops": heads * (6 if n == 2 else 14)}


# ---- the definitions in 64 bits ---------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    T = case["tokens"]
    if case["op"] == "counts":
        return None                                    # whole numbers
    start = st["start"].tolist()
    if case["op"] in ("route", "route_grad"):
        E, k, G = case["experts"], case["k"], case["groups"]
        x = st["logits"].double()
        s = torch.softmax(x, 1) if case["score"] == "softmax" else torch.sigmoid(x)
        p = s / s.sum(1, keepdim=True)
        if case["op"] == "route":
            ids = st["routes"].long() if case["replay"] else torch.argsort(-x, dim=1, stable=True)[:, :k]
            hit = torch.zeros(T, E, device="cuda", dtype=torch.float64).scatter_add_(1, ids, torch.ones(T, k, device="cuda", dtype=torch.float64))
            g = torch.take_along_dim(s, ids, 1)
            loss = 0.0
            for lo, hi in zip(start, start[1:]):
                f = hit[lo:hi].sum(0) * E / (k * (hi - lo))
                loss = loss + (f * p[lo:hi].mean(0)).sum()
            return None, g / g.sum(1, keepdim=True), None, (COEF / G * loss).view(1)
        x.requires_grad_(True)
        s = torch.softmax(x, 1) if case["score"] == "softmax" else torch.sigmoid(x)
        p = s / s.sum(1, keepdim=True)
        g = torch.take_along_dim(s, st["routes"].long(), 1)
        value = (g / g.sum(1, keepdim=True) * st["gates_grad"].double()).sum()
        for i, (lo, hi) in enumerate(zip(start, start[1:])):
            f = st["counts"][i].double() * E / (k * (hi - lo))
            value = value + st["loss_grad"].double()[0] * COEF / G * (f * p[lo:hi].mean(0)).sum()
        return torch.autograd.grad(value, x)[0]
    if case["op"] in ("attend", "attend_grad"):
        return exact_attention(case, st, start)
    r = case["rotary"]
    position = torch.cat([torch.arange(hi - lo, device="cuda") for lo, hi in zip(start, start[1:])]).double()
    if st["first"] is not None:
        position += torch.repeat_interleave(st["first"], st["start"].diff()).double()
    turn = torch.polar(torch.ones(T, r // 2, device="cuda", dtype=torch.float64), position[:, None] * st["inv_freq"])[:, None]

    def forward(x, w):
        if w is not None:
            x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w
        z = x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else x[..., :r].unflatten(-1, (r // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        z = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
        return torch.cat([z, x[..., r:]], -1)

    if case["op"] == "rotate":
        return tuple(forward(st[n].double(), None if st[n + "_weight"] is None else st[n + "_weight"].double()) for n in ("q", "k"))
    dx, dw = [], []
    for n in ("q", "k"):
        x = st[n].double().requires_grad_(True)
        w = None if st[n + "_weight"] is None else st[n + "_weight"].double().requires_grad_(True)
        got = torch.autograd.grad((forward(x, w) * st[n + "_grad"].double()).sum(), [x] if w is None else [x, w])
        dx.append(got[0])
        dw.append(None if w is None else got[1])
    return dx[0], dx[1], dw[0], dw[1]


def exact_attention(case, st, start):
    share, scale = case["q"] // case["k"], 1 / math.sqrt(case["dim"])
    back = case["op"] == "attend_grad"
    x = {n: st[n].double() for n in (("q", "k", "v", "grad") if back else ("q", "k", "v"))}
    out, lse = torch.empty_like(x["q"]), torch.empty(case["tokens"], case["q"], device="cuda", dtype=torch.float64)
    dq, dk, dv = torch.zeros_like(x["q"]), torch.zeros_like(x["k"]), torch.zeros_like(x["v"])
    for lo, hi in zip(start, start[1:]):
        for h in range(case["q"]):
            q, k, v = x["q"][lo:hi, h], x["k"][lo:hi, h // share], x["v"][lo:hi, h // share]
            s = q @ k.T * scale
            if case["causal"]:
                s += torch.full_like(s, -math.inf).triu(1)
            lse[lo:hi, h] = torch.logsumexp(s, 1)
            p = torch.softmax(s, 1)
            out[lo:hi, h] = p @ v
            if back:
                do = x["grad"][lo:hi, h]
                dp = do @ v.T
                ds = p * (dp - (p * dp).sum(1, keepdim=True))
                dq[lo:hi, h] = ds @ k * scale
                dk[lo:hi, h // share] += ds.T @ q * scale
                dv[lo:hi, h // share] += p.T @ do
    return (dq, dk, dv) if back else (out, lse)
