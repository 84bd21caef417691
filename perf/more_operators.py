"""Cases of the operators of layers with local attention and of rows that hold images or video: attention inside a packed row's samples with
a sliding window and first tokens that stay visible, its gradient, its form for one token of each sequence against a cache, and the rotation
of queries and keys by positions on several axes, with its gradient.

``own`` says which side ``run`` computes: the plain form (elementary torch operations in 32 bits, angles in 64) or the calls of this
framework's entry points.  Rows, samples' lengths and heads are of the kind that the framework's other cases have; windows, caches and the
sizes of pictures are generic.
"""
import math
import random

import torch

own = False

TYPES = {"bf16": torch.bfloat16, "f16": torch.float16, "f32": torch.float32}
SIZE = {"bf16": 2, "f16": 2, "f32": 4}
EPS = 1e-6
CHUNK = 2048                     # queries that the plain forms take at a time


def listed():
    return [
        # a row of many short samples, a window shorter than most of them, one head of keys to a head of queries
        {"name": "window ragged", "op": "window", "tokens": 4096, "samples": 23, "q": 16, "k": 16, "dim": 64, "window": 128, "sinks": 0, "type": "f16"},
        # a packed row in training, a layer with a window of 1024
        {"name": "window row", "op": "window", "tokens": 32768, "samples": 5, "q": 16, "k": 4, "dim": 128, "window": 1024, "sinks": 4, "type": "bf16"},
        # two long samples of an odd number of tokens, a wide window that is no multiple of a tile
        {"name": "window wide", "op": "window", "tokens": 12289, "samples": 2, "q": 12, "k": 4, "dim": 96, "window": 4001, "sinks": 33, "type": "bf16"},
        # the backward pass of the row
        {"name": "window grad row", "op": "window_grad", "tokens": 16384, "samples": 3, "q": 16, "k": 4, "dim": 128, "window": 1024, "sinks": 4, "type": "bf16"},
        # and of a row of short samples
        {"name": "window grad ragged", "op": "window_grad", "tokens": 3001, "samples": 11, "q": 8, "k": 8, "dim": 64, "window": 200, "sinks": 1, "type": "f16"},
        # one decoding step of a few sequences in a layer with a window
        {"name": "step few", "op": "step", "samples": 4, "room": 6000, "q": 32, "k": 8, "dim": 128, "window": 4096, "sinks": 4, "type": "bf16"},
        # of a batch of ragged sequences in a layer that sees all
        {"name": "step batch", "op": "step", "samples": 64, "room": 6250, "q": 16, "k": 4, "dim": 128, "window": 0, "sinks": 0, "type": "bf16"},
        # of a large batch with a short window, one head of keys to a head of queries
        {"name": "step window", "op": "step", "samples": 250, "room": 2000, "q": 8, "k": 8, "dim": 64, "window": 1000, "sinks": 16, "type": "f16"},
        # decoding: one token of each sequence, behind pictures and text
        {"name": "axes decode", "op": "axes", "tokens": 64, "q": 32, "k": 8, "dim": 128, "rotary": 128, "axes": 3, "order": "blocks", "layout": "half", "norm": True, "type": "bf16"},
        # a packed row of text, pictures and video in training
        {"name": "axes row", "op": "axes", "tokens": 32768, "q": 32, "k": 8, "dim": 128, "rotary": 128, "axes": 3, "order": "turns", "layout": "half", "norm": True, "type": "bf16"},
        # the backward pass of a row, a part of each head rotated, neighbours paired
        {"name": "axes grad row", "op": "axes_grad", "tokens": 16411, "q": 32, "k": 8, "dim": 128, "rotary": 64, "axes": 3, "order": "blocks", "layout": "interleaved", "norm": True, "type": "bf16"},
        # the backward pass of a tower for pictures, in 32 bits: height and width, no norm
        {"name": "axes grad picture", "op": "axes_grad", "tokens": 2501, "q": 16, "k": 16, "dim": 80, "rotary": 80, "axes": 2, "order": "blocks", "layout": "half", "norm": False, "type": "f32"},
    ]


def spread(rng, low, high):
    return int(round(math.exp(rng.uniform(math.log(low), math.log(max(low, high))))))


def draw(rng):
    op = rng.choice(["window", "window_grad", "step", "step", "axes", "axes_grad"])
    if op in ("window", "window_grad"):
        q, k = rng.choice([(16, 4), (16, 16), (8, 2), (12, 4), (5, 1)])
        dim = rng.choice([64, 96, 128])
        # (where a sample is one token, the gradients of its queries and keys are 0, and what is compared would be roundings)
        tokens = spread(rng, 1, 32768) if op == "window" else spread(rng, 100, 16384)
        most = (32768 if op == "window" else 16384) * 1024 * 16 * 128 // (tokens * q * dim)
        return {"op": op, "tokens": tokens, "samples": min(rng.choice([1, 1, 2, 5, 17, 60]), max(1, tokens // 20)), "q": q, "k": k,
                "dim": dim, "window": spread(rng, 16, max(16, min(8192, most))), "sinks": rng.choice([0, 0, 1, 4, 33, 128]), "type": rng.choice(["bf16", "f16"])}
    if op == "step":
        q, k = rng.choice([(32, 8), (16, 4), (8, 8), (5, 1), (40, 2)])
        dim = rng.choice([64, 96, 128])
        samples = spread(rng, 1, 256)
        room = spread(rng, 30, min(131072, 64 * 6250 * 4 * 128 // (samples * k * dim)))
        return {"op": op, "samples": samples, "room": room, "q": q, "k": k, "dim": dim, "window": rng.choice([0, 0, 128, 1000, 4096]),
                "sinks": rng.choice([0, 4, 16, 128]), "type": rng.choice(["bf16", "f16"])}
    q, k = rng.choice([(32, 8), (16, 2), (8, 8), (40, 8), (5, 1)])
    dim = rng.choice([64, 80, 96, 128, 192, 256])
    kind = rng.choice(["bf16", "f16", "f32"])
    most = 32768 * 40 * 128 * 2 // ((q + k) * dim * SIZE[kind] * (2 if op == "axes_grad" else 1))
    return {"op": op, "tokens": spread(rng, 1, min(65536, most)), "q": q, "k": k, "dim": dim, "rotary": rng.choice([dim, dim // 2]), "axes": rng.choice([2, 3, 3, 4]),
            "order": rng.choice(["blocks", "turns"]), "layout": rng.choice(["half", "interleaved"]), "norm": rng.random() < 0.7, "type": kind}


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


def cache_shape(case):
    """(starts of the sequences' rooms in the cache, how many of a room's rows are filled), the same for every seed: lognormal, the rest of a room is
    for the tokens to come."""
    rng = random.Random(case["samples"] * 131 + case["room"])
    weight = [math.exp(rng.gauss(0.0, 0.7)) for _ in range(case["samples"])]
    total, start, length = case["samples"] * case["room"], [0], []
    for w in weight:
        room = max(2, int(total * w / sum(weight)))
        start.append(start[-1] + room)
        length.append(max(1, int(room * rng.uniform(0.6, 1.0))))
    return start, length


def places(case, seed):
    """Positions [axes, tokens]: runs of text, where all axes go on together, between pictures and videos, where each has its own."""
    rng = random.Random(seed * 7919 + case["tokens"])
    n, T = case["axes"], case["tokens"]
    if T <= 256:                                          # one token of each sequence
        return torch.tensor([[at] * n for at in (rng.randrange(100000) for _ in range(T))]).t().contiguous()
    parts, done, at = [], 0, 0
    while done < T:
        text = rng.randrange(20, 200)
        parts.append((at + torch.arange(text)).expand(n, text))
        at += text
        grid = [rng.choice([1, 1, 8])] + [rng.randrange(8, 40) for _ in range(n - 1)] if n > 2 else [rng.randrange(8, 40) for _ in range(n)]
        axes = torch.meshgrid(*[torch.arange(g) for g in grid], indexing="ij")
        parts.append(at + torch.stack([a.reshape(-1) for a in axes]))
        at += max(grid)
        done += text + parts[-1].shape[1]
        if rng.random() < 0.2:
            at = 0                                        # another sample
    return torch.cat(parts, 1)[:, :T].contiguous()


def axis_of_pairs(case):
    half, n = case["rotary"] // 2, case["axes"]
    if case["order"] == "turns":
        return [p % n for p in range(half)]
    first = half // (n + 1) if n > 2 else half // n       # fewer pairs for time than for height and width
    return [0 if p < first else min(n - 1, 1 + (p - first) * (n - 1) // (half - first)) for p in range(half)]


def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    st = {"case": case}
    d = case["dim"]
    kind = TYPES[case["type"]]

    def normal(*shape):
        return torch.randn(*shape, generator=gen, device="cuda")

    if case["op"] in ("window", "window_grad"):
        T = case["tokens"]
        st["spans"] = list(zip(sample_starts(case), sample_starts(case)[1:]))
        st["start"] = torch.tensor(sample_starts(case), device="cuda")
        for name, heads in (("q", case["q"]), ("k", case["k"]), ("v", case["k"])):
            st[name] = normal(T, heads, d).to(kind)
        if case["op"] == "window_grad":
            st["grad"] = normal(T, case["q"], d).to(kind)
            st["out"], st["lse"] = plain_window(st)
        return st
    if case["op"] == "step":
        start, length = cache_shape(case)
        st["spans"] = list(zip(start, length))
        st["start"], st["length"] = torch.tensor(start, device="cuda"), torch.tensor(length, device="cuda")
        st["q"] = normal(case["samples"], case["q"], d).to(kind)
        st["k"], st["v"] = (normal(start[-1], case["k"], d).to(kind) for _ in range(2))
        return st
    T, r = case["tokens"], case["rotary"]
    st["position"] = places(case, seed).cuda()
    st["axis"] = torch.tensor(axis_of_pairs(case), dtype=torch.int32, device="cuda")
    scale = torch.exp(normal(T, 1, 1) * 0.5)
    st["q"] = (normal(T, case["q"], d) * scale).to(kind)
    st["k"] = (normal(T, case["k"], d) * scale).to(kind)
    st["inv_freq"] = 500000.0 ** (-torch.arange(0, r, 2, device="cuda", dtype=torch.float64) / r)
    norm = case["norm"]
    st["q_weight"] = (1 + 0.2 * normal(d)).to(kind) if norm else None
    st["k_weight"] = (1 + 0.2 * normal(d)).to(kind) if norm else None
    if case["op"] == "axes_grad":
        st["q_grad"] = normal(T, case["q"], d).to(kind)
        st["k_grad"] = normal(T, case["k"], d).to(kind)
    return st


# ---- plain forms ------------------------------------------------------------------------
def plain_pieces(st):
    """Pieces of the row whose queries are worked out together: (queries' rows, rows of the keys that they see, which of those each query sees)."""
    c = st["case"]
    window, sinks = c["window"], c["sinks"]
    for lo, hi in st["spans"]:
        for q0 in range(0, hi - lo, CHUNK):
            q1 = min(hi - lo, q0 + CHUNK)
            k0 = max(0, q0 - window + 1)
            j = torch.cat([torch.arange(0, min(sinks, k0), device="cuda"), torch.arange(k0, q1, device="cuda")])
            i = torch.arange(q0, q1, device="cuda")[:, None]
            yield slice(lo + q0, lo + q1), lo + j, (j <= i) & ((j > i - window) | (j < sinks))


def plain_weights(st, rows, keys, seen):
    """Attention weights [heads, queries, keys] of a piece, the log of each row's sum, its queries, and keys and values for each query head."""
    c = st["case"]
    share = c["q"] // c["k"]
    q = st["q"][rows].float().transpose(0, 1)
    k, v = (st[n][keys].float().transpose(0, 1).repeat_interleave(share, 0) for n in ("k", "v"))
    s = torch.matmul(q, k.transpose(1, 2)).mul_(c["dim"] ** -0.5).masked_fill_(~seen, -math.inf)
    top = s.amax(2, keepdim=True)
    p = s.sub_(top).exp_()
    total = p.sum(2, keepdim=True)
    return p.div_(total), (top + torch.log(total)).squeeze(2), q, k, v


def plain_window(st):
    c = st["case"]
    out = torch.empty_like(st["q"])
    lse = torch.empty(c["tokens"], c["q"], device="cuda")
    for rows, keys, seen in plain_pieces(st):
        p, total, _, _, v = plain_weights(st, rows, keys, seen)
        out[rows] = torch.matmul(p, v).transpose(0, 1).to(out.dtype)
        lse[rows] = total.t()
    return out, lse


def plain_window_grad(st):
    c = st["case"]
    T, d, share = c["tokens"], c["dim"], c["q"] // c["k"]
    dq = torch.empty_like(st["q"])
    dk, dv = (torch.zeros(T, c["k"], d, device="cuda") for _ in range(2))
    for rows, keys, seen in plain_pieces(st):
        p, _, q, k, v = plain_weights(st, rows, keys, seen)
        do = st["grad"][rows].float().transpose(0, 1)

        def shared(x):
            return x.view(c["k"], share, -1, d).sum(1).transpose(0, 1)

        dv.index_add_(0, keys, shared(torch.matmul(p.transpose(1, 2), do)))
        ds = torch.matmul(do, v.transpose(1, 2)).sub_((do * torch.matmul(p, v)).sum(2, keepdim=True)).mul_(p)
        dq[rows] = (torch.matmul(ds, k) * d ** -0.5).transpose(0, 1).to(dq.dtype)
        dk.index_add_(0, keys, shared(torch.matmul(ds.transpose(1, 2), q) * d ** -0.5))
    return dq, dk.to(dq.dtype), dv.to(dq.dtype)


def visible(case, length):
    """(first tokens that the newest of `length` sees, first of the last ones that it sees)"""
    first = max(0, length - case["window"]) if case["window"] else 0
    return min(case["sinks"], first), first


def plain_step(st):
    c = st["case"]
    share = c["q"] // c["k"]
    out = torch.empty_like(st["q"])
    lse = torch.empty(c["samples"], c["q"], device="cuda")
    for i, (at, n) in enumerate(st["spans"]):
        sinks, first = visible(c, n)
        k, v = (torch.cat([st[x][at:at + sinks], st[x][at + first:at + n]]).float().transpose(0, 1) for x in ("k", "v"))
        s = torch.matmul(st["q"][i].float().view(c["k"], share, -1), k.transpose(1, 2)) * c["dim"] ** -0.5
        top = s.amax(2, keepdim=True)
        p = torch.exp(s - top)
        total = p.sum(2, keepdim=True)
        out[i] = torch.matmul(p / total, v).view(c["q"], -1).to(out.dtype)
        lse[i] = (top + torch.log(total)).view(-1)
    return out, lse


def plain_angles(st):
    angle = st["position"][st["axis"].long()].t().double() * st["inv_freq"]
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


def plain_axes(st):
    c = st["case"]
    cos, sin = plain_angles(st)

    def one(x, w):
        y = x.float()
        if w is not None:
            y = y * torch.rsqrt((y * y).mean(-1, keepdim=True) + EPS) * w.float()
        return plain_turn(y, cos, sin, c).to(x.dtype)

    return one(st["q"], st["q_weight"]), one(st["k"], st["k_weight"])


def plain_axes_grad(st):
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


PLAIN = {"window": plain_window, "window_grad": plain_window_grad, "step": plain_step, "axes": plain_axes, "axes_grad": plain_axes_grad}


def run(state):
    c = state["case"]
    if not own:
        return PLAIN[c["op"]](state)
    import paper_2608_12146_b200.binding as rp

    if c["op"] == "window":
        return rp.rp_attend_window(state["q"], state["k"], state["v"], state["start"], window=c["window"], sinks=c["sinks"])
    if c["op"] == "window_grad":
        return rp.rp_attend_window_grad(state["grad"], state["q"], state["k"], state["v"], state["out"], state["lse"], state["start"],
                                        window=c["window"], sinks=c["sinks"])
    if c["op"] == "step":
        return rp.rp_attend_step(state["q"], state["k"], state["v"], state["start"], length=state["length"], window=c["window"], sinks=c["sinks"])
    if c["op"] == "axes":
        return rp.rp_rotate_axes(state["q"], state["k"], state["inv_freq"], state["axis"], state["position"], q_weight=state["q_weight"],
                                 k_weight=state["k_weight"], eps=EPS, layout=c["layout"])
    return rp.rp_rotate_axes_grad(state["q_grad"], state["k_grad"], state["q"], state["k"], state["inv_freq"], state["axis"], state["position"],
                                  q_weight=state["q_weight"], k_weight=state["k_weight"], eps=EPS, layout=c["layout"])


def work(case):
    size = SIZE[case["type"]]
    if case["op"] in ("window", "window_grad"):
        start, T, w = sample_starts(case), case["tokens"], case["window"]
        pairs = 0
        for lo, hi in zip(start, start[1:]):
            n, far = hi - lo, max(0, hi - lo - w)         # tokens that do not see all before them, and how many of the first ones each still sees
            sinks, short = min(case["sinks"], far), min(hi - lo, w)
            pairs += short * (short + 1) / 2 + (n - short) * w + sinks * (sinks + 1) / 2 + (far - sinks) * sinks
        q, kv, lse = T * case["q"] * case["dim"] * size, T * case["k"] * case["dim"] * size, T * case["q"] * 4
        if case["op"] == "window":
            return {"bytes": 2 * q + 2 * kv + lse, "flops": 4 * pairs * case["q"] * case["dim"]}
        return {"bytes": 4 * q + 4 * kv + lse, "flops": 10 * pairs * case["q"] * case["dim"]}
    if case["op"] == "step":
        keys = 0
        for n in cache_shape(case)[1]:
            sinks, first = visible(case, n)
            keys += sinks + n - first
        return {"bytes": 2 * keys * case["k"] * case["dim"] * size + case["samples"] * (case["q"] * (2 * case["dim"] * size + 4) + 16),
                "flops": 4 * keys * case["q"] * case["dim"]}
    heads = case["tokens"] * (case["q"] + case["k"]) * case["dim"]
    n = 2 if case["op"] == "axes" else 3 if case["norm"] else 2
    return {"bytes": n * heads * size + case["tokens"] * case["axes"] * 8, "flops": heads * (6 if case["op"] == "axes" else 14)}


# ---- the definitions in 64 bits ---------------------------------------------------------
def exact(case, seed):
    st = prepare(case, seed)
    if case["op"] in ("window", "window_grad"):
        return exact_window(case, st)
    if case["op"] == "step":
        return exact_step(case, st)
    T, r, n = case["tokens"], case["rotary"], case["axes"]
    angle = torch.zeros(T, r // 2, device="cuda", dtype=torch.float64)
    for p, a in enumerate(axis_of_pairs(case)):
        angle[:, p] = st["position"][a].double() * st["inv_freq"][p]
    turn = torch.polar(torch.ones_like(angle), angle)[:, None]

    def forward(x, w):
        if w is not None:
            x = x / (x.square().mean(-1, keepdim=True) + EPS).sqrt() * w
        z = x[..., :r].unflatten(-1, (2, r // 2)).transpose(-1, -2) if case["layout"] == "half" else x[..., :r].unflatten(-1, (r // 2, 2))
        z = torch.view_as_real(torch.view_as_complex(z.contiguous()) * turn)
        z = (z.transpose(-1, -2) if case["layout"] == "half" else z).flatten(-2)
        return torch.cat([z, x[..., r:]], -1)

    if case["op"] == "axes":
        return tuple(forward(st[n].double(), None if st[n + "_weight"] is None else st[n + "_weight"].double()) for n in ("q", "k"))
    dx, dw = [], []
    for n in ("q", "k"):
        x = st[n].double().requires_grad_(True)
        w = None if st[n + "_weight"] is None else st[n + "_weight"].double().requires_grad_(True)
        got = torch.autograd.grad((forward(x, w) * st[n + "_grad"].double()).sum(), [x] if w is None else [x, w])
        dx.append(got[0])
        dw.append(None if w is None else got[1])
    return dx[0], dx[1], dw[0], dw[1]


def exact_window(case, st):
    share, scale, w, sinks = case["q"] // case["k"], 1 / math.sqrt(case["dim"]), case["window"], case["sinks"]
    back = case["op"] == "window_grad"
    x = {n: st[n].double() for n in (("q", "k", "v", "grad") if back else ("q", "k", "v"))}
    out, lse = torch.zeros_like(x["q"]), torch.zeros(case["tokens"], case["q"], device="cuda", dtype=torch.float64)
    dq, dk, dv = torch.zeros_like(x["q"]), torch.zeros_like(x["k"]), torch.zeros_like(x["v"])
    start, step = sample_starts(case), 1500
    for lo, hi in zip(start, start[1:]):
        for a in range(lo, hi, step):
            b = min(hi, a + step)
            near = max(lo, a - w + 1)
            at = list(range(lo, min(lo + sinks, near))) + list(range(near, b))
            at = torch.tensor(at, device="cuda")
            gap = torch.arange(a, b, device="cuda")[:, None] - at            # how far back a key is
            hidden = (gap < 0) | ((gap >= w) & (at - lo >= sinks))
            mask = torch.zeros(b - a, len(at), device="cuda", dtype=torch.float64).masked_fill_(hidden, -math.inf)
            for h in range(case["q"]):
                q, k, v = x["q"][a:b, h], x["k"][at, h // share], x["v"][at, h // share]
                s = q @ k.T * scale + mask
                lse[a:b, h] = torch.logsumexp(s, 1)
                p = torch.softmax(s, 1)
                out[a:b, h] = p @ v
                if back:
                    do = x["grad"][a:b, h]
                    dp = do @ v.T
                    ds = p * (dp - (p * dp).sum(1, keepdim=True))
                    dq[a:b, h] = ds @ k * scale
                    dk[:, h // share].index_add_(0, at, ds.T @ q * scale)
                    dv[:, h // share].index_add_(0, at, p.T @ do)
    return (dq, dk, dv) if back else (out, lse)


def exact_step(case, st):
    share, scale = case["q"] // case["k"], 1 / math.sqrt(case["dim"])
    out = torch.zeros(st["q"].shape, device="cuda", dtype=torch.float64)
    lse = torch.zeros(case["samples"], case["q"], device="cuda", dtype=torch.float64)
    start, length = cache_shape(case)
    for i, n in enumerate(length):
        j = torch.arange(n, device="cuda")
        sees = (j < case["sinks"]) | (j >= n - (case["window"] or n))
        k, v = st["k"][start[i]:start[i] + n][sees].double(), st["v"][start[i]:start[i] + n][sees].double()
        for h in range(case["q"]):
            s = k[:, h // share] @ st["q"][i, h].double() * scale
            lse[i, h] = torch.logsumexp(s, 0)
            out[i, h] = torch.softmax(s, 0) @ v[:, h // share]
    return out, lse
