"""Router with its balance loss and gradient, against the formulas in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp


def reference(x, k, start, score="softmax", normalise=True, scale=1.0, coef=0.0, bias=None, replay=None):
    """(routes, gates, counts, loss) in 64 bits from logits [T, E]; tokens of no group: -1, 0."""
    import torch
    x = x.double().cpu()
    T, E = x.shape
    G = len(start) - 1
    group = torch.full((T,), -1)
    for g in range(G):
        group[max(start[g], 0):max(min(start[g + 1], T), 0)] = g
    if score == "softmax":
        top = x.amax(1, keepdim=True)
        s = torch.exp(x - torch.where(torch.isinf(top), torch.zeros_like(top), top))
        total = s.sum(1, keepdim=True)
        s = torch.where(total > 0, s / torch.where(total > 0, total, torch.ones_like(total)), s * 0)
    else:
        s = torch.sigmoid(x)
    total = s.sum(1, keepdim=True)
    p = torch.where(total > 0, s / torch.where(total > 0, total, torch.ones_like(total)), s * 0)
    if replay is None:
        order = x if bias is None else s + bias.double().cpu()
        routes = torch.argsort(-order, dim=1, stable=True)[:, :k].clone()
        routes[group < 0] = -1
    else:
        routes = replay.long().cpu()
    valid = (routes >= 0) & (routes < E) & (group[:, None] >= 0)
    chosen = torch.where(valid, s.gather(1, routes.clamp(0, E - 1)), torch.zeros(1, dtype=torch.float64))
    gates = chosen
    if normalise:
        z = chosen.sum(1, keepdim=True)
        gates = torch.where(z > 0, chosen / torch.where(z > 0, z, torch.ones_like(z)), chosen * 0)
    counts = torch.zeros(G, E, dtype=torch.float64)
    for t in range(T):
        for e in routes[t][valid[t]].tolist():
            counts[group[t], e] += 1
    loss = torch.zeros((), dtype=torch.float64)
    for g in range(G):
        n = int((group == g).sum())
        if n:
            loss = loss + coef / G * E / (k * n * n) * (counts[g] * p[group == g].sum(0)).sum()
    return routes, gates * scale, counts, loss


def logits_of(T, E, dtype, seed, spread=1.5):
    import torch
    g = torch.Generator().manual_seed(seed)
    return (torch.randn(T, E, generator=g) * spread + torch.randn(1, E, generator=g)).clamp(-14, 14).to(dtype)


# (ex2 and the sums of a row in 32 bits, |x| <= 14: arguments to 41 give 41 * 2^-25 * ln 2 + 41 * 1.3e-8 * ln 2, ex2 2^-22, sums 20 * 2^-24, a division)
FLOAT = 4e-6


def test_refusals():
    lib = rp.lib()
    buf = np.zeros(4096, np.float64)
    p = buf.ctypes.data

    def r(E=8, k=2, kind=0, score=0, norm=1):
        return C.byref(rp.rp_router(E, k, kind, score, norm, 1.0, 0.1))

    def fwd(router=r(), x=p, T=2, start=p, G=1, replay=0, routes=p, size=4, step=2, gates=p, counts=p, loss=p, space=p, nbytes=1 << 14):
        return lib.rp_route(router, x, 8, T, None, start, G, replay, routes, size, step, gates, counts, loss, space, nbytes, None)

    assert fwd() == -1                                   # host arrays
    for bad in (dict(router=None), dict(x=None), dict(start=None), dict(routes=None), dict(gates=None), dict(T=-1), dict(G=0), dict(size=3),
                dict(counts=None), dict(space=None), dict(nbytes=8), dict(replay=2), dict(step=1), dict(x=p + 1), dict(start=p + 4),
                dict(space=p + 8), dict(router=r(E=0)), dict(router=r(k=9)), dict(router=r(k=0)), dict(router=r(kind=3)), dict(router=r(score=2)),
                dict(router=r(norm=2))):
        assert fwd(**bad) == -1, bad
    assert fwd(router=r(E=1025)) == -5 and fwd(router=r(E=64, k=33), step=33) == -5 and fwd(T=(1 << 26) + 1) == -5
    assert fwd(router=r(E=512), size=1) == -5            # ids do not fit
    assert lib.rp_route_workspace(None, 1) == 0 and lib.rp_route_workspace(r(), 0) == 0 and lib.rp_route_workspace(r(), 3) > 3 * 8 * 8

    def bwd(router=r(), x=p, T=2, routes=p, dg=p, dl=p, start=p, counts=p, dx=p + 8192, gstep=8):
        return lib.rp_route_grad(router, x, 8, T, routes, 4, 2, dg, dl, start, 1, counts, dx, gstep, None)

    assert bwd() == -1
    for bad in (dict(router=None), dict(x=None), dict(dx=None), dict(routes=None), dict(counts=None), dict(dx=p), dict(gstep=7), dict(start=None)):
        assert bwd(**bad) == -1, bad


SHAPES = [
    # tokens, experts, k, starts
    (1, 1, 1, [0, 1]), (1, 16, 2, [0, 1]), (5, 16, 5, [0, 5]), (16, 256, 8, [0, 16]), (33, 60, 4, [0, 10, 10, 33]), (257, 64, 4, [5, 100, 250]),
    (300, 128, 8, list(range(0, 301, 4))), (77, 160, 6, [0, 40, 77]), (700, 32, 1, [0, 1, 699, 700]), (150, 256, 8, [-4, 100, 200]), (40, 300, 32, [0, 40]),
    (41, 1000, 9, [0, 20, 41]), (35, 512, 8, [0, 35]), (2000, 256, 8, [0, 1000, 2000]), (4000, 24, 3, [0, 4000]), (1200, 8, 8, [0, 300, 1200]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("score,normalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(s[:3]) for s in SHAPES])
def test_chosen_routes_gates_counts_and_loss(shape, kind, score, normalise):
    import torch
    T, E, k, start = shape
    x = logits_of(T, E, getattr(torch, kind), T + E)
    want = reference(x, k, start, score, normalise, 2.5, 0.3)
    routes, gates, counts, loss = rp.rp_route(x.cuda(), k, torch.tensor(start, device="cuda"), score=score, normalise=normalise, scale=2.5, loss_coef=0.3)
    assert (routes.cpu().long() == want[0]).all()
    assert (counts.cpu().double() == want[2]).all()
    assert ((gates.cpu().double() - want[1]).abs() <= FLOAT * want[1]).all()
    assert abs(loss.item() - want[3].item()) <= 2 * FLOAT * want[3].item()


@pytest.mark.gpu
@pytest.mark.parametrize("score,normalise", [("softmax", True), ("softmax", False), ("sigmoid", True), ("sigmoid", False)])
@pytest.mark.parametrize("kind,route_kind", [("float32", "int64"), ("float16", "uint8"), ("bfloat16", "int16")])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(s[:3]) for s in SHAPES])
def test_replayed_routes_and_gradients(shape, kind, route_kind, score, normalise):
    """Routes from a record with empty places and an expert twice; gradients against the formulas' derivatives in 64 bits."""
    import torch
    T, E, k, start = shape
    if route_kind == "uint8" and E > 250:
        pytest.skip("ids do not fit a byte")
    dtype = getattr(torch, kind)
    g = torch.Generator().manual_seed(T * 7 + E)
    ids = torch.randint(0, E, (T, k), generator=g)
    if k > 1:
        ids[::3, 1] = ids[::3, 0]                        # the same expert twice
    ids[torch.rand(T, k, generator=g) < 0.1] = 255 if route_kind == "uint8" else -1
    record = torch.zeros(T, 3, k, dtype=getattr(torch, route_kind), device="cuda")
    record[:, 1] = ids.to(record.dtype).cuda()
    replay = record[:, 1]                                # a layer's slice of the record
    x = logits_of(T, E, dtype, T + E + 1)
    wide = torch.full((T, E + 8), 3.0, dtype=dtype, device="cuda")
    xd = wide[:, :E]
    xd.copy_(x)
    st = torch.tensor(start, device="cuda")
    kw = dict(score=score, normalise=normalise, scale=1.5, loss_coef=0.7)
    routes, gates, counts, loss = rp.rp_route(xd, k, st, replay=replay, **kw)
    x64 = x.double().requires_grad_(True)
    _, w_gates, w_counts, w_loss = reference(x64, k, start, score, normalise, 1.5, 0.7, replay=ids)
    assert routes.data_ptr() == replay.data_ptr() and (replay.cpu().long() == ids).all()
    assert (counts.cpu().double() == w_counts).all()
    assert ((gates.cpu().double() - w_gates).abs() <= FLOAT * w_gates).all()
    assert abs(loss.item() - w_loss.item()) <= 2 * FLOAT * w_loss.item()

    dg = torch.randn(T, k, generator=g)
    dl = torch.tensor([float(T)])
    group_size = np.array([max(0, min(b, T) - max(a, 0)) for a, b in zip(start, start[1:])])
    b_top = max([0.0] + [T * 0.7 / (len(start) - 1) * E * w_counts[i].max().item() / (k * n * n) for i, n in enumerate(group_size) if n])
    for use_g, use_l in ((True, True), (True, False), (False, True)):
        value = (w_gates * dg.double()).sum() * use_g + w_loss * dl.double()[0] * use_l
        want, = torch.autograd.grad(value, x64, retain_graph=True)
        got = rp.rp_route_grad(xd, replay, st, counts, gates_grad=dg.cuda() if use_g else None, loss_grad=dl.cuda() if use_l else None, **kw)
        # rounded once; terms up to the largest gate's gradient and the largest slope of the loss, each with the scores' error, cancel
        tol = torch.finfo(dtype).eps / 2 * want.abs() + 4 * FLOAT * ((1.5 * dg.abs().amax(1, keepdim=True)).double() * use_g * k + b_top * use_l) + 1e-7 * (kind == "float16")
        assert got.dtype == dtype and ((got.cpu().double() - want).abs() <= tol).all(), (use_g, use_l)
    assert (wide[:, E:] == 3.0).all()


@pytest.mark.gpu
def test_gradient_against_differences():
    import torch
    T, E, k, start = 6, 12, 3, [0, 2, 6]
    x = logits_of(T, E, torch.float32, 5)
    ids = torch.topk(x, k, dim=1).indices
    dg = torch.randn(T, k, generator=torch.Generator().manual_seed(1), dtype=torch.float64)
    st = torch.tensor(start, device="cuda")
    for score in ("softmax", "sigmoid"):
        def value(z):
            _, gates, _, loss = reference(z, k, start, score, True, 1.0, 0.5, replay=ids)
            return (gates * dg).sum() + 3.0 * loss
        _, _, counts, _ = rp.rp_route(x.cuda(), k, st, replay=ids.cuda(), score=score, loss_coef=0.5)
        got = rp.rp_route_grad(x.cuda(), ids.cuda(), st, counts, gates_grad=dg.float().cuda(), loss_grad=torch.tensor([3.0], device="cuda"), score=score,
                               loss_coef=0.5).cpu().double()
        z, h = x.double(), 1e-5
        for t in range(T):
            for e in range(E):
                up, down = z.clone(), z.clone()
                up[t, e] += h
                down[t, e] -= h
                assert abs((value(up) - value(down)).item() / (2 * h) - got[t, e].item()) < 2e-5


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
def test_ties_go_to_the_lowest_expert(kind):
    import torch
    dtype = getattr(torch, kind)
    x = torch.zeros(40, 100, dtype=dtype)
    x[1] = torch.arange(100).flip(0) // 10               # ten of each number
    x[2, 50:] = 1
    x[3, ::2] = -0.0                                     # -0 and 0 are one number
    x[4] = -float("inf")
    x[4, 90:93] = 0
    x[5] = -float("inf")                                 # nothing left: the first experts, gates 0
    want = torch.argsort(-(x.double() + 0.0), dim=1, stable=True)[:, :8]
    for score in ("softmax", "sigmoid"):
        routes, gates, counts, loss = rp.rp_route(x.cuda(), 8, torch.tensor([0, 40], device="cuda"), score=score, loss_coef=1.0)
        assert (routes.cpu().long() == want).all()
        assert torch.isfinite(gates).all() and (gates[5] == 0).all() and (gates[4, 3:] == 0).all() and torch.isfinite(loss).all()
        grad = rp.rp_route_grad(x.cuda(), routes, torch.tensor([0, 40], device="cuda"), counts, gates_grad=torch.ones_like(gates),
                                loss_grad=torch.ones(1, device="cuda"), score=score, loss_coef=1.0)
        assert torch.isfinite(grad).all() and (grad[5] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
@pytest.mark.parametrize("E,k", [(16, 3), (64, 8), (256, 8), (600, 12)])
def test_bias_moves_the_choice_alone(E, k, score):
    import torch
    T = 200
    x = logits_of(T, E, torch.bfloat16, E)
    bias = torch.randn(E, generator=torch.Generator().manual_seed(2))
    want = reference(x, k, [0, T], score, bias=bias)
    routes, gates, counts, _ = rp.rp_route(x.cuda(), k, torch.tensor([0, T], device="cuda"), score=score, choice_bias=bias.cuda())
    s = torch.softmax(x.double(), 1) if score == "softmax" else torch.sigmoid(x.double())
    total = s + bias.double()
    # the k largest up to the rounding of scores and sums in 32 bits
    got = total.gather(1, routes.cpu().long())
    assert ((got - total.gather(1, want[0])).abs() <= FLOAT + 2.0 ** -23 * total.abs().amax()).all()
    assert all(len(set(r)) == k for r in routes.tolist())
    chosen = s.gather(1, routes.cpu().long())
    assert ((gates.cpu().double() - chosen / chosen.sum(1, keepdim=True)).abs() <= FLOAT).all()
    assert (counts.cpu() == torch.bincount(routes.cpu().long().flatten(), minlength=E)).all()


@pytest.mark.gpu
def test_numbers_that_are_none_stay_in_their_row():
    import torch
    x = logits_of(64, 48, torch.float32, 9)
    clean = rp.rp_route(x.cuda(), 4, torch.tensor([0, 60], device="cuda"), loss_coef=1.0)
    x[7, 3], x[9, 5], x[62] = float("nan"), float("inf"), float("nan")          # 62 is in no group
    routes, gates, counts, loss = rp.rp_route(x.cuda(), 4, torch.tensor([0, 60], device="cuda"), loss_coef=1.0)
    rows = [t for t in range(64) if t not in (7, 9)]
    assert (routes[rows] == clean[0][rows]).all() and (gates[rows] == clean[1][rows]).all()
    assert ((routes[[7, 9]] >= 0) & (routes[[7, 9]] < 48)).all() and torch.isnan(loss).all() and torch.isnan(gates[7]).all()
    assert counts.sum().item() == 240 and (routes[60:] == -1).all() and (gates[60:] == 0).all()
    grad = rp.rp_route_grad(x.cuda(), routes, torch.tensor([0, 60], device="cuda"), counts, gates_grad=torch.ones_like(gates))
    assert torch.isfinite(grad[rows]).all() and (grad[60:] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float16", "bfloat16"])
def test_order_of_every_16_bit_number(kind):
    """All bit patterns in rows of 64 neighbours of a shuffled list: falling order, NaN of either sign above all, subnormal numbers apart."""
    import torch
    bits = torch.randperm(1 << 16, generator=torch.Generator().manual_seed(4)).to(torch.int32)
    x = (bits - (1 << 15)).to(torch.int16).view(getattr(torch, kind)).view(-1, 64)
    place = torch.where(x.isnan(), math.inf, x.double().clamp(-1e300, 1e300))
    want = torch.argsort(-(place + 0.0), dim=1, stable=True)[:, :8]
    routes, _, counts, _ = rp.rp_route(x.cuda(), 8, torch.tensor([0, len(x)], device="cuda"), score="sigmoid")
    assert (routes.cpu().long() == want).all() and counts.sum().item() == 8 * len(x)


@pytest.mark.gpu
def test_routes_go_into_a_record_and_rows_behind_stay():
    import torch
    x = logits_of(100, 256, torch.bfloat16, 3).cuda()
    start = torch.tensor([0, 50, 100], device="cuda")
    want = rp.rp_route(x, 8, start)[0]
    record = torch.full((110, 3, 8), 77, dtype=torch.uint8, device="cuda")
    gates = torch.full((110, 8), 5.0, device="cuda")
    rp.rp_route(x, 8, start, routes=record[:100, 1], gates=gates[:100])
    assert (record[:100, 1].int() == want).all() and (record[:, 0] == 77).all() and (record[:, 2] == 77).all() and (record[100:] == 77).all()
    assert (gates[100:] == 5).all()
    out = torch.full((110, 256), 9.0, dtype=torch.bfloat16, device="cuda")
    rp.rp_route_grad(x, record[:100, 1], start, torch.zeros(2, 256, dtype=torch.int32, device="cuda"), gates_grad=gates[:100], logits_grad=out[:100])
    assert (out[100:] == 9).all() and torch.isfinite(out).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T", [16, 5000])
def test_repeated_streamed_and_captured_calls_agree_bit_for_bit(T):
    import torch
    x = logits_of(T, 256, torch.bfloat16, 4).cuda()
    start = torch.tensor([0, T // 3, T], device="cuda")
    kw = dict(score="sigmoid", loss_coef=0.1)
    want = rp.rp_route(x, 8, start, **kw)
    dg, dl = torch.randn_like(want[1]), torch.ones(1, device="cuda")
    want_dx = rp.rp_route_grad(x, want[0], start, want[2], gates_grad=dg, loss_grad=dl, **kw)
    torch.cuda.synchronize()
    side = [torch.cuda.Stream() for _ in range(4)]
    results = [(rp.rp_route(x, 8, start, stream=s, **kw), rp.rp_route_grad(x, want[0], start, want[2], gates_grad=dg, loss_grad=dl, stream=s, **kw))
               for s in side for _ in range(5)]
    torch.cuda.synchronize()
    for got, dx in results:
        assert all((a == b).all() for a, b in zip(got, want)) and (dx == want_dx).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = rp.rp_route(x, 8, start, **kw)
        dx = rp.rp_route_grad(x, got[0], start, got[2], gates_grad=dg, loss_grad=dl, **kw)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all((a == b).all() for a, b in zip(got, want)) and (dx == want_dx).all()


@pytest.mark.gpu
def test_no_tokens():
    import torch
    x = torch.zeros(0, 16, device="cuda")
    routes, gates, counts, loss = rp.rp_route(x, 2, torch.tensor([0, 0], device="cuda"), loss_coef=1.0)
    assert routes.shape == (0, 2) and (counts == 0).all() and loss.item() == 0
    assert rp.rp_route_grad(x, routes, torch.tensor([0, 0], device="cuda"), counts, gates_grad=gates).shape == (0, 16)


@pytest.mark.gpu
@pytest.mark.parametrize("T", [5, 3000])
def test_outputs_that_may_be_left_out(T):
    import torch
    x = torch.randn(T, 64, generator=torch.Generator().manual_seed(T)).bfloat16().cuda()
    start = torch.tensor([0, T // 2, T], device="cuda")
    want = rp.rp_route(x, 4, start)
    cfg, stream = C.byref(rp.rp_router(64, 4, 2, 0, 1, 1.0, 0.0)), torch.cuda.current_stream().cuda_stream
    for with_counts in (False, True):
        routes, gates, counts = torch.full((T, 4), 9, dtype=torch.int32, device="cuda"), torch.zeros(T, 4, device="cuda"), torch.full((2, 64), 7, dtype=torch.int32, device="cuda")
        assert rp.lib().rp_route(cfg, x.data_ptr(), 64, T, None, start.data_ptr(), 2, 0, routes.data_ptr(), 4, 4, gates.data_ptr(),
                                 counts.data_ptr() if with_counts else None, None, None, 0, stream) == 0
        assert (routes == want[0]).all() and (gates == want[1]).all() and (counts == (want[2] if with_counts else 7)).all()


@pytest.mark.gpu
def test_rows_that_repeat_or_run_backwards():
    import torch
    x = torch.randn(50, 40, generator=torch.Generator().manual_seed(2)).cuda()
    start = torch.tensor([0, 20, 50], device="cuda")
    same = x[:1].expand(50, 40)
    assert all((a == b).all() for a, b in zip(rp.rp_route(same, 3, start, loss_coef=0.1), rp.rp_route(same.contiguous(), 3, start, loss_coef=0.1)))
    want = rp.rp_route(x.flip(0), 3, start)
    cfg, stream = C.byref(rp.rp_router(40, 3, 0, 0, 1, 1.0, 0.0)), torch.cuda.current_stream().cuda_stream
    routes, gates = torch.zeros(50, 3, dtype=torch.int32, device="cuda"), torch.zeros(50, 3, device="cuda")
    assert rp.lib().rp_route(cfg, x[49:].data_ptr(), -40, 50, None, start.data_ptr(), 2, 0, routes.data_ptr(), 4, 3, gates.data_ptr(), None, None, None, 0, stream) == 0
    assert (routes == want[0]).all() and (gates == want[1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("E,k", [(16, 2), (64, 4), (300, 8)])
def test_many_groups_in_runs_of_many_shapes(E, k):
    """Groups that end inside, between and across the runs of a CTA; as many as take a launch of their own for the loss."""
    import torch
    T = 6000
    x = torch.randn(T, E, generator=torch.Generator().manual_seed(E)).cuda()
    for cuts in ([0, 1, 2, 3, 2000, 2001, 5000, T], list(range(0, T + 1, 7)) + [T], [0] * 18 + [3000] * 5 + [T], [100, 4000, 4001]):
        start = torch.tensor(cuts, device="cuda")
        routes, _, counts, loss = rp.rp_route(x, k, start, loss_coef=0.5)
        p = torch.softmax(x.double(), 1)
        want, total = torch.zeros(len(cuts) - 1, E, dtype=torch.int64), 0.0
        for i, (lo, hi) in enumerate(zip(cuts, cuts[1:])):
            if hi > lo:
                want[i] = torch.bincount(routes[lo:hi].reshape(-1).long(), minlength=E).cpu()
                total += E / (k * (hi - lo) ** 2) * (want[i].double().cuda() * p[lo:hi].sum(0)).sum().item()
        assert (counts.cpu() == want).all()
        # (p to FLOAT of itself, sums of a run and of a CTA in 32 bits: 40 terms)
        assert abs(loss.item() - 0.5 / (len(cuts) - 1) * total) <= (2 * FLOAT + 40 * 2.0 ** -24) * 0.5 / (len(cuts) - 1) * total


@pytest.mark.gpu
@pytest.mark.parametrize("constant", [0.0, 0.25])
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("E,k", [(16, 3), (64, 8), (256, 8), (600, 12)])
def test_equal_logits_under_one_bias_are_ties(E, k, kind, constant):
    """Sigmoid scores of logits in steps of 1/8 up to 8: neighbours are 4e-5 apart, so a bias that all have alike chooses what none does."""
    import torch
    x = (torch.randn(500, E, generator=torch.Generator().manual_seed(E)) * 16).round().clamp(-64, 64) / 8
    x[::7, 1] = x[::7, 0]
    x[3, 5] = float("nan")                               # counts as largest, and its neighbours by their own scores
    x[4, 2], x[4, 11] = float("nan"), float("nan")
    x = x.to(getattr(torch, kind))
    want = torch.argsort(-torch.where(x.isnan(), math.inf, x.double()), dim=1, stable=True)[:, :k]
    start = torch.tensor([0, 200, 500], device="cuda")
    bias = torch.full((E,), constant, device="cuda")
    routes, gates, counts, _ = rp.rp_route(x.cuda(), k, start, score="sigmoid", choice_bias=bias, loss_coef=0.1)
    assert (routes.cpu().long() == want).all()
    without = rp.rp_route(x.cuda(), k, start, score="sigmoid", loss_coef=0.1)
    rows = [t for t in range(500) if t not in (3, 4)]
    assert (without[0] == routes).all() and (without[1][rows] == gates[rows]).all() and (without[2] == counts).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
def test_experts_taken_out_come_last_under_a_bias(kind):
    """A score of 0 comes behind any other, however small (sigmoid(-50) = 2e-22)."""
    import torch
    x = torch.full((40, 64), -50.0)
    x[:, :20] = -math.inf
    x[:, 63] = 0.0
    x[1::2, 30:34] = torch.tensor([-48.0, -60.0, -45.0, -48.0])
    x = x.to(getattr(torch, kind))
    want = torch.argsort(-x.double(), dim=1, stable=True)[:, :6]
    routes, gates, _, _ = rp.rp_route(x.cuda(), 6, torch.tensor([0, 40], device="cuda"), score="sigmoid", choice_bias=torch.zeros(64, device="cuda"))
    assert (routes.cpu().long() == want).all()
    chosen = torch.sigmoid(x.double()).gather(1, want)
    assert ((gates.cpu().double() - chosen / chosen.sum(1, keepdim=True)).abs() <= FLOAT).all()


@pytest.mark.gpu
@pytest.mark.parametrize("E", [16, 64, 128])
def test_tokens_with_tiny_scores_leave_those_beside_them_alone(E):
    """The loss of one token's group, bit for bit, whatever a token of no group beside it holds."""
    import torch
    start = torch.tensor([0, 1], device="cuda")
    for seed in range(60):
        x = logits_of(64, E, torch.float32, seed).cuda()
        want = rp.rp_route(x, 2, start, score="sigmoid", loss_coef=1.0)
        x[1:] = -100.0
        got = rp.rp_route(x, 2, start, score="sigmoid", loss_coef=1.0)
        assert all((a == b).all() for a, b in zip(want, got)), seed


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float32", "bfloat16"])
@pytest.mark.parametrize("logit", [-22.0, -24.0, -26.0, -27.0, -40.0])
def test_one_expert_left_with_a_small_score(logit, kind):
    """All other experts taken out: its part of the scores is 1, so the loss of a token is coef E / k."""
    import torch
    x = torch.full((1, 1000), -math.inf)
    x[0, 7] = logit
    routes, gates, _, loss = rp.rp_route(x.to(getattr(torch, kind)).cuda(), 1, torch.tensor([0, 1], device="cuda"), score="sigmoid", loss_coef=1.0)
    assert routes.item() == 7 and abs(gates.item() - 1) <= FLOAT and abs(loss.item() - 1000) <= FLOAT * 1000


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("E", [16, 100, 256])
def test_rows_of_the_lowest_value_and_of_large_ones(E, kind):
    """A row whose every logit is the type's lowest value has equal scores; large logits as any others."""
    import torch
    dtype = getattr(torch, kind)
    low, high = torch.finfo(dtype).min, torch.finfo(dtype).max
    x = logits_of(8, E, dtype, E)
    x[0] = low
    x[1] = high
    x[2] = low
    x[2, 3], x[2, 9] = 1.0, 1.0
    x[3, 5] = high
    x[4] = low
    x[4, 7] = high
    x[5] = min(1e30, high)
    x[5, 1] = low
    x[6] = -min(1e9, high)
    start = [0, 1, 2, 3, 4, 5, 6, 7, 8]
    want = reference(x, 2, start, coef=0.5)
    st = torch.tensor(start, device="cuda")
    routes, gates, counts, loss = rp.rp_route(x.cuda(), 2, st, loss_coef=0.5)
    assert (routes.cpu().long() == want[0]).all() and (counts.cpu().double() == want[2]).all()
    assert ((gates.cpu().double() - want[1]).abs() <= FLOAT * want[1]).all()
    assert abs(loss.item() - want[3].item()) <= 2 * FLOAT * want[3].item()
    x64 = x.double().requires_grad_(True)
    p = torch.softmax(x64, 1)
    dg = torch.tensor([[1.0, -2.0]]).expand(8, 2).contiguous()
    g = p.gather(1, want[0])
    value = (g / g.sum(1, keepdim=True) * dg.double()).sum() + 3.0 * 0.5 / 8 * E / 2 * sum((want[2][t] * p[t]).sum() for t in range(8))
    grad = torch.autograd.grad(value, x64)[0]
    got = rp.rp_route_grad(x.cuda(), routes, st, counts, gates_grad=dg.cuda(), loss_grad=torch.tensor([3.0], device="cuda"), loss_coef=0.5)
    tol = torch.finfo(dtype).eps / 2 * grad.abs() + 4 * FLOAT * (2.0 * 2 + 3.0 * 0.5 / 8 * E / 2) + 1e-7 * (kind == "float16")
    assert ((got.cpu().double() - grad).abs() <= tol).all()


@pytest.mark.gpu
@pytest.mark.parametrize("score", ["softmax", "sigmoid"])
def test_gradient_of_gates_whose_scores_are_tiny(score):
    """Replayed experts that this pass gives next to nothing: their gates are shares of it, and so are the gradients."""
    import torch
    x = torch.zeros(4, 32)
    x[:, 4], x[:, 9], x[:, 30] = -86.0, -86.5, -85.0
    if score == "sigmoid":
        x[:, :] -= 0.5
    ids = torch.tensor([[4, 9, 30]]).expand(4, 3).contiguous()
    start = torch.tensor([0, 4], device="cuda")
    _, gates, counts, _ = rp.rp_route(x.cuda(), 3, start, score=score, replay=ids.cuda())
    dg = torch.tensor([[100.0, -300.0, 7.0], [1.0, 2.0, 3.0], [1e4, 0.0, 0.0], [0.0, 0.0, 1e-3]])
    x64 = x.double().requires_grad_(True)
    want_gates = reference(x64, 3, [0, 4], score, replay=ids)[1]
    want = torch.autograd.grad((want_gates * dg.double()).sum(), x64)[0]
    assert ((gates.cpu().double() - want_gates).abs() <= 16 * FLOAT * want_gates).all()
    got = rp.rp_route_grad(x.cuda(), ids.cuda(), start, counts, gates_grad=dg.cuda(), score=score)
    # (logits to 87: ex2's argument to 125 is off by 2^-18, so a score by 6e-6)
    assert ((got.cpu().double() - want).abs() <= 16 * FLOAT * dg.abs().amax(1, keepdim=True).double()).all()
