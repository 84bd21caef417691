"""Per-expert counts of recorded routes, and a window loaded from a record."""
import ctypes as C

import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp
from paper_2608_12146_b200.windows import make_window


def count(routes, start, n_experts):
    """The counts in plain loops over samples and layers."""
    T, L, _ = routes.shape
    out = np.zeros((len(start) - 1, L, n_experts), np.int64)
    for i, (lo, hi) in enumerate(zip(start, start[1:])):
        for l in range(L):
            ids = routes[max(lo, 0):max(min(hi, T), 0), l].astype(np.int64).ravel()
            ids = ids[(ids >= 0) & (ids < n_experts)]
            out[i, l] = np.bincount(ids, minlength=n_experts)
    return out


def test_refusals():
    lib = rp.lib()
    buf = np.zeros(64, np.int64)                    # host memory: refused before anything runs
    p = buf.ctypes.data

    def call(routes=p, size=1, T=2, L=2, k=2, E=4, start=p, N=1, demand=p):
        return lib.rp_count_routes(routes, size, T, L, k, E, 4, 2, start, N, demand, None)

    assert call() == -1                             # host arrays
    assert call(routes=None) == -1 and call(start=None) == -1 and call(demand=None) == -1
    assert call(size=3) == -1 and call(size=0) == -1 and call(T=-1) == -1 and call(L=0) == -1 and call(k=0) == -1 and call(N=0) == -1
    assert call(routes=p + 1, size=2) == -1 and call(start=p + 4) == -1 and call(demand=p + 2) == -1
    assert call(E=1025) == -5 and call(k=1025) == -5 and call(L=65536) == -5 and call(T=(1 << 36) + 1) == -5
    out = C.c_void_p(123)
    assert lib.rp_window_load_routes(C.byref(out), None, None, None, 1, 1, 1, 1, None) == -1 and out.value is None


def test_binding_refuses_what_it_cannot_pass_on():
    import torch
    start = torch.zeros(2, dtype=torch.int64)
    with pytest.raises(ValueError):
        rp.rp_count_routes(torch.zeros(4, 2, 2, dtype=torch.uint8), start, 4)
    with pytest.raises(ValueError):
        rp.rp_count_routes(torch.zeros(4, 2, dtype=torch.uint8), start, 4)
    with pytest.raises(ValueError):
        rp.rp_count_routes(torch.zeros(4, 2, 2), start, 4)


CASES = [
    # tokens, layers, k, experts, starts
    (1, 1, 1, 1, [0, 1]),
    (1, 4, 2, 16, [0, 1]),
    (37, 3, 2, 5, [0, 0, 1, 20, 20, 37]),              # empty samples, odd sizes
    (300, 4, 2, 16, [7, 100, 290]),                    # tokens before the first and behind the last sample
    (300, 5, 8, 256, [-3, 100, 400]),                  # starts outside the tokens
    (4099, 16, 4, 64, [0, 1, 2, 3, 700, 4000, 4099]),
    (2500, 7, 6, 160, [0, 2500]),
    (9000, 3, 8, 1024, list(range(0, 9001, 3))),       # many short samples
    (700, 48, 8, 256, [0, 350, 700]),
    (5000, 2, 1, 200, [0, 2500, 5000]),
    (3, 2, 33, 40, [0, 3]),
]


@pytest.mark.gpu
@pytest.mark.parametrize("order", ["token", "layer", "strided"])
@pytest.mark.parametrize("kind", ["uint8", "int16", "int32", "int64"])
@pytest.mark.parametrize("case", CASES, ids=[str(c[:4]) for c in CASES])
def test_counts(case, kind, order):
    import torch
    T, L, k, E, start = case
    if kind == "uint8" and E > 256:
        pytest.skip("ids do not fit a byte")
    rng = np.random.default_rng(T + L)
    p = rng.dirichlet(np.full(E, 0.2))
    ids = rng.choice(E, size=(T, L, k), p=p)
    ids[rng.random(ids.shape) < 0.05] = E if kind == "uint8" and E < 256 else (0 if kind == "uint8" else -1)    # empty places
    if kind != "uint8" and T > 2:
        ids[T // 2, 0, 0] = E + 7
    np_kind = getattr(np, kind)
    host = ids.astype(np_kind)
    dtype = getattr(torch, kind)
    if order == "token":
        routes = torch.from_numpy(host).cuda()
    elif order == "layer":
        routes = torch.from_numpy(np.ascontiguousarray(host.transpose(1, 0, 2))).cuda().transpose(0, 1)
    else:                                              # a slice of a wider record, one element off its start
        wide = torch.full((T, L + 1, k + 3), 1, dtype=dtype, device="cuda")
        routes = wide[:, 1:, 1:k + 1]
        routes.copy_(torch.from_numpy(host))
    got = rp.rp_count_routes(routes, torch.tensor(start, device="cuda"), E)
    want = count(host, start, E)
    assert got.dtype == torch.int32 and (got.cpu().numpy() == want).all()


@pytest.mark.gpu
@pytest.mark.parametrize("E", [257, 512, 1000, 1024])
@pytest.mark.parametrize("L,k", [(1, 8), (3, 2), (8, 8)])
def test_bytes_where_there_are_more_experts_than_a_byte_names(E, L, k):
    import torch
    host = np.random.default_rng(E + L).integers(0, 256, (2000, L, k)).astype(np.uint8)
    start = [0, 3, 1200, 1990]
    got = rp.rp_count_routes(torch.from_numpy(host).cuda(), torch.tensor(start, device="cuda"), E)
    assert (got.cpu().numpy() == count(host, start, E)).all()


@pytest.mark.gpu
def test_output_is_written_whole_and_nothing_behind_it():
    import torch
    out = torch.full((4, 2, 8), -7, dtype=torch.int32, device="cuda")
    routes = torch.zeros(5, 2, 2, dtype=torch.uint8, device="cuda")
    rp.rp_count_routes(routes, torch.tensor([0, 2, 2, 5], device="cuda"), 8, demand=out[:3])
    assert out[:3, :, 0].tolist() == [[4, 4], [0, 0], [6, 6]] and (out[:3, :, 1:] == 0).all() and (out[3] == -7).all()
    none = rp.rp_count_routes(routes[:0], torch.tensor([0, 0], device="cuda"), 8)
    assert (none == 0).all()


@pytest.mark.gpu
def test_records_that_repeat():
    import torch
    start = torch.tensor([0, 5, 700], device="cuda")
    for wide in (torch.randint(0, 32, (1, 6, 8), device="cuda"), torch.randint(0, 32, (700, 1, 8), device="cuda")):
        for kind in (torch.uint8, torch.int16, torch.int32):
            routes = wide.to(kind).expand(700, 6, 8)
            assert (rp.rp_count_routes(routes, start, 32) == rp.rp_count_routes(routes.contiguous(), start, 32)).all()


@pytest.mark.gpu
def test_far_elements_of_a_long_record():
    """Offsets that pass 32 bits: the last tokens of a record of 2^32 + bytes."""
    import torch
    T, L, k = (1 << 25) + 5, 16, 8
    routes = torch.zeros(T, L, k, dtype=torch.uint8, device="cuda")
    routes[-3:] = 3
    got = rp.rp_count_routes(routes, torch.tensor([0, T - 4, T], device="cuda"), 4)
    assert got[0, :, 0].tolist() == [(T - 4) * k] * L and got[1, :, 3].tolist() == [3 * k] * L and got[1, :, 0].tolist() == [k] * L


@pytest.mark.gpu
def test_on_another_stream_and_captured():
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(1)
    routes = torch.randint(0, 64, (3000, 4, 4), device="cuda", generator=g).to(torch.int16)
    start = torch.tensor([0, 1000, 3000], device="cuda")
    want = rp.rp_count_routes(routes, start, 64).clone()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    got = rp.rp_count_routes(routes, start, 64, stream=side)
    side.synchronize()
    assert (got == want).all()
    got = rp.rp_count_routes(routes, start, 64, stream=side.cuda_stream)
    side.synchronize()
    assert (got == want).all()
    graph, out = torch.cuda.CUDAGraph(), torch.zeros_like(want)
    with torch.cuda.graph(graph):
        rp.rp_count_routes(routes, start, 64, demand=out)
    for _ in range(2):
        out.fill_(5)
        graph.replay()
        torch.cuda.synchronize()
        assert (out == want).all()


@pytest.mark.gpu
@pytest.mark.parametrize("host_lengths", [True, False])
def test_window_from_a_record_plans_as_from_its_demand(host_lengths):
    """The same window twice: from routes drawn to match the window's demand tensor, and from the tensor itself."""
    import torch
    w = make_window("tiny")
    s = w.spec
    T, k = int(w.lengths.sum()), s.top_k
    n, L, E = w.demand.shape
    routes = np.empty((T, L, k), np.uint8)
    lo = 0
    for i, t in enumerate(w.lengths):
        for l in range(L):
            routes[lo:lo + t, l] = np.repeat(np.arange(E), w.demand[i, l]).reshape(t, k)
        lo += int(t)
    kw = dict(token_cap=s.token_cap, dp_width=s.dp_width, ep_width=s.ep_width, pop_size=s.pop_size, alpha=s.alpha, beta=s.beta, seed=3)
    lengths = w.lengths if host_lengths else torch.from_numpy(w.lengths).cuda()
    plans = []
    record = torch.from_numpy(routes).cuda()
    for ctx in (rp.rp_window_load(w.lengths, w.demand, top_k=k, **kw),
                rp.rp_window_load_routes(lengths, record, E, **kw)):
        pi, load = rp.rp_place_experts(ctx)
        rows = rp.rp_pack_rows(ctx)
        rp.rp_anneal(ctx, n_levels=4, steps_per_level=20, t0=1e-2, t_ratio=0.5, p_reloc=0.25, p_guide=0.8)
        plans.append((pi, load, rows, *rp.rp_best(ctx)))
        rp.rp_destroy(ctx)
    for a, b in zip(*plans):
        assert np.array_equal(np.asarray(a), np.asarray(b))
    bad = record.clone()
    bad[5, 0, 0] = 200                                 # an empty place: sum over experts is not k * t
    with pytest.raises(rp.RpError, match="CONSERVATION"):
        rp.rp_window_load_routes(lengths, bad, E, **kw)
    with pytest.raises(rp.RpError, match="CONSERVATION"):
        rp.rp_window_load_routes(lengths, record[:-1], E, **kw)
    with pytest.raises(rp.RpError, match="ARG"):
        rp._check(rp.lib().rp_window_load_routes(C.byref(C.c_void_p()), C.byref(rp._window_config(n, L, E, k, s.token_cap, s.dp_width, s.ep_width, 2, None, (1.0,), (0.0,), 0, 0)[0]),
                                                 w.lengths.ctypes.data, routes.ctypes.data, 1, T, L * k, k, None), "host record")


@pytest.mark.gpu
@pytest.mark.parametrize("order", ["token", "layer"])
@pytest.mark.parametrize("kind", ["uint8", "int16", "int32", "int64"])
def test_window_from_records_of_every_type_and_order(kind, order):
    import torch
    rng = np.random.default_rng(3)
    lengths = np.array([30, 1, 64, 17, 40, 40, 9, 55], np.int32)
    T, L, E, k = int(lengths.sum()), 3, 16, 2
    host = rng.integers(0, E, (T, L, k)).astype(getattr(np, kind))
    record = torch.from_numpy(host if order == "token" else np.ascontiguousarray(host.transpose(1, 0, 2))).cuda()
    record = record if order == "token" else record.transpose(0, 1)
    kw = dict(token_cap=128, dp_width=2, ep_width=4, pop_size=8, seed=1)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    demand = count(host, [0] + np.cumsum(lengths).tolist(), E).astype(np.int32)
    got = []
    for ctx in (rp.rp_window_load(lengths, demand, top_k=k, **kw), rp.rp_window_load_routes(lengths, record, E, stream=side, **kw)):
        got.append(rp.rp_place_experts(ctx))
        rp.rp_destroy(ctx)
    for a, b in zip(*got):
        assert np.array_equal(np.asarray(a), np.asarray(b))


@pytest.mark.gpu
def test_lengths_that_make_no_window_are_refused():
    import torch
    record = torch.zeros(100, 2, 1, dtype=torch.uint8, device="cuda")
    kw = dict(token_cap=128, dp_width=1, ep_width=1, pop_size=8)
    for lengths in ([40, -20, 80], [-1, 50, 51], [0, 50, 50], [100, 100, 100], [200, -50, -50]):
        with pytest.raises(rp.RpError, match="CONSERVATION"):
            rp.rp_window_load_routes(np.array(lengths, np.int32), record, 4, **kw)


@pytest.mark.gpu
def test_starts_that_decrease_read_nothing_else():
    """Not allowed, and without a promise for the counts; nothing outside the record is counted all the same."""
    import torch
    routes = torch.full((500, 2, 3), 1, dtype=torch.int16, device="cuda")
    for start in ([0, 400, 100, 500], [500, 0, 500], [300, 200, 100, 0], [10 ** 12, -10 ** 12, 10 ** 12]):
        got = rp.rp_count_routes(routes, torch.tensor(start, device="cuda"), 4)
        assert (got[:, :, [0, 2, 3]] == 0).all() and (got >= 0).all() and got.sum().item() <= 500 * 2 * 3 * (len(start) - 1)


@pytest.mark.gpu
def test_window_from_a_record_that_the_current_stream_still_writes():
    import torch
    rng = np.random.default_rng(8)
    lengths = np.array([30, 1, 64, 17, 40, 40, 9, 55], np.int32)
    T, L, E, k = int(lengths.sum()), 3, 16, 2
    host = rng.integers(0, E, (T, L, k)).astype(np.uint8)
    kw = dict(token_cap=128, dp_width=2, ep_width=4, pop_size=8, seed=1)
    want = rp.rp_window_load(lengths, count(host, [0] + np.cumsum(lengths).tolist(), E).astype(np.int32), top_k=k, **kw)
    right, record = torch.from_numpy(host).cuda(), torch.zeros(T, L, k, dtype=torch.uint8, device="cuda")
    rp.rp_destroy(rp.rp_window_load_routes(lengths, record, E, **kw))          # (kernels are loaded, which waits for the GPU)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda._sleep(100_000_000)                   # about 50 ms
        record.copy_(right)
        got = rp.rp_window_load_routes(lengths, record, E, **kw)
        for a, b in zip(rp.rp_place_experts(got), rp.rp_place_experts(want)):
            assert np.array_equal(np.asarray(a), np.asarray(b))
    rp.rp_destroy(got)
    rp.rp_destroy(want)


@pytest.mark.gpu
def test_window_from_counts_that_the_current_stream_still_makes():
    """Record, counts and window one after the other on a stream of the caller's."""
    import torch
    rng = np.random.default_rng(9)
    lengths = np.array([30, 1, 64, 17, 40, 40, 9, 55], np.int32)
    T, L, E, k = int(lengths.sum()), 3, 16, 2
    host, cuts = rng.integers(0, E, (T, L, k)).astype(np.uint8), [0] + np.cumsum(lengths).tolist()
    kw = dict(top_k=k, token_cap=128, dp_width=2, ep_width=4, pop_size=8, seed=1)
    want = rp.rp_window_load(lengths, count(host, cuts, E).astype(np.int32), **kw)
    record, start = torch.from_numpy(host).cuda(), torch.tensor(cuts, device="cuda")
    demand = rp.rp_count_routes(torch.zeros_like(record), start, E)
    rp.rp_destroy(rp.rp_window_load(lengths, demand, **kw))                    # (kernels are loaded, which waits for the GPU)
    torch.cuda.synchronize()
    with torch.cuda.stream(torch.cuda.Stream()):
        torch.cuda._sleep(100_000_000)                   # about 50 ms
        rp.rp_count_routes(record, start, E, demand=demand)
        got = rp.rp_window_load(lengths, demand, **kw)
        for a, b in zip(rp.rp_place_experts(got), rp.rp_place_experts(want)):
            assert np.array_equal(np.asarray(a), np.asarray(b))
    rp.rp_destroy(got)
    rp.rp_destroy(want)
