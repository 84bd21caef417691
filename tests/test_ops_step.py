"""Attention of one token of each sequence against its cache, against the formula in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp


def sees(filled, window, sinks):
    """Rows of a sequence that its newest token sees."""
    first = max(0, filled - window) if window else 0
    return list(range(min(sinks, first))) + list(range(first, filled))


def filled_rows(start, length, T):
    for i, (lo, hi) in enumerate(zip(start, start[1:])):
        lo, hi = max(lo, 0), min(hi, T)
        room = max(hi - lo, 0)
        yield lo, room if length is None else min(max(length[i], 0), room)


def check(q, k, v, start, length, window, sinks, scale, out, lse):
    import torch
    half, share = torch.finfo(q.dtype).eps / 2, q.shape[1] // k.shape[1]
    for i, (lo, n) in enumerate(filled_rows(start, length, k.shape[0])):
        j = torch.tensor(sees(n, window, sinks), dtype=torch.long, device="cuda") + lo
        if not len(j):
            assert (out[i] == 0).all() and (lse[i] == -math.inf).all()
            continue
        for hk in range(k.shape[1]):
            rows = slice(hk * share, (hk + 1) * share)
            s = q[i, rows].double() @ k[j, hk].double().T * scale
            p, v64 = torch.softmax(s, 1), v[j, hk].double()
            want, size, top = p @ v64, p @ v64.abs(), s.abs().amax().item()
            # the output rounded once; a weight by its score's 32 bits (a product of up to 128 terms, 2^-22 of their sizes, and the rounding of its exponent)
            # and by what two roundings to the type leave: 2^-16 for bf16, less for float16; values under the 16-bit types' normal range
            near = 2.0 ** -15 * size + 2.0 ** -20 * (1 + top) * size
            assert ((out[i, rows].double() - want).abs() <= half * want.abs() + near * (1 + half) + 1e-7).all()
            assert ((lse[i, rows].double() - torch.logsumexp(s, 1)).abs() <= 4e-6 * (1 + torch.logsumexp(s, 1).abs() + top)).all()


def test_refusals():
    lib = rp.lib()
    buf = np.zeros(4096, np.float64)
    p = (buf.ctypes.data + 15) // 16 * 16

    def a(hq=2, hk=1, d=64, kind=2, scale=0.1):
        return C.byref(rp.rp_attend_config(hq, hk, d, kind, 1, scale))
    ok, off = C.byref(rp.rp_view(p, 128, 64)), C.byref(rp.rp_view(p, 100, 64))

    def call(cfg=a(), window=0, sinks=0, T=2, q=ok, k=ok, v=ok, start=p, N=1, length=None, out=C.byref(rp.rp_view(p + 256, 128, 64)), nbytes=1 << 14, space=p):
        return lib.rp_attend_step(cfg, window, sinks, T, q, k, v, start, N, length, out, None, space, nbytes, None)
    assert call() == -1                                  # host arrays
    for bad in (dict(cfg=None), dict(window=-1), dict(sinks=-1), dict(T=-1), dict(q=None), dict(k=off), dict(v=None), dict(start=None), dict(start=p + 4), dict(N=0),
                dict(length=p + 4), dict(out=None), dict(out=ok), dict(nbytes=16), dict(space=None), dict(space=p + 8), dict(cfg=a(kind=0)), dict(cfg=a(scale=0.0))):
        assert call(**bad) == -1, bad
    assert call(cfg=a(d=136)) == -5 and call(cfg=a(d=60)) == -2 and call(cfg=a(hq=3, hk=2)) == -2
    assert call(cfg=a(hq=64, hk=64), N=1 << 24) == -5 and lib.rp_attend_step_workspace(a(hq=64, hk=64), 0, 0, 2, 1 << 24) == 0          # more units than 32 bits count
    size = lib.rp_attend_step_workspace
    assert size(None, 0, 0, 1, 1) == 0 and size(a(), -1, 0, 1, 1) == 0 and size(a(), 0, -1, 1, 1) == 0
    # a chunk of a sequence leaves two sums and the values of each query head; with a window there are fewer, and never more than 128 of a sequence
    assert size(a(), 0, 0, 5000, 1) >= 20 * 2 * (64 + 2) * 4 and size(a(), 300, 0, 5000, 1) < size(a(), 0, 0, 5000, 1)
    assert size(a(), 0, 0, 1 << 24, 1) == size(a(), 0, 0, 1 << 25, 1)


CASES = [
    # query heads, key heads, head size, lengths, spare rows, window, first tokens
    (1, 1, 64, [1], 0, 0, 0), (4, 2, 128, [1, 2, 15, 16, 17], 3, 0, 0), (8, 1, 128, [255, 256, 257, 0, 64], 1, 0, 0), (16, 1, 64, [600, 3], 0, 100, 0),
    (20, 1, 96, [511, 512, 513, 1], 5, 200, 7), (40, 2, 128, [1000, 30], 2, 256, 300), (5, 5, 80, [700], 9, 1, 0), (3, 3, 8, [300, 299], 0, 1, 1), (33, 1, 64, [90, 270], 4, 64, 64),
    (6, 2, 128, [4097, 100, 0, 2000], 0, 4096, 0), (8, 8, 64, [17000, 12], 11, 0, 0), (2, 2, 120, [20001], 0, 20000, 128), (9, 1, 72, [16384, 16385], 1, 0, 0),
    (4, 1, 128, [2175, 2176, 2177, 2303, 2304], 0, 0, 0), (3, 3, 64, [3000] + [0, 1, 260] * 13, 2, 2170, 9),
]


def inputs(case, kind):
    import torch
    hq, hk, d, lengths, spare, window, sinks = case
    start = [2]
    for n in lengths:
        start.append(start[-1] + n + spare)
    T = start[-1] + 3
    g = torch.Generator().manual_seed(T + d)
    q = torch.randn(hq, len(lengths), d + 8, generator=g).to(getattr(torch, kind)).cuda()[:, :, :d].transpose(0, 1)
    wide = torch.randn(T, 2 * hk, d, generator=g).to(getattr(torch, kind)).cuda()
    return q, wide[:, :hk], wide[:, hk:], start


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("case", CASES, ids=[f"{c[0]}-{c[1]}-{c[2]}-{max(c[3])}-w{c[5]}-s{c[6]}" for c in CASES])
def test_step(case, kind):
    import torch
    q, k, v, start = inputs(case, kind)
    lengths, window, sinks = case[3], case[5], case[6]
    st = torch.tensor(start, device="cuda")
    out, lse = rp.rp_attend_step(q, k, v, st, length=torch.tensor(lengths, device="cuda"), window=window, sinks=sinks, scale=0.2)
    check(q, k, v, start, lengths, window, sinks, 0.2, out, lse)
    out, lse = rp.rp_attend_step(q, k, v, st, window=window, sinks=sinks)
    check(q, k, v, start, None, window, sinks, q.shape[2] ** -0.5, out, lse)


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(0, 0), (300, 5), (4000, 128)])
def test_the_last_token_of_each_sample_as_the_packed_row_has_it(window, sinks):
    import torch
    lengths = [1, 700, 129, 2500]
    start = torch.tensor([0] + np.cumsum(lengths).tolist(), device="cuda")
    g = torch.Generator().manual_seed(3)
    q, k, v = (torch.randn(sum(lengths), n, 128, generator=g).bfloat16().cuda() for n in (8, 2, 2))
    want, w_lse = rp.rp_attend_window(q, k, v, start, window=window or 10000, sinks=sinks)
    last = start[1:] - 1
    out, lse = rp.rp_attend_step(q[last], k, v, start, window=window, sinks=sinks)
    # (there the weights are rounded once to 2^-8, and both outputs)
    assert (out.double() - want[last].double()).abs().max() <= 2.0 ** -8 * 5 and (lse - w_lse[last]).abs().max() <= 1e-4


@pytest.mark.gpu
@pytest.mark.parametrize("hq,hk", [(5, 1), (6, 3)])
def test_many_sequences_of_a_few_chunks_and_of_many(hq, hk):
    """More query heads in all than the joining kernel has CTAs, sequences on both sides of what a warp of it takes; some again alone, bit for bit."""
    import torch
    lengths = [[130, 300, 255, 0, 2400, 511, 1, 700, 2175, 2176][i * 7 % 10] for i in range(500)]
    q, k, v, start = inputs((hq, hk, 64, lengths, 0, 0, 0), "bfloat16")
    st = torch.tensor(start, device="cuda")
    out, lse = rp.rp_attend_step(q, k, v, st)
    check(q, k, v, start, None, 0, 0, 64 ** -0.5, out, lse)
    for i in (0, 1, 2, 3, 5, 8, 250, 499):
        o, l = rp.rp_attend_step(q[i:i + 1], k, v, st[i:i + 2].contiguous())
        assert (o[0] == out[i]).all() and (l[0] == lse[i]).all()


@pytest.mark.gpu
def test_lengths_outside_their_room_and_rows_that_are_not_seen():
    """NaN and infinities wherever the tokens do not look: spare rows, other sequences, rows before the window, the cache's ends."""
    import torch
    q, k, v, start = inputs((4, 2, 128, [900, 40, 300, 20], 6, 0, 0), "bfloat16")
    st = torch.tensor(start, device="cuda")
    length = [900, -3, 10 ** 12, 0]
    kw = dict(length=torch.tensor(length, device="cuda"), window=100, sinks=3)
    want = rp.rp_attend_step(q, k, v, st, **kw)
    check(q, k, v, start, length, 100, 3, 128 ** -0.5, *want)
    bad = [x.clone() for x in (k, v)]
    keep = torch.zeros(k.shape[0], dtype=torch.bool, device="cuda")
    for lo, n in filled_rows(start, length, k.shape[0]):
        keep[[lo + j for j in sees(n, 100, 3)]] = True
    for x, value in zip(bad, (float("nan"), float("inf"))):
        x[~keep] = value
    big, lse = torch.full((9, 4, 128), 3.0, dtype=torch.bfloat16, device="cuda"), torch.full((9, 4), 3.0, device="cuda")
    rp.rp_attend_step(q, *bad, st, out=big[:4], lse=lse[:4], **kw)
    assert (big[:4] == want[0]).all() and (lse[:4] == want[1]).all() and (big[4:] == 3).all() and (lse[4:] == 3).all()
    # starts before the cache and behind it, and samples that run backwards
    st = torch.tensor([-50, 60, 40, k.shape[0] + 99], device="cuda")
    out, lse = rp.rp_attend_step(q[:3], k, v, st)
    check(q[:3], k, v, st.tolist(), None, 0, 0, 128 ** -0.5, out, lse)
    empty = rp.rp_attend_step(q, k[:0], v[:0], torch.zeros(5, dtype=torch.int64, device="cuda"))
    assert (empty[0] == 0).all() and (empty[1] == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
def test_scores_far_apart(kind):
    """One key that takes all, many small weights beside a large one, keys at -inf, and a token whose keys all are."""
    import torch
    T, d = 140000, 64
    dt = getattr(torch, kind)
    q = torch.zeros(1, 1, d, device="cuda", dtype=dt)
    q[..., 0] = 1
    k = torch.zeros(T, 1, d, device="cuda", dtype=dt)
    v = torch.rand(T, 1, d, generator=torch.Generator().manual_seed(2)).cuda().to(dt) + 1
    st = torch.tensor([0, T], device="cuda")
    for under in (0.0, 12.0, 17.5, 60.0, math.inf):
        k[:, 0, 0] = -under
        k[77777, 0, 0] = 0.0
        out, lse = rp.rp_attend_step(q, k, v, st, scale=1.0)
        s = k[:, 0, 0].double()
        p = torch.softmax(s, 0)
        want = p @ v[:, 0].double()
        # sums of 140000 terms in 32 bits, cut off by the matrix unit at 2^-23 of what a chunk's tile of 16 has: 137 tiles to a warp; the output's rounding
        assert ((out[0, 0].double() - want).abs() <= (torch.finfo(dt).eps / 2 + 137 * 2.0 ** -22 + 2.0 ** -15) * want).all()
        assert abs(lse.item() - torch.logsumexp(s, 0).item()) <= 137 * 2.0 ** -23 + 4e-6 * 12
    k[:, 0, 0] = -math.inf
    out, lse = rp.rp_attend_step(q, k, v, st, scale=1.0)
    assert torch.isnan(out).all() and lse.item() == -math.inf
    k[:, 0, 0] = torch.linspace(-300, 300, T, device="cuda").to(dt)
    out, lse = rp.rp_attend_step(q, k, v, st, scale=1.0)
    p = torch.softmax(k[:, 0, 0].double(), 0)
    want = p @ v[:, 0].double()
    # (scores of 300 as 433 powers of two: their exponents' rounding leaves a weight 2^-15)
    assert ((out[0, 0].double() - want).abs() <= (torch.finfo(dt).eps / 2 + 2.0 ** -13) * want).all()


@pytest.mark.gpu
def test_a_sequence_gets_alone_what_it_gets_among_others():
    import torch
    q, k, v, start = inputs((8, 2, 128, [3000, 1, 17000, 256, 0, 300], 0, 0, 0), "bfloat16")
    st = torch.tensor(start, device="cuda")
    for kw in (dict(), dict(window=2000, sinks=50)):
        out, lse = rp.rp_attend_step(q, k, v, st, **kw)
        for i in range(6):
            o, l = rp.rp_attend_step(q[i:i + 1], k, v, st[i:i + 2].contiguous(), **kw)
            assert (o[0] == out[i]).all() and (l[0] == lse[i]).all()
    many = torch.arange(0, 5001, device="cuda")
    x = torch.randn(5000, 3, 64, generator=torch.Generator().manual_seed(4)).half().cuda()
    out, lse = rp.rp_attend_step(x[:, :1], x[:, 1:2], x[:, 2:], many)
    assert (out == x[:, 2:]).all()                       # one key each: its values


@pytest.mark.gpu
@pytest.mark.parametrize("apart", [False, True])
def test_caches_whose_rows_lie_beyond_32_bits(apart):
    """Elements 2^31 and more from the cache's first one: a long cache, and a short one with its rows far apart."""
    import torch
    T, hk, d, step = (1600, 2, 64, 1 << 21) if apart else (1100000, 8, 128, 2048)
    n, lengths = (800, [700, 800]) if apart else (6000, [5000, 5990])
    buf = torch.empty(T, step, dtype=torch.bfloat16, device="cuda")
    g = torch.Generator().manual_seed(9)
    seen = torch.randn(2, n, 2 * hk * d, generator=g).bfloat16().cuda()
    start = [T - 2 * n, T - n, T]
    for i in range(2):
        buf[start[i]:start[i + 1], :2 * hk * d] = seen[i]
    k, v = buf[:, :hk * d].view(T, hk, d), buf[:, hk * d:2 * hk * d].view(T, hk, d)
    q = torch.randn(2, 4 * hk, d, generator=g).bfloat16().cuda()
    length = torch.tensor(lengths, device="cuda")
    small = seen.view(2 * n, 2, hk, d)
    for kw in (dict(), dict(window=500, sinks=30)):
        out, lse = rp.rp_attend_step(q, k, v, torch.tensor(start, device="cuda"), length=length, **kw)
        o, l = rp.rp_attend_step(q, small[:, 0], small[:, 1], torch.tensor([0, n, 2 * n], device="cuda"), length=length, **kw)
        assert (out == o).all() and (lse == l).all()


@pytest.mark.gpu
def test_repeated_streamed_and_captured_calls_agree_bit_for_bit():
    """Lengths that grow between replays are read anew."""
    import torch
    q, k, v, start = inputs((8, 2, 128, [3000, 5000, 20000], 64, 0, 0), "bfloat16")
    st, length = torch.tensor(start, device="cuda"), torch.tensor([3000, 5000, 20000], device="cuda")
    kw = dict(length=length, window=18000, sinks=4)
    want = rp.rp_attend_step(q, k, v, st, **kw)
    torch.cuda.synchronize()
    results = [rp.rp_attend_step(q, k, v, st, stream=s, **kw) for s in [torch.cuda.Stream() for _ in range(4)] for _ in range(3)]
    torch.cuda.synchronize()
    for got in results:
        assert all((a == b).all() for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = rp.rp_attend_step(q, k, v, st, **kw)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))
    length += 33
    graph.replay()
    want = rp.rp_attend_step(q, k, v, st, **kw)
    torch.cuda.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))
    check(q, k, v, start, length.tolist(), 18000, 4, 128 ** -0.5, *got)


@pytest.mark.gpu
def test_arguments_in_python():
    import torch
    q, k, v, start = inputs((4, 2, 64, [30, 40], 0, 0, 0), "float16")
    st = torch.tensor(start, device="cuda")
    for bad in (dict(q=q[:1]), dict(k=k[:, :, :32]), dict(v=v.bfloat16()), dict(length=torch.tensor([1], device="cuda")), dict(window=1.5),
                dict(length=torch.tensor([1, 2], device="cuda", dtype=torch.int32)), dict(out=q[:, :2]), dict(lse=torch.zeros(2, 3, device="cuda"))):
        args = dict(q=q, k=k, v=v, start=st)
        args.update(bad)
        with pytest.raises(ValueError):
            rp.rp_attend_step(**args)
    with pytest.raises(rp.RpError, match="ARG"):
        rp.rp_attend_step(q, k, v, st, out=q)
    with pytest.raises(rp.RpError, match="ARG"):
        rp.rp_attend_step(q, k, v, st, window=-1)
    with pytest.warns(UserWarning, match="rp_attend_step"):
        rp.rp_attend_step(q.clone().requires_grad_(True), k, v, st)


@pytest.mark.gpu
def test_waits_that_run_out_leave_nan_and_a_status():
    import torch
    q, k, v, start = inputs((8, 2, 128, [3000, 1, 0, 200], 0, 0, 0), "bfloat16")
    st = torch.tensor(start, device="cuda")
    status = [torch.full((1,), 7, dtype=torch.int32, device="cuda") for _ in range(3)]
    want = rp.rp_attend_step(q, k, v, st, status=status[0])
    rp.rp_debug_set_wait_limit(0)
    try:
        got = rp.rp_attend_step(q, k, v, st, status=status[1])
        torch.cuda.synchronize()
    finally:
        rp.rp_debug_set_wait_limit()
    again = rp.rp_attend_step(q, k, v, st, status=status[2])
    assert [s.item() for s in status] == [0, -8, 0] and all(torch.isnan(x).all() for x in got) and all((a == b).all() for a, b in zip(again, want))


@pytest.mark.gpu
@pytest.mark.parametrize("limit", [1, 1500, 4000])
def test_short_limits_leave_right_rows_or_nan(limit):
    import torch
    q, k, v, start = inputs((8, 2, 128, [30000, 1, 0, 200, 9000], 0, 0, 0), "bfloat16")
    st, status = torch.tensor(start, device="cuda"), torch.full((1,), 7, dtype=torch.int32, device="cuda")
    want = rp.rp_attend_step(q, k, v, st)
    rp.rp_debug_set_wait_limit(limit)
    try:
        got = rp.rp_attend_step(q, k, v, st, status=status)
        torch.cuda.synchronize()
    finally:
        rp.rp_debug_set_wait_limit()
    for x, y in zip(got, want):
        lost = torch.isnan(x)
        assert (x[~lost] == y[~lost]).all() and (status.item() == -8 or not lost.any())
    assert status.item() in (0, -8)


@pytest.mark.gpu
@pytest.mark.parametrize("window", [0, 700])
def test_short_limits_with_more_units_than_warps(window):
    """Waits that run out while warps of the same CTA look for their next sequence: every call ends, rows are right or NaN, and NaN comes with the status."""
    import torch
    lengths = [[30, 900, 0, 3000, 257, 1][i % 6] for i in range(400)]
    q, k, v, start = inputs((8, 4, 128, lengths, 3, 0, 0), "bfloat16")
    st, length, kw = torch.tensor(start, device="cuda"), torch.tensor(lengths, device="cuda"), dict(window=window, sinks=4)
    want = rp.rp_attend_step(q, k, v, st, length=length, **kw)
    check(q, k, v, start, lengths, window, 4, 128 ** -0.5, *want)
    for limit in (1, 300, 700, 1000, 1500, 2000, 3000, 5000, 10000):
        status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
        rp.rp_debug_set_wait_limit(limit)
        try:
            got = rp.rp_attend_step(q, k, v, st, length=length, status=status, **kw)
            torch.cuda.synchronize()
        finally:
            rp.rp_debug_set_wait_limit()
        assert status.item() in (0, -8)
        for x, y in zip(got, want):
            lost = torch.isnan(x)
            assert (x[~lost] == y[~lost]).all() and (status.item() == -8 or not lost.any())
    again = rp.rp_attend_step(q, k, v, st, length=length, **kw)
    assert all((a == b).all() for a, b in zip(again, want))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("d,keys", [(64, 32), (128, 16)])
def test_sums_over_a_long_cache(d, keys, kind):
    """140000 equal or small weights beside a large one, with the sums' roundings counted from the cut: 128 chunks, tiles of 4 KB (`keys` keys), of which a chunk has every 128th."""
    import torch
    T, dt = 140000, getattr(torch, kind)
    tiles = -(-(-(-T // keys)) // 128)
    q = torch.zeros(1, 1, d, device="cuda", dtype=dt)
    q[..., 0] = 1
    k = torch.zeros(T, 1, d, device="cuda", dtype=dt)
    v = torch.rand(T, 1, d, generator=torch.Generator().manual_seed(5)).cuda().to(dt) + 1
    st = torch.tensor([0, T], device="cuda")
    for under in (0.0, 9.0, 12.0, 17.5):
        k[:, 0, 0] = -under
        k[77777, 0, 0] = 0.0
        out, lse = rp.rp_attend_step(q, k, v, st, scale=1.0)
        s = k[:, 0, 0].double()
        p, w_lse = torch.softmax(s, 0), torch.logsumexp(s, 0).item()
        want = p @ v[:, 0].double()
        # a lane adds a pair of weights for each 8 keys of its tiles, then 3 times with its neighbours, 32 and 3 times over the chunks: half a step of 32 bits each.  A weight by
        # its exponent's two roundings (as powers of two, of the small ones' part of the sum) and by the power's 2 steps; two of those, the chunk's and its factor
        small = under * math.log2(math.e) * 2.0 ** -23 * (1 - math.exp(-w_lse)) + 2 * 2.0 ** -22
        assert abs(lse.item() - w_lse) <= (tiles * keys // 8 * 2 + 38) * 2.0 ** -24 + small + 3 * 2.0 ** -23 * (1 + w_lse)
        # values: a product of 16 keys is added with what lies under 2^-23 of the sum cut off, of the sum so far and of the product; a weight keeps 2^-17
        near = tiles * keys // 16 * 2.0 ** -22 + 38 * 2.0 ** -24 + small + 2.0 ** -17 + (tiles * keys // 8 * 2 + 38) * 2.0 ** -24
        assert ((out[0, 0].double() - want).abs() <= (torch.finfo(dt).eps / 2 * (1 + near) + near) * want).all()
