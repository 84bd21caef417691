"""Attention with a sliding window and first tokens that stay visible, and its gradient, against the formulas in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp


def hidden(n, window, sinks, device="cuda"):
    import torch
    i = torch.arange(n, device=device)
    gap = i[:, None] - i
    return (gap < 0) | ((gap >= window) & (i >= sinks))


def weights(q, k, scale, mask):
    """Softmax weights [n, n] of one sample and one head, and the log of each row's sum, in 64 bits."""
    import torch
    s = (q @ k.T * scale).masked_fill(mask, -math.inf)
    return torch.softmax(s, 1), torch.logsumexp(s, 1)


def samples(start, T):
    for lo, hi in zip(start, start[1:]):
        lo, hi = max(lo, 0), min(hi, T)
        if hi > lo:
            yield lo, hi


def test_refusals():
    lib = rp.lib()
    buf = np.zeros(4096, np.float64)
    p = (buf.ctypes.data + 15) // 16 * 16

    def a(hq=2, hk=1, d=64, kind=2, causal=1, scale=0.1):
        return C.byref(rp.rp_attend_config(hq, hk, d, kind, causal, scale))
    ok = C.byref(rp.rp_view(p, 128, 64))
    off = C.byref(rp.rp_view(p, 100, 64))

    def fwd(cfg=a(), window=4, sinks=0, T=2, q=ok, k=ok, start=p, nbytes=1 << 14, space=p):
        return lib.rp_attend_window(cfg, window, sinks, T, q, k, ok, start, 1, ok, None, space, nbytes, None)

    def back(cfg=a(), window=4, sinks=0, T=2, q=ok, k=ok, start=p, nbytes=1 << 14, space=p):
        return lib.rp_attend_window_grad(cfg, window, sinks, T, q, k, ok, ok, ok, ok, start, 1, ok, ok, ok, space, nbytes, None)
    for call in (fwd, back):
        assert call() == -1                              # host arrays
        for bad in (dict(cfg=None), dict(T=-1), dict(start=None), dict(space=None), dict(space=p + 8), dict(nbytes=8), dict(q=off), dict(k=None), dict(window=0),
                    dict(window=-5), dict(sinks=-1), dict(cfg=a(causal=0)), dict(cfg=a(kind=0))):
            assert call(**bad) == -1, bad
        assert call(sinks=129) == -5 and call(T=(1 << 30) - 512) == -5 and call(cfg=a(d=136)) == -5 and call(cfg=a(hq=3, hk=2)) == -2
    size = lib.rp_attend_window_grad_workspace
    assert size(None, 4, 0, 1, 1) == 0 and size(a(), 0, 0, 1, 1) == 0 and size(a(), 4, 129, 1, 1) == 0 and size(a(), 4, 0, 100, 1) >= 100 * 2 * 8
    # chunks of 2048 tokens for the first tokens' sums: two places of [key heads][dv, dk][sinks][d] to a stretch
    assert size(a(), 4, 5, 5000, 1) - size(a(), 4, 0, 5000, 1) >= 2 * 3 * 2 * 5 * 64 * 4 + 2 * 8


def test_whole_numbers_outside_32_bits():
    assert rp._int32(1 << 40, "window") == 0x7fffffff and rp._int32(-(1 << 40), "window") == -0x80000000 and rp._int32(np.int64(7), "window") == 7
    with pytest.raises(ValueError, match="window"):
        rp._int32(4.0, "window")


SHAPES = [
    # tokens, query heads, key heads, head size, starts, window, first tokens
    (1, 1, 1, 64, [0, 1], 1, 0), (1, 4, 2, 128, [0, 1], 5, 128), (64, 2, 2, 64, list(range(65)), 3, 1), (127, 2, 1, 128, [0, 127], 1, 0),
    (128, 1, 1, 64, [0, 128], 127, 1), (129, 1, 1, 128, [0, 129], 128, 0), (257, 3, 1, 64, [0, 256, 257], 129, 2), (300, 2, 1, 128, [0, 0, 5, 133, 133, 300], 40, 7),
    (500, 4, 4, 64, [17, 200, 444], 100, 128), (384, 2, 1, 96, [0, 100, 384], 1, 1), (640, 2, 2, 80, [-7, 300, 700], 256, 4), (700, 2, 1, 8, [0, 700], 255, 127),
    (1000, 5, 1, 128, [0, 1, 2, 130, 600, 1000], 64, 33), (2049, 2, 1, 64, [0, 2049], 300, 3), (1500, 6, 2, 120, [0, 700, 1500], 513, 0),
    (4096, 1, 1, 128, [0, 1024, 4096], 130, 1), (777, 16, 4, 128, [0, 777], 10000, 20), (4999, 4, 2, 64, [0, 300, 4999], 129, 9), (2177, 2, 1, 128, [0, 2177], 2, 128),
    (2500, 3, 1, 72, [0, 2300, 2500], 1000, 100),
]
IDS = [f"{s[0]}-{s[1]}-{s[2]}-{s[3]}-w{s[5]}-s{s[6]}" for s in SHAPES]


def inputs(shape, kind, extra=0):
    """q, k, v as slices of one tensor, as a projection of all three leaves them."""
    import torch
    T, hq, hk, d = shape[:4]
    g = torch.Generator().manual_seed(T + d)
    wide = torch.randn(T, hq + 2 * hk, d + extra, generator=g).to(getattr(torch, kind)).cuda()
    return wide[:, :hq, :d], wide[:, hq:hq + hk, :d], wide[:, hq + hk:, :d], g


@pytest.mark.gpu
@pytest.mark.parametrize("kind,extra", [("bfloat16", 0), ("float16", 8)])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_forward(shape, kind, extra):
    import torch
    T, hq, hk, d, start, window, sinks = shape
    q, k, v, _ = inputs(shape, kind, extra)
    out, lse = rp.rp_attend_window(q, k, v, torch.tensor(start, device="cuda"), window=window, sinks=sinks, scale=0.2)
    half = torch.finfo(q.dtype).eps / 2
    held = torch.zeros(T, dtype=torch.bool)
    for lo, hi in samples(start, T):
        held[lo:hi] = True
        mask = hidden(hi - lo, window, sinks)
        for h in range(hq):
            p, w_lse = weights(q[lo:hi, h].double(), k[lo:hi, h // (hq // hk)].double(), 0.2, mask)
            v64 = v[lo:hi, h // (hq // hk)].double()
            want, size = p @ v64, p @ v64.abs()
            # every weight and the output rounded once; scores in 32 bits (|s| <= 20: 1e-5 of a weight); values under the 16-bit types' normal range
            assert ((out[lo:hi, h].double() - want).abs() <= half * (size + want.abs()) + 1e-5 * size + 1e-7).all()
            assert ((lse[lo:hi, h].double() - w_lse).abs() <= 4e-6 * (1 + w_lse.abs())).all()
    assert (out[~held.cuda()] == 0).all() and (lse[~held.cuda()] == 0).all()


def gradients(q, k, v, do, scale, mask):
    """Gradients of one sample and head in 64 bits, and the sums of magnitudes that their roundings go by."""
    p, _ = weights(q, k, scale, mask)
    o = p @ v
    dp = do @ v.T
    delta = (do * o).sum(1, keepdim=True)
    ds = p * (dp - delta)
    # ds is off by its own rounding, and by what o's rounding does to delta
    slip = p * (do * o).abs().sum(1, keepdim=True)
    return (ds @ k * scale, ds.T @ q * scale, p.T @ do), (ds.abs() @ k.abs() * scale, ds.abs().T @ q.abs() * scale, p.T @ do.abs()), \
        (slip @ k.abs() * scale, slip.T @ q.abs() * scale, 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("kind,extra", [("bfloat16", 0), ("float16", 8)])
@pytest.mark.parametrize("shape", SHAPES, ids=IDS)
def test_gradient(shape, kind, extra):
    import torch
    T, hq, hk, d, start, window, sinks = shape
    q, k, v, g = inputs(shape, kind, extra)
    st, scale, share = torch.tensor(start, device="cuda"), 0.2, hq // hk
    do = torch.randn(hq, T, d + 8, generator=g).to(q.dtype).cuda()[:, :, :d].transpose(0, 1)
    out, lse = rp.rp_attend_window(q, k, v, st, window=window, sinks=sinks, scale=scale)
    got = rp.rp_attend_window_grad(do, q, k, v, out, lse, st, window=window, sinks=sinks, scale=scale)
    half = torch.finfo(q.dtype).eps / 2
    held = torch.zeros(T, dtype=torch.bool)
    for lo, hi in samples(start, T):
        held[lo:hi] = True
        mask = hidden(hi - lo, window, sinks)
        want, size, slip = [[torch.zeros(hi - lo, n, d, dtype=torch.float64, device="cuda") for n in (hq, hk, hk)] for _ in range(3)]
        for h in range(hq):
            a = [x[lo:hi, h // n].double() for x, n in ((q, 1), (k, share), (v, share), (do, 1))]
            for to, parts in zip((want, size, slip), gradients(*a, scale, mask)):
                for i, n in enumerate((1, share, share)):
                    to[i][:, h // n] += parts[i]
        for x, w, s, e in zip(got, want, size, slip):
            # each weight (or gradient of a score) and the result rounded once, delta by the rounding of o; 32 bits: 1e-5 of the weights;
            # float16 numbers of less than 2^-14 are off by 2^-25 at most, in up to T terms of |x| <= 6
            tol = half * (s + w.abs() + e) + 2e-5 * (s + e) + (1e-7 + 2.0 ** -25 * 6 * (hi - lo) * share * (kind == "float16"))
            assert ((x[lo:hi].double() - w).abs() <= tol).all()
    for x in got:
        assert x.dtype == q.dtype and (x[~held.cuda()] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("d", [64, 128])
def test_a_window_as_long_as_the_samples_is_none(d, kind):
    """The same bits as the attention without a window, whatever the first tokens are; the gradients of queries from each sample's 33rd token on, and of values (the scores'
    gradients of tokens before that are worked out from the weights here, from the rounded output there)."""
    import torch
    start = [0, 500, 501, 3000]
    q, k, v, g = inputs((3000, 4, 2, d), kind)
    st = torch.tensor(start, device="cuda")
    do = torch.randn(3000, 4, d, generator=g).to(q.dtype).cuda()
    want = rp.rp_attend(q, k, v, st)
    back = rp.rp_attend_grad(do, q, k, v, *want, st)
    for window, sinks in ((2499, 0), (2600, 17), (1 << 40, 128)):
        got = rp.rp_attend_window(q, k, v, st, window=window, sinks=sinks)
        assert all((a == b).all() for a, b in zip(got, want))
        dq, dk, dv = rp.rp_attend_window_grad(do, q, k, v, *got, st, window=window, sinks=sinks)
        assert (dv == back[2]).all() and torch.isfinite(dk).all()
        for lo, hi in samples(start, 3000):
            assert (dq[lo + 32:hi] == back[0][lo + 32:hi]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("window,sinks", [(1, 0), (100, 0), (100, 5), (700, 128)])
def test_samples_of_a_row_get_what_they_get_alone(window, sinks):
    """Bit for bit, with rows of no sample, samples of no token and one whose first tokens' gradients meet in chunks."""
    import torch
    lengths = [0, 1, 127, 128, 129, 255, 256, 257, 0, 0, 700, 4500, 2, 0] + [1] * 40 + [0] * 1500 + [2100, 33]
    start = [3] + (3 + np.cumsum(lengths)).tolist()
    T = start[-1] + 5
    q, k, v, g = inputs((T, 2, 1, 64), "bfloat16")
    st = torch.tensor(start, device="cuda")
    do = torch.randn(T, 2, 64, generator=g).bfloat16().cuda()
    kw = dict(window=window, sinks=sinks)
    out, lse = rp.rp_attend_window(q, k, v, st, **kw)
    grads = rp.rp_attend_window_grad(do, q, k, v, out, lse, st, **kw)
    for lo, hi in samples(start, T):
        one = torch.tensor([0, hi - lo], device="cuda")
        o, l = rp.rp_attend_window(q[lo:hi], k[lo:hi], v[lo:hi], one, **kw)
        assert (o == out[lo:hi]).all() and (l == lse[lo:hi]).all()
        for a, b in zip(rp.rp_attend_window_grad(do[lo:hi], q[lo:hi], k[lo:hi], v[lo:hi], o, l, one, **kw), grads):
            assert (a == b[lo:hi]).all()
    for x in (out, lse, *grads):
        assert (x[:3] == 0).all() and (x[-5:] == 0).all()


@pytest.mark.gpu
def test_rows_that_lie_beyond_32_bits():
    """Elements 2^31 and more from a tensor's first one, inputs and outputs of both directions."""
    import torch
    T, hq, hk, d, step = 1300, 4, 2, 64, 1 << 21
    g = torch.Generator().manual_seed(6)
    start, kw = torch.tensor([0, 900, T], device="cuda"), dict(window=300, sinks=5)

    def apart(heads, x=None):
        y = torch.empty(T, step, dtype=torch.bfloat16, device="cuda")[:, :heads * d].view(T, heads, d)
        return y if x is None else y.copy_(x)
    q, k, v, do = (torch.randn(T, h, d, generator=g).bfloat16().cuda() for h in (hq, hk, hk, hq))
    out, lse = rp.rp_attend_window(q, k, v, start, **kw)
    grads = rp.rp_attend_window_grad(do, q, k, v, out, lse, start, **kw)
    q, k, v, do = apart(hq, q), apart(hk, k), apart(hk, v), apart(hq, do)
    o, l = rp.rp_attend_window(q, k, v, start, out=apart(hq), **kw)
    assert (o == out).all() and (l == lse).all()
    for a, b in zip(rp.rp_attend_window_grad(do, q, k, v, o, l, start, q_grad=apart(hq), k_grad=apart(hk), v_grad=apart(hk), **kw), grads):
        assert (a == b).all()


@pytest.mark.gpu
def test_other_samples_and_keys_out_of_sight_do_not_matter():
    """Infinities and NaN in the tokens of other samples, in the row's padding, and in keys that no query near them sees."""
    import torch
    shape = (3200, 2, 1, 128, [0, 70, 2900, 3100])
    st = torch.tensor(shape[4], device="cuda")
    q, k, v, g = inputs(shape, "bfloat16")
    do = torch.randn(3200, 2, 128, generator=g).bfloat16().cuda()
    kw = dict(window=50, sinks=3)
    want = rp.rp_attend_window(q, k, v, st, **kw)
    back = rp.rp_attend_window_grad(do, q, k, v, *want, st, **kw)
    bad = [x.clone() for x in (q, k, v, do, *want)]
    for x in bad:
        x[:70] = float("nan")
        x[2900:3100] = float("inf")
        x[3100:] = float("nan")
    big = torch.full((3205, 2, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((3205, 2), 3.0, device="cuda")
    rp.rp_attend_window(*bad[:3], st, out=big[:3200], lse=lse[:3200], **kw)
    assert (big[70:2900] == want[0][70:2900]).all() and (lse[70:2900] == want[1][70:2900]).all()
    assert (big[3100:3200] == 0).all() and (big[3200:] == 3).all() and (lse[3200:] == 3).all()
    big = [torch.full((3205, n, 128), 3.0, dtype=torch.bfloat16, device="cuda") for n in (2, 1, 1)]
    rp.rp_attend_window_grad(bad[3], *bad[:3], *bad[4:], st, q_grad=big[0][:3200], k_grad=big[1][:3200], v_grad=big[2][:3200], **kw)
    for x, w in zip(big, back):
        assert (x[70:2900] == w[70:2900]).all() and (x[3100:3200] == 0).all() and (x[3200:] == 3).all()
    # keys (not values) that the last 1000 tokens do not see
    far = k.clone()
    far[80:1800] = float("nan")
    got = rp.rp_attend_window(q, far, v, st, **kw)
    assert (got[0][1900:2900] == want[0][1900:2900]).all() and (got[1][1900:2900] == want[1][1900:2900]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
def test_low_scores_in_the_window_and_far_first_tokens(kind):
    """Windows whose scores are -inf but for the first tokens, or the other way round; a maximum that falls as the window moves on."""
    import torch
    T, d = 900, 64
    q = torch.zeros(T, 1, d, device="cuda", dtype=getattr(torch, kind))
    k, v = torch.zeros_like(q), torch.randn(T, 1, d, generator=torch.Generator().manual_seed(1)).cuda().to(q.dtype)
    st = torch.tensor([0, T], device="cuda")
    q[:, :, 0] = 1
    for first, rest in ((0.0, -math.inf), (-math.inf, 0.0), (0.0, -3e4), (-3e4, 0.0), (3e4, -3e4)):
        k[:, :, 0] = rest
        k[:4, :, 0] = first
        out, lse = rp.rp_attend_window(q, k, v, st, window=60, sinks=4, scale=1.0)
        p, w = weights(q[:, 0].double(), k[:, 0].double().clamp(min=-1e30), 1.0, hidden(T, 60, 4))
        rows = torch.isfinite(q[:, 0].double() @ k[:, 0].double().T).logical_and(~hidden(T, 60, 4)).any(1)      # (rows of nothing but -inf have no weights)
        want, half = p @ v[:, 0].double(), torch.finfo(q.dtype).eps / 2
        size = p @ v[:, 0].double().abs()
        assert rows.sum() >= T - 4 and ((out[:, 0].double() - want).abs() <= half * (size + want.abs()) + 1e-5 * size + 1e-7)[rows].all()
        assert ((lse[:, 0].double() - w).abs() <= 4e-6 * (1 + w.abs()))[rows].all()
    ramp = torch.linspace(30, -30, T, device="cuda")
    k[:, 0, 0] = ramp.to(k.dtype)
    out, lse = rp.rp_attend_window(q, k, v, st, window=200, sinks=2, scale=1.0)
    p, w = weights(q[:, 0].double(), k[:, 0].double(), 1.0, hidden(T, 200, 2))
    want, size = p @ v[:, 0].double(), p @ v[:, 0].double().abs()
    assert ((out[:, 0].double() - want).abs() <= torch.finfo(q.dtype).eps / 2 * (size + want.abs()) + 1e-5 * size + 1e-7).all()
    assert ((lse[:, 0].double() - w).abs() <= 4e-6 * (1 + w.abs())).all()


@pytest.mark.gpu
def test_gradient_against_differences():
    import torch
    T, start = 14, [0, 4, 14]
    g = torch.Generator().manual_seed(8)
    q, k, v, do = [(torch.randn(T, 2 if i in (0, 3) else 1, 16, generator=g) * 0.5).half() for i in range(4)]
    st = torch.tensor(start, device="cuda")
    dev = [x.cuda() for x in (q, k, v)]
    out, lse = rp.rp_attend_window(*dev, st, window=3, sinks=2)
    got = rp.rp_attend_window_grad(do.cuda(), *dev, out, lse, st, window=3, sinks=2)

    def value(q, k, v):
        total = 0.0
        for lo, hi in samples(start, T):
            for h in range(2):
                p, _ = weights(q[lo:hi, h], k[lo:hi, 0], 0.25, hidden(hi - lo, 3, 2, "cpu"))
                total += (p @ v[lo:hi, 0] * do[lo:hi, h].double()).sum().item()
        return total
    leaves = [x.double() for x in (q, k, v)]
    for i, x in enumerate(leaves):
        for at in [(0, 0, 0), (3, 0, 5), (4, 0, 15), (5, 0, 2), (8, 0, 1), (13, 0, 7)] + ([(13, 1, 2)] if i == 0 else []):
            up, down = [y.clone() for y in leaves], [y.clone() for y in leaves]
            up[i][at] += 1e-4
            down[i][at] -= 1e-4
            # (roundings of float16, 2^-11 each of sums of a few terms below 2)
            assert abs((value(*up) - value(*down)) / 2e-4 - got[i][at].item()) < 4e-3


@pytest.mark.gpu
def test_repeated_streamed_and_captured_calls_agree_bit_for_bit():
    import torch
    shape = (6000, 8, 2, 128, [0, 500, 501, 6000])
    q, k, v, g = inputs(shape, "bfloat16")
    st = torch.tensor(shape[4], device="cuda")
    do = torch.randn(6000, 8, 128, generator=g).bfloat16().cuda()
    kw = dict(window=333, sinks=6)

    def both(**more):
        o, l = rp.rp_attend_window(q, k, v, st, **kw, **more)
        return (o, l, *rp.rp_attend_window_grad(do, q, k, v, o, l, st, **kw, **more))
    want = both()
    torch.cuda.synchronize()
    results = [both(stream=s) for s in [torch.cuda.Stream() for _ in range(4)] for _ in range(3)]
    torch.cuda.synchronize()
    for got in results:
        assert all((a == b).all() for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))


@pytest.mark.gpu
def test_no_tokens_and_places_that_are_shared():
    import torch
    q = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    start, status = torch.tensor([0, 0], device="cuda"), torch.full((1,), 7, dtype=torch.int32, device="cuda")
    out, lse = rp.rp_attend_window(q, q, q, start, window=4, status=status)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2) and status.item() == 0
    q, k, v, o = [torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    start = torch.tensor([0, 4], device="cuda")
    with pytest.raises(rp.RpError, match="ARG"):
        rp.rp_attend_window(q, k, v, start, window=4, out=q)
    out, lse = rp.rp_attend_window(q, k, v, start, window=4)
    with pytest.raises(rp.RpError, match="ARG"):
        rp.rp_attend_window_grad(o, q, k, v, out, lse, start, window=4, q_grad=q)
    for kw in (dict(window=0), dict(window=4, sinks=-1)):
        with pytest.raises(rp.RpError, match="ARG"):
            rp.rp_attend_window(q, k, v, start, **kw)
    with pytest.raises(rp.RpError, match="RANGE"):
        rp.rp_attend_window(q, k, v, start, window=4, sinks=129)


@pytest.mark.gpu
def test_waits_that_run_out_leave_nan_and_a_status():
    import torch
    shape = (5000, 4, 2, 128, [0, 500, 5000])
    q, k, v, g = inputs(shape, "bfloat16")
    st, kw = torch.tensor(shape[4], device="cuda"), dict(window=200, sinks=4)
    do = torch.randn(5000, 4, 128, generator=g).bfloat16().cuda()
    status = [torch.full((1,), 7, dtype=torch.int32, device="cuda") for _ in range(4)]
    want = rp.rp_attend_window(q, k, v, st, status=status[0], **kw)
    back = rp.rp_attend_window_grad(do, q, k, v, *want, st, status=status[1], **kw)
    rp.rp_debug_set_wait_limit(0)
    try:
        got = rp.rp_attend_window(q, k, v, st, status=status[2], **kw)
        grads = rp.rp_attend_window_grad(do, q, k, v, *want, st, status=status[3], **kw)
        torch.cuda.synchronize()
    finally:
        rp.rp_debug_set_wait_limit()
    assert [s.item() for s in status] == [0, 0, -8, -8]
    assert all(torch.isnan(x).all() for x in (*got, *grads))
    again = rp.rp_attend_window(q, k, v, st, **kw)
    assert all((a == b).all() for a, b in zip(again, want))
    assert all((a == b).all() for a, b in zip(rp.rp_attend_window_grad(do, q, k, v, *again, st, **kw), back))


@pytest.mark.gpu
@pytest.mark.parametrize("limit", [1, 2000, 8000, 40000])
def test_short_limits_leave_right_rows_or_nan(limit):
    """Whatever wait runs out first: a row is right to the last bit or NaN, and NaN anywhere comes with the status."""
    import torch
    shape = (9000, 4, 2, 64, [0, 400, 9000])
    q, k, v, g = inputs(shape, "bfloat16")
    st, kw = torch.tensor(shape[4], device="cuda"), dict(window=300, sinks=4)
    do = torch.randn(9000, 4, 64, generator=g).bfloat16().cuda()
    want = rp.rp_attend_window(q, k, v, st, **kw)
    back = rp.rp_attend_window_grad(do, q, k, v, *want, st, **kw)
    status = [torch.full((1,), 7, dtype=torch.int32, device="cuda") for _ in range(2)]
    rp.rp_debug_set_wait_limit(limit)
    try:
        got = rp.rp_attend_window(q, k, v, st, status=status[0], **kw)
        grads = rp.rp_attend_window_grad(do, q, k, v, *want, st, status=status[1], **kw)
        torch.cuda.synchronize()
    finally:
        rp.rp_debug_set_wait_limit()
    for s, a, b in ((status[0], got, want), (status[1], grads, back)):
        assert s.item() in (0, -8)
        for x, y in zip(a, b):
            lost = torch.isnan(x)
            assert (x[~lost] == y[~lost]).all() and (s.item() == -8 or not lost.any())


@pytest.mark.gpu
def test_rows_without_samples_and_many_short_ones():
    """No block at all, and more CTAs than blocks: zeros, no wait runs out; thousands of samples of a few tokens."""
    import torch
    q, k, v, g = inputs((1300, 2, 1, 64), "bfloat16")
    do = torch.randn(1300, 2, 64, generator=g).bfloat16().cuda()
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    for start in ([0, 0], [1300, 1300], [5, 5, 5, 5], [-9, 0], [1200, 100]):
        st = torch.tensor(start, device="cuda")
        out, lse = rp.rp_attend_window(q, k, v, st, window=7, sinks=3, status=status)
        assert (out == 0).all() and (lse == 0).all() and status.item() == 0
        for x in rp.rp_attend_window_grad(do, q, k, v, out, lse, st, window=7, sinks=3, status=status):
            assert (x == 0).all() and status.item() == 0
    x = torch.randn(12000, 4, 64, generator=torch.Generator().manual_seed(9)).half().cuda()
    st = torch.arange(0, 12001, 3, device="cuda")
    out, lse = rp.rp_attend_window(x[:, :2], x[:, 2:3], x[:, 3:], st, window=2)
    want, w_lse = rp.rp_attend(x[:, :2], x[:, 2:3], x[:, 3:], st)
    two = torch.arange(12000, device="cuda") % 3 < 2                     # (the third token of each sees two of three)
    assert (out[two] == want[two]).all() and (lse[two] == w_lse[two]).all() and not (out[~two] == want[~two]).all()


FEW = [
    # tokens, query heads, key heads, head size, starts, window, first tokens: no token sees more than 32 keys
    (1, 1, 1, 64, [0, 1], 1, 0), (700, 2, 1, 64, [3, 20, 20, 21, 300, 690], 1, 0), (900, 4, 2, 128, [0, 17, 600, 900], 2, 0), (1000, 2, 2, 64, [-5, 1, 400, 1200], 4, 1),
    (2500, 3, 1, 96, [0, 2300, 2500], 16, 16), (1300, 2, 1, 8, [0, 129, 1300], 1, 31), (600, 5, 1, 72, [0, 33, 97, 600], 8, 0), (3000, 2, 1, 128, [0, 500, 2999], 32, 0),
    (640, 8, 2, 64, list(range(0, 641, 32)), 1000, 3), (500, 2, 1, 120, [0] + list(range(2, 500, 31)), 33, 128),
]


@pytest.mark.gpu
@pytest.mark.parametrize("kind,extra", [("bfloat16", 0), ("float16", 8)])
@pytest.mark.parametrize("shape", FEW, ids=[f"{s[0]}-{s[1]}-{s[2]}-{s[3]}-w{s[5]}-s{s[6]}" for s in FEW])
def test_gradient_where_few_keys_are_seen(shape, kind, extra):
    """As exact as one rounding of each weight, score's gradient and result: what the rounding of `out` would do to the sum of out_grad * out does not come in, nor does `out`."""
    import torch
    T, hq, hk, d, start, window, sinks = shape
    q, k, v, g = inputs(shape, kind, extra)
    st, scale, share = torch.tensor(start, device="cuda"), 0.2, hq // hk
    do = torch.randn(hq, T, d + 8, generator=g).to(q.dtype).cuda()[:, :, :d].transpose(0, 1)
    out, lse = rp.rp_attend_window(q, k, v, st, window=window, sinks=sinks, scale=scale)
    got = rp.rp_attend_window_grad(do, q, k, v, out, lse, st, window=window, sinks=sinks, scale=scale)
    half = torch.finfo(q.dtype).eps / 2
    for lo, hi in samples(start, T):
        mask = hidden(hi - lo, window, sinks)
        want, size, slip = [[torch.zeros(hi - lo, n, d, dtype=torch.float64, device="cuda") for n in (hq, hk, hk)] for _ in range(3)]
        for h in range(hq):
            a = [x[lo:hi, h // n].double() for x, n in ((q, 1), (k, share), (v, share), (do, 1))]
            for to, parts in zip((want, size, slip), gradients(*a, scale, mask)):
                for i, n in enumerate((1, share, share)):
                    to[i][:, h // n] += parts[i]
        for x, w, s, e in zip(got, want, size, slip):
            # each weight (or gradient of a score) and the result rounded once; 32 bits: 1e-5 of the weights and of the products with values, whose difference the
            # gradient of a score is; float16 numbers of less than 2^-14 are off by 2^-25 at most, in up to T terms of |x| <= 6
            tol = half * (s + w.abs() + half * s) + 2e-5 * (s + e) + (1e-7 + 2.0 ** -25 * 6 * (hi - lo) * share * (kind == "float16"))
            assert ((x[lo:hi].double() - w).abs() <= tol).all()
    nothing = torch.full_like(out, float("nan"))
    for x, w in zip(rp.rp_attend_window_grad(do, q, k, v, nothing, lse, st, window=window, sinks=sinks, scale=scale), got):
        assert (x == w).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
def test_first_tokens_do_not_go_by_the_rounded_output(kind):
    """The first 32 of each sample, with a window in which the others see more: `out` there may be anything; the 33rd goes by it."""
    import torch
    shape = (1500, 4, 2, 128, [2, 30, 62, 95, 1490], 200, 5)
    q, k, v, g = inputs(shape, kind)
    st, kw = torch.tensor(shape[4], device="cuda"), dict(window=200, sinks=5)
    do = torch.randn(1500, 4, 128, generator=g).to(q.dtype).cuda()
    out, lse = rp.rp_attend_window(q, k, v, st, **kw)
    want = rp.rp_attend_window_grad(do, q, k, v, out, lse, st, **kw)
    other = out.clone()
    for lo, hi in samples(shape[4], 1500):
        other[lo:min(lo + 32, hi)] = float("nan")
    assert all((x == w).all() for x, w in zip(rp.rp_attend_window_grad(do, q, k, v, other, lse, st, **kw), want))
    other = out.clone()
    other[62 + 32] += 1
    assert (rp.rp_attend_window_grad(do, q, k, v, other, lse, st, **kw)[0] != want[0])[62 + 32].any()
    # the keys' gradient as the definition has it, where the attention without a window takes the rounded output
    lo, hi = 62, 95
    for h in range(2):
        dk = sum(gradients(*(x[lo:hi, y].double() for x, y in ((q, 2 * h + i), (k, h), (v, h), (do, 2 * h + i))), 128 ** -0.5, hidden(hi - lo, 200, 5))[0][1] for i in range(2))
        plain = rp.rp_attend_grad(do, q, k, v, *rp.rp_attend(q, k, v, st), st)[1][lo:hi, h].double()
        assert (want[1][lo:hi, h].double() - dk).norm() < (plain - dk).norm()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("window,sinks", [(9, 5), (32, 0), (2, 30)])
def test_few_keys_alone_in_a_row_far_apart_and_captured(window, sinks, kind):
    """Where no token sees more than 32 keys: a sample's bits are the same alone and among samples of NaN and infinities, with rows 2^31 elements from the first, on another
    stream and replayed."""
    import torch
    T, hq, hk, d, step = 1300, 6, 2, 64, 1 << 21
    start = [4, 4, 5, 38, 200, 201, 1290]
    q, k, v, g = inputs((T, hq, hk, d), kind)
    do = torch.randn(T, hq, d, generator=g).to(q.dtype).cuda()
    st, kw = torch.tensor(start, device="cuda"), dict(window=window, sinks=sinks)
    out, lse = rp.rp_attend_window(q, k, v, st, **kw)
    want = rp.rp_attend_window_grad(do, q, k, v, out, lse, st, **kw)
    for lo, hi in samples(start, T):
        one, cut = torch.tensor([0, hi - lo], device="cuda"), slice(lo, hi)
        for a, b in zip(rp.rp_attend_window_grad(do[cut], q[cut], k[cut], v[cut], out[cut], lse[cut], one, **kw), want):
            assert (a == b[cut]).all()
        bad = [x.clone() for x in (do, q, k, v, out, lse)]
        for x in bad:
            x[:lo], x[hi:] = float("nan"), float("inf")
        for a, b in zip(rp.rp_attend_window_grad(*bad, st, **kw), want):
            assert (a[cut] == b[cut]).all() and (a[:4] == 0).all() and (a[1290:] == 0).all()

    def apart(heads, x=None):
        y = torch.empty(T, step, dtype=q.dtype, device="cuda")[:, :heads * d].view(T, heads, d)
        return y if x is None else y.copy_(x)
    far = [apart(x.shape[1], x) for x in (do, q, k, v)]
    for a, b in zip(rp.rp_attend_window_grad(*far, out, lse, st, q_grad=apart(hq), k_grad=apart(hk), v_grad=apart(hk), **kw), want):
        assert (a == b).all()
    del far
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    results = [rp.rp_attend_window_grad(do, q, k, v, out, lse, st, stream=side, **kw) for _ in range(3)]
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        results.append(rp.rp_attend_window_grad(do, q, k, v, out, lse, st, **kw))
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    for got in results:
        assert all((a == b).all() for a, b in zip(got, want))
