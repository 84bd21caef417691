"""Attention inside the samples of a packed row, and its gradient, against the formulas in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp


def weights(q, k, scale, causal):
    """Softmax weights [n, n] of one sample and one head, and the log of each row's sum, in 64 bits."""
    import torch
    s = q @ k.T * scale
    if causal:
        s = s.masked_fill(torch.ones_like(s, dtype=torch.bool).triu(1), -math.inf)
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

    def view(x=p, token=128, head=64):
        return C.byref(rp.rp_view(x, token, head))

    def fwd(cfg=a(), T=2, q=view(), k=view(), v=view(), start=p, N=1, out=view(), lse=None, space=p, nbytes=1 << 14):
        return lib.rp_attend(cfg, T, q, k, v, start, N, out, lse, space, nbytes, None)

    assert fwd() == -1                                   # host arrays
    for bad in (dict(cfg=None), dict(T=-1), dict(N=0), dict(start=None), dict(start=p + 4), dict(space=None), dict(space=p + 8), dict(nbytes=8), dict(q=None),
                dict(k=view(x=None)), dict(v=view(x=p + 8)), dict(out=view(token=0)), dict(q=view(head=-64)), dict(k=view(token=100)), dict(cfg=a(hq=0)),
                dict(cfg=a(kind=0)), dict(cfg=a(causal=2)), dict(cfg=a(scale=0.0)), dict(cfg=a(scale=-1.0)), dict(cfg=a(scale=math.inf)),
                dict(cfg=a(scale=math.nan))):
        assert fwd(**bad) == -1, bad
    assert fwd(cfg=a(hq=3, hk=2)) == -2 and fwd(cfg=a(d=60)) == -2 and fwd(cfg=a(d=136)) == -5 and fwd(T=(1 << 31) - 512) == -5
    assert lib.rp_attend_workspace(None, 1, 1) == 0 and lib.rp_attend_workspace(a(), 1, 0) == 0 and lib.rp_attend_workspace(a(), 1000, 3) > 0


SHAPES = [
    # tokens, query heads, key heads, head size, starts
    (1, 1, 1, 64, [0, 1]), (1, 4, 2, 128, [0, 1]), (64, 2, 2, 64, list(range(65))), (127, 2, 1, 128, [0, 127]), (128, 1, 1, 64, [0, 128]),
    (129, 1, 1, 128, [0, 129]), (257, 3, 1, 64, [0, 256, 257]), (300, 2, 1, 128, [0, 0, 5, 133, 133, 300]), (500, 4, 4, 64, [17, 200, 444]),
    (384, 2, 1, 96, [0, 100, 384]), (640, 2, 2, 80, [-7, 300, 700]), (700, 2, 1, 8, [0, 700]), (1000, 5, 1, 128, [0, 1, 2, 130, 600, 1000]),
    (2049, 2, 1, 64, [0, 2049]), (1500, 6, 2, 120, [0, 700, 1500]), (4096, 1, 1, 128, [0, 1024, 4096]), (777, 16, 4, 128, [0, 777]),
]


def inputs(shape, kind, extra=0):
    """q, k, v as slices of one tensor, as a projection of all three leaves them."""
    import torch
    T, hq, hk, d, start = shape
    g = torch.Generator().manual_seed(T + d)
    wide = torch.randn(T, hq + 2 * hk, d + extra, generator=g).to(getattr(torch, kind)).cuda()
    return wide[:, :hq, :d], wide[:, hq:hq + hk, :d], wide[:, hq + hk:, :d], g


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,extra", [("bfloat16", 0), ("float16", 8)])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(s[:4]) for s in SHAPES])
def test_forward(shape, kind, extra, causal):
    import torch
    T, hq, hk, d, start = shape
    q, k, v, _ = inputs(shape, kind, extra)
    out, lse = rp.rp_attend(q, k, v, torch.tensor(start, device="cuda"), causal=causal, scale=0.2)
    half = torch.finfo(q.dtype).eps / 2
    seen = torch.zeros(T, dtype=torch.bool)
    for lo, hi in samples(start, T):
        seen[lo:hi] = True
        for h in range(hq):
            p, w_lse = weights(q[lo:hi, h].double(), k[lo:hi, h // (hq // hk)].double(), 0.2, causal)
            v64 = v[lo:hi, h // (hq // hk)].double()
            want, size = p @ v64, p @ v64.abs()
            # every weight and the output rounded once; scores in 32 bits (|s| <= 20: 1e-5 of a weight); values under the 16-bit types' normal range
            assert ((out[lo:hi, h].double() - want).abs() <= half * (size + want.abs()) + 1e-5 * size + 1e-7).all()
            assert ((lse[lo:hi, h].double() - w_lse).abs() <= 4e-6 * (1 + w_lse.abs())).all()
    assert (out[~seen.cuda()] == 0).all() and (lse[~seen.cuda()] == 0).all()


@pytest.mark.gpu
def test_other_samples_do_not_matter():
    """Infinities and NaN in the tokens of other samples and in the row's padding; the rows behind the outputs stay."""
    import torch
    shape = (400, 2, 1, 128, [0, 70, 211, 330])
    start = torch.tensor(shape[4], device="cuda")
    q, k, v, g = inputs(shape, "bfloat16")
    want = rp.rp_attend(q, k, v, start)
    bad = [x.clone() for x in (q, k, v)]
    for x in bad:
        x[:70] = float("nan")
        x[211:300] = float("inf")
        x[330:] = float("nan")
    big = torch.full((405, 2, 128), 3.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((405, 2), 3.0, device="cuda")
    rp.rp_attend(*bad, start, out=big[:400], lse=lse[:400])
    assert (big[70:211] == want[0][70:211]).all() and (lse[70:211] == want[1][70:211]).all()
    assert (big[330:400] == 0).all() and (big[400:] == 3).all() and (lse[400:] == 3).all()


@pytest.mark.gpu
def test_scores_far_apart():
    """Rows whose maximum grows by much from tile to tile, and rows that one key takes whole."""
    import torch
    T = 1024
    q, k, v, g = inputs((T, 1, 1, 64, [0, T]), "bfloat16")
    k = (k * torch.linspace(0.1, 30, T, device="cuda")[:, None, None]).bfloat16()
    out, lse = rp.rp_attend(q, k, v, torch.tensor([0, T], device="cuda"), causal=True, scale=0.125)
    p, w_lse = weights(q[:, 0].double(), k[:, 0].double(), 0.125, True)
    size = p @ v[:, 0].double().abs()
    # (scores to 250: 32 bits leave them 2e-5, so 3e-5 of a weight)
    assert ((out[:, 0].double() - p @ v[:, 0].double()).abs() <= 2.0 ** -8 * (size + (p @ v[:, 0].double()).abs()) + 6e-5 * size).all()
    assert ((lse[:, 0].double() - w_lse).abs() <= 4e-6 * (1 + w_lse.abs())).all()


@pytest.mark.gpu
def test_repeated_streamed_and_captured_calls_agree_bit_for_bit():
    import torch
    shape = (3000, 8, 2, 128, [0, 500, 501, 3000])
    q, k, v, _ = inputs(shape, "bfloat16")
    start = torch.tensor(shape[4], device="cuda")
    want = rp.rp_attend(q, k, v, start)
    torch.cuda.synchronize()
    results = [rp.rp_attend(q, k, v, start, stream=s) for s in [torch.cuda.Stream() for _ in range(4)] for _ in range(3)]
    torch.cuda.synchronize()
    for got in results:
        assert all((a == b).all() for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = rp.rp_attend(q, k, v, start)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))


@pytest.mark.gpu
def test_no_tokens():
    import torch
    q = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda")
    start = torch.tensor([0, 0], device="cuda")
    out, lse = rp.rp_attend(q, q, q, start)
    assert out.shape == (0, 2, 64) and lse.shape == (0, 2)
    space, view = torch.full((64,), 7, dtype=torch.int32, device="cuda"), C.byref(rp.rp_view(start.data_ptr(), 128, 64))
    cfg, stream = C.byref(rp.rp_attend_config(2, 2, 64, 2, 1, 0.1)), torch.cuda.current_stream().cuda_stream
    assert rp.lib().rp_attend(cfg, 0, view, view, view, start.data_ptr(), 1, view, None, space.data_ptr(), 256, stream) == 0 and space[0].item() == 0
    space.fill_(7)
    views = [view] * 6
    assert rp.lib().rp_attend_grad(cfg, 0, *views, start.data_ptr(), 1, view, view, view, space.data_ptr(), 256, stream) == 0 and space[0].item() == 0


@pytest.mark.gpu
def test_without_the_logs_of_the_sums():
    import torch
    q, k, v, _ = inputs((300, 2, 1, 64, [0, 100, 300]), "bfloat16")
    start = torch.tensor([0, 100, 300], device="cuda")
    want, _ = rp.rp_attend(q, k, v, start)
    out, space = torch.zeros(300, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.zeros(1024, dtype=torch.int32, device="cuda")

    def view(x):
        return C.byref(rp.rp_view(x.data_ptr(), x.stride(0), x.stride(1)))
    cfg, stream = C.byref(rp.rp_attend_config(2, 1, 64, 2, 1, 64 ** -0.5)), torch.cuda.current_stream().cuda_stream
    for lse in (None, C.byref(rp.rp_view(None, 0, 0))):
        out.zero_()
        assert rp.lib().rp_attend(cfg, 300, view(q), view(k), view(v), start.data_ptr(), 2, view(out), lse, space.data_ptr(), 4096, stream) == 0
        assert (out == want).all() and space[0].item() == 0


@pytest.mark.gpu
def test_samples_of_every_short_length():
    """Lists of samples of 0 to 6 blocks, many of no token."""
    import torch
    lengths = [0, 1, 127, 128, 129, 255, 256, 257, 0, 0, 700, 1400, 2, 0] + [1] * 40 + [0] * 1500 + [33]
    start = [0] + np.cumsum(lengths).tolist()
    q, k, v, g = inputs((start[-1], 2, 1, 64, start), "bfloat16")
    out, lse = rp.rp_attend(q, k, v, torch.tensor(start, device="cuda"))
    do = torch.randn(start[-1], 2, 64, generator=g).bfloat16().cuda()
    grads = rp.rp_attend_grad(do, q, k, v, out, lse, torch.tensor(start, device="cuda"))
    for lo, hi in samples(start, start[-1]):
        st = torch.tensor([0, hi - lo], device="cuda")
        o, l = rp.rp_attend(q[lo:hi], k[lo:hi], v[lo:hi], st)
        assert (o == out[lo:hi]).all() and (l == lse[lo:hi]).all()
        for a, b in zip(rp.rp_attend_grad(do[lo:hi], q[lo:hi], k[lo:hi], v[lo:hi], o, l, st), grads):
            assert (a == b[lo:hi]).all()


@pytest.mark.gpu
def test_outputs_in_the_place_of_inputs_are_refused():
    import torch
    q, k, v, o = [torch.zeros(4, 1, 64, dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    start = torch.tensor([0, 4], device="cuda")
    for bad in (q, k, v):
        with pytest.raises(rp.RpError, match="ARG"):
            rp.rp_attend(q, k, v, start, out=bad)
    out, lse = rp.rp_attend(q, k, v, start)
    for kw in (dict(q_grad=q), dict(q_grad=o), dict(k_grad=out), dict(v_grad=v), dict(k_grad=q.clone(), v_grad=None)):
        if kw.get("v_grad", 0) is None:
            kw["v_grad"] = kw["k_grad"]
        with pytest.raises(rp.RpError, match="ARG"):
            rp.rp_attend_grad(o, q, k, v, out, lse, start, **kw)


# ---- gradient ---------------------------------------------------------------------------
def gradients(q, k, v, do, scale, causal):
    """Gradients of one sample and head in 64 bits, and the sums of magnitudes that their roundings go by."""
    p, _ = weights(q, k, scale, causal)
    o = p @ v
    dp = do @ v.T
    delta = (do * o).sum(1, keepdim=True)
    ds = p * (dp - delta)
    # ds is off by its own rounding, and by what o's rounding does to delta
    slip = p * (do * o).abs().sum(1, keepdim=True)
    return (ds @ k * scale, ds.T @ q * scale, p.T @ do), (ds.abs() @ k.abs() * scale, ds.abs().T @ q.abs() * scale, p.T @ do.abs()), \
        (slip @ k.abs() * scale, slip.T @ q.abs() * scale, 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind,extra", [("bfloat16", 0), ("float16", 8)])
@pytest.mark.parametrize("shape", SHAPES, ids=[str(s[:4]) for s in SHAPES])
def test_gradient(shape, kind, extra, causal):
    import torch
    T, hq, hk, d, start = shape
    q, k, v, g = inputs(shape, kind, extra)
    st, scale, share = torch.tensor(start, device="cuda"), 0.2, hq // hk
    do = torch.randn(hq, T, d + 8, generator=g).to(q.dtype).cuda()[:, :, :d].transpose(0, 1)
    out, lse = rp.rp_attend(q, k, v, st, causal=causal, scale=scale)
    got = rp.rp_attend_grad(do, q, k, v, out, lse, st, causal=causal, scale=scale)
    half = torch.finfo(q.dtype).eps / 2
    seen = torch.zeros(T, dtype=torch.bool)
    for lo, hi in samples(start, T):
        seen[lo:hi] = True
        want, size, slip = [[torch.zeros(hi - lo, n, d, dtype=torch.float64, device="cuda") for n in (hq, hk, hk)] for _ in range(3)]
        for h in range(hq):
            a = [x[lo:hi, h // n].double() for x, n in ((q, 1), (k, share), (v, share), (do, 1))]
            for to, parts in zip((want, size, slip), gradients(*a, scale, causal)):
                for i, n in enumerate((1, share, share)):
                    to[i][:, h // n] += parts[i]
        for x, w, s, e in zip(got, want, size, slip):
            # each weight (or gradient of a score) and the result rounded once, delta by the rounding of o; 32 bits: 1e-5 of the weights;
            # float16 numbers of less than 2^-14 are off by 2^-25 at most, in up to T terms of |x| <= 6
            tol = half * (s + w.abs() + e) + 2e-5 * (s + e) + (1e-7 + 2.0 ** -25 * 6 * (hi - lo) * share * (kind == "float16"))
            assert ((x[lo:hi].double() - w).abs() <= tol).all()
    for x in got:
        assert x.dtype == q.dtype and (x[~seen.cuda()] == 0).all()


@pytest.mark.gpu
def test_gradient_against_differences():
    import torch
    T, start = 10, [0, 4, 10]
    g = torch.Generator().manual_seed(8)
    q, k, v, do = [(torch.randn(T, 2 if i in (0, 3) else 1, 16, generator=g) * 0.5).half() for i in range(4)]
    st = torch.tensor(start, device="cuda")
    dev = [x.cuda() for x in (q, k, v)]
    out, lse = rp.rp_attend(*dev, st)
    got = rp.rp_attend_grad(do.cuda(), *dev, out, lse, st)

    def value(q, k, v):
        total = 0.0
        for lo, hi in samples(start, T):
            for h in range(2):
                p, _ = weights(q[lo:hi, h], k[lo:hi, 0], 0.25, True)
                total += (p @ v[lo:hi, 0] * do[lo:hi, h].double()).sum().item()
        return total
    leaves = [x.double() for x in (q, k, v)]
    for i, x in enumerate(leaves):
        for at in [(0, 0, 0), (3, 0, 5), (4, 0, 15), (9, 0, 7)] + ([(9, 1, 2)] if i == 0 else []):
            up, down = [y.clone() for y in leaves], [y.clone() for y in leaves]
            up[i][at] += 1e-4
            down[i][at] -= 1e-4
            # (roundings of float16, 2^-11 each of sums of a few terms below 2)
            assert abs((value(*up) - value(*down)) / 2e-4 - got[i][at].item()) < 4e-3


@pytest.mark.gpu
def test_gradients_of_other_samples_do_not_matter():
    import torch
    shape = (400, 4, 2, 64, [0, 70, 211, 330])
    st = torch.tensor(shape[4], device="cuda")
    q, k, v, g = inputs(shape, "bfloat16")
    do = torch.randn(400, 4, 64, generator=g).bfloat16().cuda()
    out, lse = rp.rp_attend(q, k, v, st)
    want = rp.rp_attend_grad(do, q, k, v, out, lse, st)
    bad = [x.clone() for x in (do, q, k, v, out, lse)]
    for x in bad:
        x[:70] = float("nan")
        x[211:300] = float("inf")
        x[330:] = float("nan")
    big = [torch.full((405, n, 64), 3.0, dtype=torch.bfloat16, device="cuda") for n in (4, 2, 2)]
    rp.rp_attend_grad(*bad, st, q_grad=big[0][:400], k_grad=big[1][:400], v_grad=big[2][:400])
    for x, w in zip(big, want):
        assert (x[70:211] == w[70:211]).all() and (x[330:400] == 0).all() and (x[400:] == 3).all()


@pytest.mark.gpu
def test_repeated_streamed_and_captured_gradients_agree_bit_for_bit():
    import torch
    shape = (3000, 8, 2, 128, [0, 500, 501, 3000])
    q, k, v, g = inputs(shape, "bfloat16")
    st = torch.tensor(shape[4], device="cuda")
    do = torch.randn(3000, 8, 128, generator=g).bfloat16().cuda()
    out, lse = rp.rp_attend(q, k, v, st)
    want = rp.rp_attend_grad(do, q, k, v, out, lse, st)
    torch.cuda.synchronize()
    results = [rp.rp_attend_grad(do, q, k, v, out, lse, st, stream=s) for s in [torch.cuda.Stream() for _ in range(4)] for _ in range(3)]
    torch.cuda.synchronize()
    for got in results:
        assert all((a == b).all() for a, b in zip(got, want))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        o, l = rp.rp_attend(q, k, v, st)
        got = rp.rp_attend_grad(do, q, k, v, o, l, st)
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))


def test_refusals_of_the_gradient():
    lib = rp.lib()
    buf = np.zeros(4096, np.float64)
    p = (buf.ctypes.data + 15) // 16 * 16
    cfg = rp.rp_attend_config(2, 1, 64, 2, 1, 0.1)
    ok, bad = C.byref(rp.rp_view(p, 128, 64)), C.byref(rp.rp_view(p, 100, 64))

    def call(at=None, lse=ok, nbytes=1 << 14, space=p):
        views = [ok] * 8
        if at is not None:
            views[at] = bad
        q, k, v, o, g, dq, dk, dv = views
        return lib.rp_attend_grad(C.byref(cfg), 2, q, k, v, o, lse, g, p, 1, dq, dk, dv, space, nbytes, None)
    assert call() == -1 and all(call(at=i) == -1 for i in range(8)) and call(lse=None) == -1 and call(nbytes=16) == -1 and call(space=None) == -1
    assert lib.rp_attend_grad_workspace(None, 1, 1) == 0 and lib.rp_attend_grad_workspace(C.byref(cfg), 100, 1) >= 100 * 2 * 8


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("d,n", [(64, 128), (128, 128), (128, 300), (64, 512)])
def test_keys_at_minus_infinity_before_low_scores(d, n, kind, causal):
    """The first n keys give scores of -inf, those behind them scores around -200: rows that see any of those have an ordinary softmax."""
    import torch
    T, scale = n + 200, 0.5
    q, k, v, _ = inputs((T, 2, 1, d, [0, T]), kind)
    q, k = q.clone(), k.clone()
    q[..., 0], q[..., 1] = 1.0, 20.0
    k[:n, :, 0], k[n:, :, 0], k[:, :, 1] = -math.inf, 0.0, -20.0
    out, lse = rp.rp_attend(q, k, v, torch.tensor([0, T], device="cuda"), causal=causal, scale=scale)
    half = torch.finfo(q.dtype).eps / 2
    rows = slice(n, T) if causal else slice(0, T)
    for h in range(2):
        p, w_lse = weights(q[:, h].double(), k[:, 0].double(), scale, causal)
        want, size = (p @ v[:, 0].double())[rows], (p @ v[:, 0].double().abs())[rows]
        # (scores to 250: 32 bits leave them 2e-5, so 3e-5 of a weight)
        assert ((out[rows, h].double() - want).abs() <= half * (size + want.abs()) + 6e-5 * size + 1e-7).all()
        assert ((lse[rows, h].double() - w_lse[rows]).abs() <= 4e-6 * (1 + w_lse[rows].abs())).all()
    if causal:
        assert (lse[:n] == -math.inf).all()


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("n", [130, 140, 400])
def test_large_scores_of_the_next_sample_change_no_bit(n, causal):
    """Queries behind a sample's end, in the tile of its last ones, whose scores with its later keys are far above those with its first."""
    import torch
    q, k, v, _ = inputs((n + 100, 16, 16, 64, [0, n]), "bfloat16")
    k = k.clone()
    k[128:n] *= 1.7
    want = rp.rp_attend(q[:n], k[:n], v[:n], torch.tensor([0, n], device="cuda"), causal=causal)
    q = q.clone()
    q[n:] = 40 * k[n - 1]
    got = rp.rp_attend(q, k, v, torch.tensor([0, n, n + 100], device="cuda"), causal=causal)
    assert (got[0][:n] == want[0]).all() and (got[1][:n] == want[1]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("under", [10.0, 17.0, 17.5, 20.0])
def test_many_small_weights_beside_a_large_one(under, kind):
    """131072 keys whose scores are far under that of one: what they add up to is not lost."""
    import torch
    T = 131073
    q, k, v = [torch.zeros(T, 1, 64, dtype=getattr(torch, kind), device="cuda") for _ in range(3)]
    q[:, 0, 0], k[1:, 0, 0] = 1.0, -under
    v[1:, 0, :], v[0, 0, 1] = 1.0, 1.0
    out, lse = rp.rp_attend(q, k, v, torch.tensor([0, T], device="cuda"), causal=True, scale=1.0)
    part = (T - 1) * math.exp(-under)
    want = part / (1 + part)
    half = torch.finfo(q.dtype).eps / 2
    # (weights and output rounded once; float16 weights under its normal range off by half a step, 2^-25, of 2^7 times their size; T / 16 additions to a sum of 32 bits that grows by
    # numbers of one sign, which the tensor cores cut off: 2^-23 of it each at most)
    off = 2 * half + 1e-5 + T / 16 * 2.0 ** -23
    assert abs(out[-1, 0, 0].item() - want) <= off * want + (T - 1) * 2.0 ** -32 * (kind == "float16")
    # (where the sum has the large weight from the start, each product is cut off at 2^-23 of it before they are added: T of them)
    assert abs(out[-1, 0, 1].item() - 1) <= off + T * 2.0 ** -23
    # (a sum in 32 bits that takes T / 128 more numbers, each time to 2^-24 of itself)
    assert abs(lse[-1, 0].item() - math.log1p(part)) <= 4e-6 * (1 + math.log1p(part)) + (T / 128 + 1) * 2.0 ** -24


def test_refusals_of_the_status_and_the_limit():
    assert rp.lib().rp_debug_set_wait_limit(-1) == -1
    rp.rp_debug_set_wait_limit()


def run_out_inputs(shape, kind="bfloat16"):
    """(q, k, v, do, start, right results, views of which rows a sample holds)"""
    import torch
    T, hq, hk, d, start = shape
    q, k, v, g = inputs(shape, kind)
    st = torch.tensor(start, device="cuda")
    do = torch.randn(T, hq, d, generator=g).to(q.dtype).cuda()
    out, lse = rp.rp_attend(q, k, v, st)
    grads = rp.rp_attend_grad(do, q, k, v, out, lse, st)
    held = torch.zeros(T, dtype=torch.bool, device="cuda")
    for lo, hi in samples(start, T):
        held[lo:hi] = True
    return q, k, v, do, st, out, lse, grads, held


RUN_OUT = [(2000, 4, 2, 128, [5, 700, 701, 1990]), (3000, 16, 4, 64, [0, 3000]), (900, 8, 8, 64, list(range(0, 900, 9)))]


@pytest.mark.gpu
@pytest.mark.parametrize("shape", RUN_OUT, ids=[str(s[:4]) for s in RUN_OUT])
def test_waits_that_run_out_leave_nan_and_a_status(shape):
    """A limit of 0, with which the kernels give up before their first wait; the calls before and after are as ever."""
    import torch
    q, k, v, do, st, out, lse, grads, held = run_out_inputs(shape)
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    o, l = torch.full_like(out, 3.0), torch.full_like(lse, 3.0)
    try:
        rp.rp_debug_set_wait_limit(0)
        rp.rp_attend(q, k, v, st, out=o, lse=l, status=status)
        assert status.item() == -8
        assert o[held].isnan().all() and l[held].isnan().all() and (o[~held] == 0).all() and (l[~held] == 0).all()
        status.fill_(7)
        got = [torch.full(x.shape, 3.0, dtype=x.dtype, device="cuda") for x in grads]
        rp.rp_attend_grad(do, q, k, v, out, lse, st, q_grad=got[0], k_grad=got[1], v_grad=got[2], status=status)
        assert status.item() == -8
        for x in got[1:]:
            assert x[held].isnan().all() and (x[~held] == 0).all()
    finally:
        rp.rp_debug_set_wait_limit()
    o, l = rp.rp_attend(q, k, v, st, status=status)
    assert status.item() == 0 and (o == out).all() and (l == lse).all()
    status.fill_(7)
    got = rp.rp_attend_grad(do, q, k, v, out, lse, st, status=status)
    assert status.item() == 0 and all((a == b).all() for a, b in zip(got, grads))


@pytest.mark.gpu
def test_status_of_no_tokens():
    import torch
    q, start = torch.zeros(0, 2, 64, dtype=torch.bfloat16, device="cuda"), torch.tensor([0, 0], device="cuda")
    status = torch.full((1,), 7, dtype=torch.int32, device="cuda")
    out, lse = rp.rp_attend(q, q, q, start, status=status)
    assert status.item() == 0
    status.fill_(7)
    rp.rp_attend_grad(q, q, q, q, out, lse, start, status=status)
    assert status.item() == 0
    with pytest.raises(ValueError, match="status"):
        rp.rp_attend(q, q, q, start, status=torch.zeros(2, dtype=torch.int32, device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["bfloat16", "float16"])
@pytest.mark.parametrize("shape", RUN_OUT, ids=[str(s[:4]) for s in RUN_OUT])
def test_waits_that_run_out_leave_no_row_of_the_queries_gradient(shape, kind):
    """Blocks that a CTA took and did not hand over, and those that nobody took."""
    import torch
    q, k, v, do, st, out, lse, grads, held = run_out_inputs(shape, kind)
    status, got = torch.full((1,), 7, dtype=torch.int32, device="cuda"), torch.full_like(grads[0], 3.0)
    try:
        rp.rp_debug_set_wait_limit(0)
        rp.rp_attend_grad(do, q, k, v, out, lse, st, q_grad=got, status=status)
        assert status.item() == -8 and got[held].isnan().all() and (got[~held] == 0).all()
    finally:
        rp.rp_debug_set_wait_limit()


@pytest.mark.gpu
@pytest.mark.parametrize("limit", [1, 2000, 20000])
@pytest.mark.parametrize("shape", RUN_OUT, ids=[str(s[:4]) for s in RUN_OUT])
def test_short_limits_leave_right_rows_or_nan(shape, limit):
    """Waits that run out anywhere or not at all: what is not NaN is right, and NaN comes with a status."""
    import torch
    q, k, v, do, st, out, lse, grads, held = run_out_inputs(shape)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    try:
        rp.rp_debug_set_wait_limit(limit)
        for _ in range(5):
            o, l = torch.full_like(out, 3.0), torch.full_like(lse, 3.0)
            rp.rp_attend(q, k, v, st, out=o, lse=l, status=status)
            pairs = [(o, out), (l, lse)]
            assert status.item() in (0, -8) and all(((a == b) | a.isnan()).all() for a, b in pairs)
            assert status.item() == -8 or not any(a.isnan().any() for a, _ in pairs)
            got = [torch.full(x.shape, 3.0, dtype=x.dtype, device="cuda") for x in grads]
            rp.rp_attend_grad(do, q, k, v, out, lse, st, q_grad=got[0], k_grad=got[1], v_grad=got[2], status=status)
            assert status.item() in (0, -8) and all(((a == b) | a.isnan()).all() for a, b in zip(got, grads))
            assert status.item() == -8 or not any(a.isnan().any() for a in got)
    finally:
        rp.rp_debug_set_wait_limit()
    assert all((a == b).all() for a, b in zip(rp.rp_attend_grad(do, q, k, v, out, lse, st), grads))


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
def test_many_short_blocks_before_a_long_one_are_no_wait(causal):
    """Two of the forward kernel's warp groups share a block of 256 queries; one of them has nothing to do in the blocks of 60000 samples of one token, and does not count
    that as a wait: milliseconds, with a limit of 0.1."""
    import torch
    start = list(range(60000)) + list(range(60000, 100001, 200))
    q, k, v, _ = inputs((100000, 1, 1, 64, start), "bfloat16")
    st, status = torch.tensor(start, device="cuda"), torch.full((1,), 7, dtype=torch.int32, device="cuda")
    want = rp.rp_attend(q, k, v, st, causal=causal)
    try:
        rp.rp_debug_set_wait_limit(100_000)
        got = rp.rp_attend(q, k, v, st, causal=causal, status=status)
        assert status.item() == 0 and all((a == b).all() for a, b in zip(got, want))
    finally:
        rp.rp_debug_set_wait_limit()
    assert (want[0][:60000] == v[:60000]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("causal", [True, False])
@pytest.mark.parametrize("size,T,scale", [(1e-5, 1500, 0.125), (1e-4, 2048, 0.125), (1e-3, 2048, 0.125), (1.0, 700, 0.125), (1e4, 300, 0.02)])
def test_gradients_of_any_size_in_float16(size, T, scale, causal):
    """Gradients whose scores' gradients lie under float16's normal range or beyond its largest number, beside a sample with ordinary ones."""
    import torch
    q, k, v, g = inputs((T + 100, 1, 1, 64, [0, T]), "float16")
    do = torch.randn(T + 100, 1, 64, generator=g).cuda()
    do[:T] *= size
    do = do.half()
    v = v * 4 if size > 1 else v                         # (do v^T to 10^6)
    st = torch.tensor([0, T, T + 100], device="cuda")
    out, lse = rp.rp_attend(q, k, v, st, causal=causal, scale=scale)
    got = rp.rp_attend_grad(do, q, k, v, out, lse, st, causal=causal, scale=scale)
    for lo, hi in ((0, T), (T, T + 100)):
        q64, k64, v64, d64 = [x[lo:hi, 0].double() for x in (q, k, v, do)]
        p, _ = weights(q64, k64, scale, causal)
        o = p @ v64
        ds = p * (d64 @ v64.T - (d64 * o).sum(1, keepdim=True))
        slip = p * (d64 * o).abs().sum(1, keepdim=True)
        # Norms over all elements: weights and gradients of scores are off by 2^-11 of themselves (or by half a step of 2^-24 where they were multiplied with 2^15, with 8 over the
        # largest row's norm or more), the latter by the rounding of o too, both by 2e-5 for 32 bits; a product is off by that times the other factor's largest singular
        # value, and each result is rounded once
        n = hi - lo
        off_p = (2.0 ** -11 + 2e-5) * p.norm() + n * 2.0 ** -40
        off_ds = (2.0 ** -11 + 2e-5) * (ds.norm() + slip.norm()) + n * 2.0 ** -25 * d64.norm(dim=1).max() / 8
        want = (ds @ k64 * scale, ds.T @ q64 * scale, p.T @ d64)
        offs = (off_ds * torch.linalg.matrix_norm(k64, 2) * scale, off_ds * torch.linalg.matrix_norm(q64, 2) * scale, off_p * torch.linalg.matrix_norm(d64, 2))
        for x, w, off in zip(got, want, offs):
            assert torch.isfinite(x).all()
            assert (x[lo:hi, 0].double() - w).norm() <= off + (2.0 ** -11 * w.abs() + 2.0 ** -25).norm()
