"""Norm and rotation of queries and keys in packed rows, and the gradient, against the formulas in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp


def positions(T, start, first=None):
    """(position of every token, whether a sample holds it)"""
    import torch
    pos, held = torch.zeros(T, dtype=torch.float64), torch.zeros(T, dtype=torch.bool)
    for i, (lo, hi) in enumerate(zip(start, start[1:])):
        for t in range(max(lo, 0), min(hi, T)):
            pos[t] = t - lo + (0 if first is None else int(first[i]))
            held[t] = True
    return pos, held


def reference(x, w, pos, held, inv_freq, layout="half", eps=1e-6, mscale=1.0):
    import torch
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w
    r = 2 * len(inv_freq)
    angle = (pos[:, None] * inv_freq)[:, None]
    c, s = torch.cos(angle) * mscale, torch.sin(angle) * mscale
    head = x[..., :r]
    if layout == "half":
        a, b = head[..., :r // 2], head[..., r // 2:]
        head = torch.cat([a * c - b * s, a * s + b * c], -1)
    else:
        a, b = head[..., ::2], head[..., 1::2]
        head = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    return torch.cat([head, x[..., r:]], -1) * held[:, None, None]


# (32 bits: angle 2^-25 of a turn, sine and cosine 2 ulp, mean of squares and root 20 * 2^-24 at most, four products and a sum)
FLOAT = 3e-6


def test_refusals():
    lib = rp.lib()
    buf = np.zeros(4096, np.float64)
    p = buf.ctypes.data

    def r(d=8, rot=8, layout=0, kind=0, wkind=0, eps=1e-6):
        return C.byref(rp.rp_rotary(d, rot, layout, kind, wkind, eps, 1.0))

    def heads(n=1, x=p, y=p, w=None, g=None, dw=None):
        return C.byref(rp.rp_heads(n, x, 8, 8, y, 8, 8, w, g, 8, 8, dw))

    def fwd(cfg=r(), T=2, freq=p, start=p, N=1, first=None, q=heads(), k=None):
        return lib.rp_rotate(cfg, T, freq, start, N, first, q, k, None)

    assert fwd() == -1                                   # host arrays
    for bad in (dict(cfg=None), dict(T=-1), dict(freq=None), dict(start=None), dict(N=0), dict(q=None), dict(q=heads(n=0)), dict(q=heads(n=-1)),
                dict(q=heads(x=None)), dict(q=heads(y=None)), dict(cfg=r(d=0)), dict(cfg=r(rot=7)), dict(cfg=r(rot=10)), dict(cfg=r(layout=2)),
                dict(cfg=r(kind=3)), dict(cfg=r(kind=1, wkind=2)), dict(cfg=r(eps=-1.0)), dict(cfg=r(eps=math.nan)), dict(freq=p + 4), dict(q=heads(x=p + 2))):
        assert fwd(**bad) == -1, bad
    assert fwd(cfg=r(d=1025)) == -5
    assert lib.rp_rotate_workspace(None) == 0 and lib.rp_rotate_workspace(r()) > 0

    def bwd(q=heads(g=p), space=None, nbytes=0):
        return lib.rp_rotate_grad(r(), 2, p, p, 1, None, q, None, space, nbytes, None)

    assert bwd() == -1 and bwd(q=heads()) == -1 and bwd(q=heads(g=p, dw=p)) == -1 and bwd(q=heads(g=p, w=p, dw=p)) == -1


CASES = [
    # tokens, query heads, key heads, head size, rotary size, starts, first positions
    (1, 1, 0, 2, 2, [0, 1], None),
    (1, 32, 8, 128, 128, [0, 1], [1048575]),
    (64, 32, 8, 128, 128, list(range(65)), "far"),
    (37, 5, 1, 64, 64, [0, 0, 10, 11, 37], None),
    (50, 4, 2, 80, 40, [3, 20, 45], None),               # tokens of no sample
    (50, 4, 2, 96, 96, [-5, 20, 70], "far"),
    (41, 3, 3, 192, 64, [0, 41], None),
    (29, 2, 1, 256, 256, [0, 13, 29], "far"),
    (23, 3, 2, 72, 24, [0, 23], None),
    (20, 3, 1, 33, 10, [0, 7, 20], None),                # odd sizes
    (15, 2, 2, 1000, 1000, [0, 15], None),
    (9, 2, 2, 512, 128, [0, 9], "far"),
    (600, 40, 8, 128, 32, [0, 100, 600], None),
    (31, 2, 1, 64, 0, [0, 31], None),                    # norm alone
    (3000, 2, 1, 16, 16, [0, 1000, 1001, 3000], None),
]


def inputs(case, kind, seed=0, offset=0):
    """q, k on the GPU as slices of one wider tensor (`offset` elements off its start), and the rest of a call."""
    import torch
    T, hq, hk, d, r, start, first = case
    g = torch.Generator().manual_seed(T * 31 + d + seed)
    wide = (torch.randn(T, hq + hk + 1, d + offset, generator=g) * torch.exp(torch.randn(T, 1, 1, generator=g))).to(getattr(torch, kind)).cuda()
    q, k = wide[:, :hq, offset:], wide[:, hq:hq + hk, offset:] if hk else None
    if first == "far":
        first = torch.randint(0, 1 << 20, (len(start) - 1,), generator=g).tolist()
    inv = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / max(r, 1))
    return q, k, inv, first, g


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind,w_kind,offset", [("float32", "float32", 0), ("float16", "float32", 0), ("bfloat16", "bfloat16", 0), ("bfloat16", None, 0),
                                                ("float32", None, 0), ("bfloat16", "bfloat16", 3), ("float16", None, 8)])
@pytest.mark.parametrize("case", CASES, ids=[str(c[:5]) for c in CASES])
def test_rows(case, kind, w_kind, offset, layout):
    import torch
    T, hq, hk, d, r, start, first = case
    dtype = getattr(torch, kind)
    q, k, inv, first, g = inputs(case, kind, offset=offset)
    mscale = 1.25
    pos, held = positions(T, start, first)
    weights = [None, None] if w_kind is None else [(1 + 0.3 * torch.randn(d, generator=g)).to(getattr(torch, w_kind)).cuda() for _ in range(2)]
    kw = dict(first_position=None if first is None else torch.tensor(first, device="cuda"), q_weight=weights[0], k_weight=weights[1] if hk else None,
              layout=layout, mscale=mscale)
    freq, st = inv.cuda() if r else None, torch.tensor(start, device="cuda")
    before = [None if x is None else x.clone() for x in (q, k)]
    outs = rp.rp_rotate(q, k, freq, st, **kw)
    wants, leaves = [], []
    for x, w, out in zip((q, k), weights, outs):
        if x is None:
            assert out is None
            continue
        x64 = x.double().cpu().requires_grad_(True)
        w64 = None if w is None else w.double().cpu().requires_grad_(True)
        want = reference(x64, w64, pos, held, inv, layout, 1e-6, mscale)
        wants.append(want)
        leaves.append((x64, w64))
        flat = want.detach()
        tol = torch.finfo(dtype).eps / 2 * flat.abs() + FLOAT * flat.abs().amax(-1, keepdim=True) + 6e-8 * (kind == "float16")
        assert out.dtype == dtype and ((out.cpu().double() - flat).abs() <= tol).all()
    # the gradient, whose input lies apart by token and by head
    grads = []
    for x in (q, k):
        if x is None:
            grads.append(None)
            continue
        big = torch.randn(x.shape[1], T, d + 8, generator=g).to(dtype).cuda()
        grads.append(big[:, :, :d].transpose(0, 1))
    got = rp.rp_rotate_grad(grads[0], grads[1], q, k, freq, st, **kw)
    for i, x in enumerate((q, k)):
        if x is None:
            assert got[i] is None and got[i + 2] is None
            continue
        x64, w64 = leaves[i]
        g64 = grads[i].double().cpu()
        want = torch.autograd.grad((wants[i] * g64).sum(), [v for v in (x64, w64) if v is not None], retain_graph=True)
        size = mscale * 1.5 * g64.abs().amax(-1, keepdim=True)
        if w64 is not None:
            rstd = torch.rsqrt((x64 * x64).mean(-1, keepdim=True) + 1e-6).detach()
            hat = (x64 * rstd).detach()
            size = size * w64.detach().abs().max() * rstd * (1 + hat.abs().amax(-1, keepdim=True))
        tol = torch.finfo(dtype).eps / 2 * want[0].abs() + 2 * FLOAT * size + 6e-8 * (kind == "float16")
        assert got[i].dtype == dtype and ((got[i].cpu().double() - want[0]).abs() <= tol).all()
        assert (got[i][~held.cuda()] == 0).all()
        if w64 is not None:
            total = (mscale * 1.5 * g64.abs().amax(-1, keepdim=True) * hat.abs() * held[:, None, None]).sum((0, 1))
            assert got[i + 2].dtype == torch.float32 and ((got[i + 2].cpu().double() - want[1]).abs() <= FLOAT * total + 1e-30).all()
        else:
            assert got[i + 2] is None
    for x, was in zip((q, k), before):
        assert x is None or (x == was).all()


@pytest.mark.gpu
def test_gradient_against_differences():
    import torch
    start, inv = [0, 2, 5], 100.0 ** (-torch.arange(0, 6, 2, dtype=torch.float64) / 6)
    g = torch.Generator().manual_seed(3)
    x, dy, w = torch.randn(5, 2, 8, generator=g, dtype=torch.float64), torch.randn(5, 2, 8, generator=g, dtype=torch.float64), 1 + 0.1 * torch.randn(8, generator=g, dtype=torch.float64)
    pos, held = positions(5, start)
    dx, _, dw, _ = rp.rp_rotate_grad(dy.float().cuda(), None, x.float().cuda(), None, inv.cuda(), torch.tensor(start, device="cuda"), q_weight=w.float().cuda())

    def value(x, w):
        return (reference(x, w, pos, held, inv) * dy).sum().item()
    h = 1e-6
    for at in np.ndindex(5, 2, 8):
        up, down = x.clone(), x.clone()
        up[at] += h
        down[at] -= h
        assert abs((value(up, w) - value(down, w)) / (2 * h) - dx[at].item()) < 2e-5
    for i in range(8):
        up, down = w.clone(), w.clone()
        up[i] += h
        down[i] -= h
        assert abs((value(x, up) - value(x, down)) / (2 * h) - dw[i].item()) < 2e-5


@pytest.mark.gpu
@pytest.mark.parametrize("d,r", [(128, 128), (33, 10)])
def test_in_place_and_rows_behind(d, r):
    import torch
    case = (40, 4, 2, d, r, [0, 30, 36], None)
    q, k, inv, _, g = inputs(case, "bfloat16")
    q[36:], k[36:] = float("nan"), float("inf")          # padding of the row
    st, w = torch.tensor([0, 30, 36], device="cuda"), torch.ones(d, device="cuda")
    want = rp.rp_rotate(q, k, inv.cuda(), st, q_weight=w)
    assert (want[0][36:] == 0).all() and (want[1][36:] == 0).all()
    big = torch.full((44, 4, d), 7.0, dtype=torch.bfloat16, device="cuda")
    big[:40] = q
    got = rp.rp_rotate(big[:40], k.clone(), inv.cuda(), st, q_weight=w, q_out=big[:40])
    assert got[0].data_ptr() == big.data_ptr() and (big[:40] == want[0]).all() and (big[40:] == 7).all()
    dy = torch.randn(40, 4, d, generator=g).bfloat16().cuda()
    dy[36:] = float("nan")
    grad = rp.rp_rotate_grad(dy, None, q, None, inv.cuda(), st, q_weight=w)
    assert (grad[0][36:] == 0).all() and torch.isfinite(grad[2]).all()
    same = dy.clone()
    again = rp.rp_rotate_grad(same, None, q, None, inv.cuda(), st, q_weight=w, q_grad=same)
    assert (same == grad[0]).all() and (again[2] == grad[2]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("d,heads", [(128, 3), (96, 1), (33, 2)])
def test_norm_without_eps(d, heads):
    """eps = 0: what a warp has no head or no token for is not a row of zeros to be divided by its norm."""
    import torch
    q, _, inv, _, g = inputs((40, heads, 0, d, 16, [2, 30, 36], None), "float32")
    st, w = torch.tensor([2, 30, 36], device="cuda"), torch.rand(d, generator=g).cuda() + 0.5
    dy = torch.randn(40, heads, d, generator=g).cuda()
    out = rp.rp_rotate(q, None, inv.cuda(), st, q_weight=w, eps=0.0)[0]
    grad = rp.rp_rotate_grad(dy, None, q, None, inv.cuda(), st, q_weight=w, eps=0.0)
    pos, held = positions(40, [2, 30, 36])
    x, w64 = q.double().cpu().requires_grad_(), w.double().cpu().requires_grad_()
    y = reference(x, w64, pos, held, inv, eps=0.0)
    y.backward(dy.double().cpu())
    rstd = torch.rsqrt((x * x).mean(-1, keepdim=True)).detach()
    hat, top = (x * rstd).detach(), 1.5 * dy.double().cpu().abs().amax(-1, keepdim=True)
    half = torch.finfo(torch.float32).eps / 2
    # (bounds as in test_rows)
    assert ((out.double().cpu() - y).abs() <= (half * y.abs() + FLOAT * y.abs().amax(-1, keepdim=True)).detach()).all()
    size = top * w64.detach().max() * rstd * (1 + hat.abs().amax(-1, keepdim=True))
    assert ((grad[0].double().cpu() - x.grad).abs() <= half * x.grad.abs() + 2 * FLOAT * size).all()
    total = (top * hat.abs() * held[:, None, None]).sum((0, 1))
    assert ((grad[2].double().cpu() - w64.grad).abs() <= FLOAT * total + 1e-30).all()


@pytest.mark.gpu
def test_repeated_streamed_and_captured_calls_agree_bit_for_bit():
    import torch
    case = (3000, 8, 2, 128, 64, [0, 1000, 3000], None)
    q, k, inv, _, g = inputs(case, "bfloat16")
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    freq, st, w = inv.cuda(), torch.tensor([0, 1000, 3000], device="cuda"), torch.ones(128, device="cuda")
    kw = dict(q_weight=w, k_weight=w, layout="interleaved")

    def both(**more):
        return (*rp.rp_rotate(q, k, freq, st, **kw, **more), *rp.rp_rotate_grad(dq, dk, q, k, freq, st, **kw, **more))
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
def test_two_outputs_in_one_place_are_refused():
    import torch
    q, w, dw = torch.zeros(2, 1, 8, device="cuda"), torch.ones(8, device="cuda"), torch.zeros(8, device="cuda")
    y = [torch.zeros_like(q) for _ in range(2)]
    freq, st, space = torch.ones(4, dtype=torch.float64, device="cuda"), torch.tensor([0, 2], device="cuda"), torch.zeros(1 << 20, device="cuda")
    with pytest.raises(rp.RpError, match="ARG"):
        rp.rp_rotate(q, q, freq, st, q_out=y[0], k_out=y[0])
    cfg, stream = C.byref(rp.rp_rotary(8, 8, 0, 0, 0, 1e-6, 1.0)), torch.cuda.current_stream().cuda_stream

    def call(dk):
        sides = [C.byref(rp.rp_heads(1, q.data_ptr(), 8, 8, out.data_ptr(), 8, 8, w.data_ptr(), q.data_ptr(), 8, 8, at.data_ptr())) for out, at in zip(y, (dw, dk))]
        return rp.lib().rp_rotate_grad(cfg, 2, freq.data_ptr(), st.data_ptr(), 1, None, *sides, space.data_ptr(), 4 << 20, stream)
    assert call(dw) == -1 and call(torch.zeros_like(dw)) == 0


@pytest.mark.gpu
def test_no_tokens():
    import torch
    q = torch.zeros(0, 4, 64, device="cuda")
    w = torch.ones(64, device="cuda")
    inv, st = torch.ones(32, dtype=torch.float64, device="cuda"), torch.tensor([0, 0], device="cuda")
    assert rp.rp_rotate(q, None, inv, st)[0].shape == (0, 4, 64)
    assert (rp.rp_rotate_grad(q, None, q, None, inv, st, q_weight=w)[2] == 0).all()


@pytest.mark.gpu
@pytest.mark.parametrize("d", [128, 34])
def test_heads_and_tokens_that_repeat(d):
    import torch
    g = torch.Generator().manual_seed(d)
    inv, st, w = 100.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d), torch.tensor([0, 4, 30], device="cuda"), torch.rand(d, generator=g).cuda()
    for base in (torch.randn(30, 1, d, generator=g), torch.randn(1, 5, d, generator=g)):
        q = base.bfloat16().cuda().expand(30, 5, d)
        dy = torch.randn(30, 1, d, generator=g).bfloat16().cuda().expand(30, 5, d)
        for a, b in zip(rp.rp_rotate(q, q, inv, st, q_weight=w), rp.rp_rotate(q.contiguous(), q.contiguous(), inv, st, q_weight=w)):
            assert (a == b).all()
        one, two = rp.rp_rotate_grad(dy, None, q, None, inv, st, q_weight=w), rp.rp_rotate_grad(dy.contiguous(), None, q.contiguous(), None, inv, st, q_weight=w)
        assert (one[0] == two[0]).all() and (one[2] == two[2]).all()


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("d,r", [(128, 64), (64, 16), (64, 24), (256, 64), (80, 40), (32, 0), (96, 90)])
def test_elements_that_are_not_turned_are_handed_on_alone(d, r, kind, layout):
    """What stands behind rotary_dim, infinities and NaN too, comes out as it is and reaches no other element."""
    import torch
    T = 50
    q, _, inv, _, g = inputs((T, 3, 0, d, r, [0, 20, 45], None), kind)
    q = q.contiguous()
    start, inv = torch.tensor([0, 20, 45], device="cuda"), inv.cuda() if r else None
    clean, dirty = rp.rp_rotate(q, None, inv, start, layout=layout)[0], q.clone()
    places = sorted({r, r + 1, d - 1})
    for i, e in enumerate(places):
        dirty[::2, :2, e] = (math.inf, math.nan, -math.inf)[i % 3]
    y = rp.rp_rotate(dirty, None, inv, start, layout=layout)[0]
    dx = rp.rp_rotate_grad(dirty, None, q, None, inv, start, layout=layout)[0]
    back = rp.rp_rotate_grad(q, None, q, None, inv, start, layout=layout)[0]
    rest = [e for e in range(d) if e not in places]
    assert (y[..., rest] == clean[..., rest]).all() and (dx[..., rest] == back[..., rest]).all()
    for got in (y, dx):
        assert torch.equal(got[:45, :, places].nan_to_num(7.0), dirty[:45, :, places].nan_to_num(7.0)) and (got[45:] == 0).all()


@pytest.mark.gpu
def test_weights_of_no_heads_have_a_gradient_of_zero():
    import torch
    q, k, inv, _, g = inputs((20, 0, 2, 64, 64, [0, 20], None), "float32")
    start, w = torch.tensor([0, 20], device="cuda"), torch.ones(64, device="cuda")
    junk = [torch.full((64,), math.nan, device="cuda") for _ in range(64)]
    torch.cuda.synchronize()
    del junk                                             # (what the allocator hands out next)
    dq, dk, dwq, dwk = rp.rp_rotate_grad(q, k, q, k, inv.cuda(), start, q_weight=w, k_weight=w)
    assert dq.shape == (20, 0, 64) and (dwq == 0).all() and torch.isfinite(dwk).all() and (dwk != 0).any()
