"""Norm and rotation of queries and keys by positions on several axes, and the gradient, against the formulas in 64 bits."""
import ctypes as C
import math

import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp


def reference(x, w, place, inv_freq, layout="half", eps=1e-6, mscale=1.0):
    """`place` [T, rotary / 2]: where each pair of a token is."""
    import torch
    if w is not None:
        x = x * torch.rsqrt((x * x).mean(-1, keepdim=True) + eps) * w
    r = 2 * len(inv_freq)
    angle = (place.double() * inv_freq)[:, None]
    c, s = torch.cos(angle) * mscale, torch.sin(angle) * mscale
    head = x[..., :r]
    if layout == "half":
        a, b = head[..., :r // 2], head[..., r // 2:]
        head = torch.cat([a * c - b * s, a * s + b * c], -1)
    else:
        a, b = head[..., ::2], head[..., 1::2]
        head = torch.stack([a * c - b * s, a * s + b * c], -1).flatten(-2)
    return torch.cat([head, x[..., r:]], -1)


def places(position, axis):
    import torch
    n = position.shape[0]
    table = torch.cat([position, torch.zeros_like(position[:1])])           # (what is on no axis is at 0)
    return table[torch.tensor([a if 0 <= a < n else n for a in axis])].t()


# (32 bits: angle 2^-25 of a turn, sine and cosine 2 ulp, mean of squares and root 20 * 2^-24 at most, four products and a sum)
FLOAT = 3e-6


def test_refusals():
    lib = rp.lib()
    buf = np.zeros(4096, np.float64)
    p = buf.ctypes.data

    def r(d=8, rot=8, layout=0, kind=0, wkind=0, eps=1e-6):
        return C.byref(rp.rp_rotary(d, rot, layout, kind, wkind, eps, 1.0))

    def axes(n=2, axis=p, position=p):
        return C.byref(rp.rp_axes(n, axis, position, 2, 1))

    def heads(n=1, x=p, y=p, w=None, g=None, dw=None):
        return C.byref(rp.rp_heads(n, x, 8, 8, y, 8, 8, w, g, 8, 8, dw))

    def fwd(cfg=r(), T=2, freq=p, ax=axes(), q=heads()):
        return lib.rp_rotate_axes(cfg, T, freq, ax, q, None, None)
    assert fwd() == -1                                   # host arrays
    for bad in (dict(cfg=None), dict(T=-1), dict(freq=None), dict(ax=None), dict(ax=axes(n=0)), dict(ax=axes(n=-1)), dict(ax=axes(axis=None)),
                dict(ax=axes(position=None)), dict(ax=axes(axis=p + 2)), dict(ax=axes(position=p + 4)), dict(q=None), dict(q=heads(n=0)), dict(q=heads(x=None)),
                dict(cfg=r(rot=0)), dict(cfg=r(rot=7)), dict(cfg=r(rot=10)), dict(cfg=r(layout=2)), dict(cfg=r(eps=-1.0))):
        assert fwd(**bad) == -1, bad
    assert fwd(ax=axes(n=9)) == -5 and fwd(cfg=r(d=1025)) == -5

    def bwd(q=heads(g=p), ax=axes(), space=None, nbytes=0):
        return lib.rp_rotate_axes_grad(r(), 2, p, ax, q, None, space, nbytes, None)
    assert bwd() == -1 and bwd(q=heads()) == -1 and bwd(ax=None) == -1 and bwd(q=heads(g=p, w=p, dw=p)) == -1 and bwd(ax=axes(n=9)) == -5


CASES = [
    # tokens, query heads, key heads, head size, rotary size, axes
    (1, 1, 0, 2, 2, 1), (1, 32, 8, 128, 128, 3), (64, 32, 8, 128, 128, 3), (37, 5, 1, 64, 64, 2), (50, 4, 2, 80, 40, 4), (41, 3, 3, 192, 64, 3), (29, 2, 1, 256, 256, 8),
    (23, 3, 2, 72, 24, 3), (20, 3, 1, 33, 10, 5), (15, 2, 2, 1000, 1000, 2), (9, 2, 2, 512, 128, 7), (600, 40, 8, 128, 32, 1), (3000, 2, 1, 16, 16, 2), (2500, 40, 8, 64, 64, 3),
]


def inputs(case, kind, offset=0):
    """q, k on the GPU as slices of one wider tensor (`offset` elements off its start), positions of any sign and size, pairs on all axes and on none."""
    import torch
    T, hq, hk, d, r, n = case
    g = torch.Generator().manual_seed(T * 31 + d)
    wide = (torch.randn(T, hq + hk + 1, d + offset, generator=g) * torch.exp(torch.randn(T, 1, 1, generator=g))).to(getattr(torch, kind)).cuda()
    q, k = wide[:, :hq, offset:], wide[:, hq:hq + hk, offset:] if hk else None
    position = torch.randint(-1000, 1 << 20, (n, T), generator=g)
    axis = torch.randint(0, n, (r // 2,), generator=g).tolist()
    axis[-1] = n if T % 2 else axis[-1]
    axis[0] = -1 if r > 10 else axis[0]
    inv = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64) / max(r, 1))
    return q, k, inv, axis, position, g


@pytest.mark.gpu
@pytest.mark.parametrize("layout", ["half", "interleaved"])
@pytest.mark.parametrize("kind,w_kind,offset", [("float32", "float32", 0), ("float16", "float32", 0), ("bfloat16", "bfloat16", 0), ("float32", None, 0),
                                                ("bfloat16", "bfloat16", 3), ("float16", None, 8)])
@pytest.mark.parametrize("case", CASES, ids=[str(c) for c in CASES])
def test_rows(case, kind, w_kind, offset, layout):
    import torch
    T, hq, hk, d, r, n = case
    dtype = getattr(torch, kind)
    q, k, inv, axis, position, g = inputs(case, kind, offset)
    mscale = 1.25
    place = places(position, axis)
    weights = [None, None] if w_kind is None else [(1 + 0.3 * torch.randn(d, generator=g)).to(getattr(torch, w_kind)).cuda() for _ in range(2)]
    kw = dict(q_weight=weights[0], k_weight=weights[1] if hk else None, layout=layout, mscale=mscale)
    # (a table of [T, axes] as well as one of [axes, T])
    table = (inv.cuda(), torch.tensor(axis, dtype=torch.int32, device="cuda"), position.t().contiguous().cuda().t() if offset else position.cuda())
    before = [None if x is None else x.clone() for x in (q, k)]
    outs = rp.rp_rotate_axes(q, k, *table, **kw)
    wants, leaves = [], []
    for x, w, out in zip((q, k), weights, outs):
        if x is None:
            assert out is None
            continue
        x64 = x.double().cpu().requires_grad_(True)
        w64 = None if w is None else w.double().cpu().requires_grad_(True)
        want = reference(x64, w64, place, inv, layout, 1e-6, mscale)
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
    got = rp.rp_rotate_axes_grad(grads[0], grads[1], q, k, *table, **kw)
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
        if w64 is not None:
            total = (mscale * 1.5 * g64.abs().amax(-1, keepdim=True) * hat.abs()).sum((0, 1))
            assert got[i + 2].dtype == torch.float32 and ((got[i + 2].cpu().double() - want[1]).abs() <= FLOAT * total + 1e-30).all()
        else:
            assert got[i + 2] is None
    for x, was in zip((q, k), before):
        assert x is None or (x == was).all()


@pytest.mark.gpu
@pytest.mark.parametrize("T,d,r,layout", [(700, 128, 128, "half"), (700, 128, 64, "interleaved"), (9000, 64, 64, "half"), (50, 33, 10, "half")])
def test_axes_that_go_on_together_are_positions_in_the_sample(T, d, r, layout):
    """Bit for bit what rp_rotate gives, for rows of any number of tokens to a warp."""
    import torch
    g = torch.Generator().manual_seed(T)
    q, k, dq, dk = (torch.randn(T, n, d, generator=g).bfloat16().cuda() for n in (6, 2, 6, 2))
    w = torch.rand(d, generator=g).cuda() + 0.5
    start = torch.tensor([0, 17, T // 2, T], device="cuda")
    inv = 10000.0 ** (-torch.arange(0, r, 2, dtype=torch.float64, device="cuda") / r)
    place = torch.arange(T, device="cuda") - start[torch.searchsorted(start, torch.arange(T, device="cuda"), right=True) - 1]
    axis = torch.arange(r // 2, dtype=torch.int32, device="cuda") % 3
    kw = dict(q_weight=w, k_weight=w, layout=layout)
    table = (inv, axis, place.expand(3, T))
    for a, b in zip(rp.rp_rotate_axes(q, k, *table, **kw), rp.rp_rotate(q, k, inv, start, **kw)):
        assert (a == b).all()
    for a, b in zip(rp.rp_rotate_axes_grad(dq, dk, q, k, *table, **kw), rp.rp_rotate_grad(dq, dk, q, k, inv, start, **kw)):
        assert (a == b).all()


@pytest.mark.gpu
def test_gradient_against_differences():
    import torch
    inv, axis = 100.0 ** (-torch.arange(0, 6, 2, dtype=torch.float64) / 6), [1, 0, 1]
    g = torch.Generator().manual_seed(3)
    x, dy, w = torch.randn(5, 2, 8, generator=g, dtype=torch.float64), torch.randn(5, 2, 8, generator=g, dtype=torch.float64), 1 + 0.1 * torch.randn(8, generator=g, dtype=torch.float64)
    position = torch.randint(0, 50, (2, 5), generator=g)
    place = places(position, axis)
    dx, _, dw, _ = rp.rp_rotate_axes_grad(dy.float().cuda(), None, x.float().cuda(), None, inv.cuda(), torch.tensor(axis, dtype=torch.int32, device="cuda"), position.cuda(),
                                          q_weight=w.float().cuda())

    def value(x, w):
        return (reference(x, w, place, inv) * dy).sum().item()
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
def test_in_place_streamed_and_captured_calls_agree_bit_for_bit():
    """Positions that change between replays are read anew."""
    import torch
    q, k, inv, axis, position, g = inputs((3000, 8, 2, 128, 64, 3), "bfloat16")
    dq, dk = torch.randn_like(q), torch.randn_like(k)
    table, w = [inv.cuda(), torch.tensor(axis, dtype=torch.int32, device="cuda"), position.cuda()], torch.ones(128, device="cuda")
    kw = dict(q_weight=w, k_weight=w, layout="interleaved")

    def both(**more):
        return (*rp.rp_rotate_axes(q, k, *table, **kw, **more), *rp.rp_rotate_axes_grad(dq, dk, q, k, *table, **kw, **more))
    want = both()
    torch.cuda.synchronize()
    results = [both(stream=s) for s in [torch.cuda.Stream() for _ in range(4)] for _ in range(3)]
    torch.cuda.synchronize()
    for got in results:
        assert all((a == b).all() for a, b in zip(got, want))
    same = q.clone()
    assert (rp.rp_rotate_axes(same, None, *table, q_weight=w, layout="interleaved", q_out=same)[0] == want[0]).all() and (same == want[0]).all()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        got = both()
    for _ in range(3):
        graph.replay()
    torch.cuda.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))
    table[2] += 5
    graph.replay()
    want = both()
    torch.cuda.synchronize()
    assert all((a == b).all() for a, b in zip(got, want))


@pytest.mark.gpu
def test_rows_that_lie_beyond_32_bits():
    """Elements 2^31 and more from a tensor's first one."""
    import torch
    T, h, d, step = 1200, 3, 64, 1 << 21
    g = torch.Generator().manual_seed(8)
    x, dy = (torch.randn(T, h, d, generator=g).bfloat16().cuda() for _ in range(2))
    w = torch.rand(d, generator=g).bfloat16().cuda()
    inv, axis = 1000.0 ** -torch.arange(0, 1, 2 / d, dtype=torch.float64).cuda(), torch.arange(d // 2, dtype=torch.int32).cuda() % 2
    position = torch.randint(0, 5000, (2, T), generator=g).cuda()

    def apart(x=None):
        y = torch.empty(T, step, dtype=torch.bfloat16, device="cuda")[:, :h * d].view(T, h, d)
        return y if x is None else y.copy_(x)
    want, _ = rp.rp_rotate_axes(x, None, inv, axis, position, q_weight=w)
    dx, _, dw, _ = rp.rp_rotate_axes_grad(dy, None, x, None, inv, axis, position, q_weight=w)
    far = apart(x)
    got, _ = rp.rp_rotate_axes(far, None, inv, axis, position, q_weight=w, q_out=apart())
    assert (got == want).all()
    got, _, dw2, _ = rp.rp_rotate_axes_grad(apart(dy), None, far, None, inv, axis, position, q_weight=w, q_grad=apart())
    assert (got == dx).all() and (dw2 == dw).all()


@pytest.mark.gpu
def test_no_tokens_and_arguments_in_python():
    import torch
    q, w = torch.zeros(0, 4, 64, device="cuda"), torch.ones(64, device="cuda")
    inv, axis = torch.ones(32, dtype=torch.float64, device="cuda"), torch.zeros(32, dtype=torch.int32, device="cuda")
    none = torch.zeros(3, 0, dtype=torch.int64, device="cuda")
    assert rp.rp_rotate_axes(q, None, inv, axis, none)[0].shape == (0, 4, 64)
    assert (rp.rp_rotate_axes_grad(q, None, q, None, inv, axis, none, q_weight=w)[2] == 0).all()
    q, place = torch.zeros(5, 4, 64, device="cuda"), torch.zeros(3, 5, dtype=torch.int64, device="cuda")
    for args in ((None, axis, place), (inv, axis.long(), place), (inv, axis[:31], place), (inv, None, place), (inv, axis, place[:, :4]), (inv, axis, place.int()), (inv, axis, place[0])):
        with pytest.raises((ValueError, rp.RpError)):
            rp.rp_rotate_axes(q, None, *args)
    with pytest.raises(rp.RpError, match="RANGE"):
        rp.rp_rotate_axes(q, None, inv, axis, torch.zeros(9, 5, dtype=torch.int64, device="cuda"))
    with pytest.warns(UserWarning, match="rp_rotate_axes_grad"):
        rp.rp_rotate_axes(q.clone().requires_grad_(True), None, inv, axis, place)


@pytest.mark.gpu
@pytest.mark.parametrize("d,r", [(128, 64), (96, 90)])
def test_elements_that_are_not_turned_are_handed_on_alone(d, r):
    """What stands behind rotary_dim, infinities and NaN too, comes out as it is and reaches no other element; far positions are turned exactly."""
    import torch
    q, _, inv, axis, position, g = inputs((50, 3, 0, d, r, 3), "float32")
    dirty = q.clone()
    dirty[::2, :2, d - 1], dirty[::2, :2, r] = math.inf, math.nan
    table = (inv.cuda(), torch.tensor(axis, dtype=torch.int32, device="cuda"), position.cuda())
    clean, y = rp.rp_rotate_axes(q, None, *table)[0], rp.rp_rotate_axes(dirty, None, *table)[0]
    rest = [e for e in range(d) if e not in (r, d - 1)]
    assert (y[..., rest] == clean[..., rest]).all() and torch.equal(y[..., [r, d - 1]].nan_to_num(7.0), dirty[..., [r, d - 1]].nan_to_num(7.0))
