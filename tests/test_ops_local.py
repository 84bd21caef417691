"""The operators of a layer with local attention as they are used together: rows of text and pictures in training, the same tokens one by one in decoding."""
import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp

LENGTHS = [300, 1, 129, 17, 2600, 64]
HQ, HK, D, WINDOW, SINKS = 8, 2, 64, 200, 4


def places(n, seed):
    """Positions [3, n] of a sample: text, then a picture of some rows, then text."""
    import torch
    text = min(n, 7 + seed)
    rows = torch.arange(max(n - text, 0))
    picture = torch.stack([torch.full_like(rows, text), text + rows // 12, text + rows % 12])
    return torch.cat([torch.arange(text).expand(3, text), picture], 1)


def window_row():
    import torch
    g = torch.Generator().manual_seed(21)
    T = sum(LENGTHS)
    x = {name: torch.randn(T, heads, D, generator=g).bfloat16().cuda() for name, heads in (("q", HQ), ("k", HK), ("v", HK), ("grad", HQ))}
    x["start"] = torch.tensor(np.concatenate([[0], np.cumsum(LENGTHS)]), device="cuda")
    x["place"] = torch.cat([places(n, i) for i, n in enumerate(LENGTHS)], 1).cuda()
    x["weight"] = (torch.rand(D, generator=g) + 0.5).cuda()
    x["inv"] = 10000.0 ** (-torch.arange(0, D, 2, dtype=torch.float64, device="cuda") / D)
    x["axis"] = torch.tensor([0] * 8 + [1, 2] * 12, dtype=torch.int32, device="cuda")
    return x


def layer(q, k, v, grad, place, start, x, **more):
    """A layer's attention there and back: (outputs of each token), (gradients of the weights)."""
    kw = dict(q_weight=x["weight"], k_weight=x["weight"], **more)
    local = dict(window=WINDOW, sinks=SINKS, **more)
    qr, kr = rp.rp_rotate_axes(q, k, x["inv"], x["axis"], place, **kw)
    out, lse = rp.rp_attend_window(qr, kr, v, start, **local)
    dqr, dkr, dv = rp.rp_attend_window_grad(grad, qr, kr, v, out, lse, start, **local)
    dq, dk, dqw, dkw = rp.rp_rotate_axes_grad(dqr, dkr, q, k, x["inv"], x["axis"], place, **kw)
    return (qr, kr, out, lse, dq, dk, dv), (dqw, dkw)


@pytest.mark.gpu
def test_a_row_gives_each_sample_what_it_gets_alone():
    import torch
    x = window_row()
    row, weights = layer(x["q"], x["k"], x["v"], x["grad"], x["place"], x["start"], x)
    total = [torch.zeros(D, dtype=torch.float64, device="cuda") for _ in weights]
    for lo, hi in zip(x["start"].tolist(), x["start"].tolist()[1:]):
        alone, dw = layer(*(x[n][lo:hi] for n in ("q", "k", "v", "grad")), x["place"][:, lo:hi], torch.tensor([0, hi - lo], device="cuda"), x)
        for a, b in zip(row, alone):
            assert (a[lo:hi] == b).all()
        for t, w in zip(total, dw):
            t += w.double()
    for a, t in zip(weights, total):
        # sums of the same numbers in 32 bits, in another order: at most 2^12 of them a column
        assert ((a.double() - t).abs() <= 2.0 ** -12 * t.abs().max()).all()


@pytest.mark.gpu
def test_decoding_gives_a_sample_s_last_token_what_the_row_gave_it():
    """A cache with room, filled with the row's keys; the token's own query and key rotated alone."""
    import torch
    x = window_row()
    (qr, kr, out, lse, *_), _ = layer(x["q"], x["k"], x["v"], x["grad"], x["place"], x["start"], x)
    N, last = len(LENGTHS), x["start"][1:] - 1
    room = [n + 5 + i for i, n in enumerate(LENGTHS)]
    start = torch.tensor(np.concatenate([[0], np.cumsum(room)]), device="cuda")
    k, v = (torch.full((sum(room), HK, D), float("nan"), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q1, k1 = rp.rp_rotate_axes(x["q"][last], x["k"][last], x["inv"], x["axis"], x["place"][:, last], q_weight=x["weight"], k_weight=x["weight"])
    assert (q1 == qr[last]).all() and (k1 == kr[last]).all()
    for i, n in enumerate(LENGTHS):
        at, lo = int(start[i]), int(x["start"][i])
        k[at:at + n - 1], v[at:at + n] = kr[lo:lo + n - 1], x["v"][lo:lo + n]
    k[start[:-1] + torch.tensor(LENGTHS, device="cuda") - 1] = k1
    got, glse = rp.rp_attend_step(q1, k, v, start, length=torch.tensor(LENGTHS, device="cuda"), window=WINDOW, sinks=SINKS)
    for i, n in enumerate(LENGTHS):
        lo, j = int(x["start"][i]), torch.tensor([j for j in range(n) if j < SINKS or n - 1 - j < WINDOW], device="cuda")
        for h in range(HQ):
            p = torch.softmax(kr[lo + j, h // (HQ // HK)].double() @ q1[i, h].double() * D ** -0.5, 0)
            size = p @ x["v"][lo + j, h // (HQ // HK)].double().abs()
            # the row's weights rounded once, both outputs; 32 bits beside that
            tol = 2.0 ** -8 * (size + 2 * out[last[i], h].double().abs()) * (1 + 2.0 ** -8) + 2.0 ** -14 * size
            assert ((got[i, h].double() - out[last[i], h].double()).abs() <= tol).all()
        assert ((glse[i] - lse[last[i]]).abs() <= 8e-6 * (1 + lse[last[i]].abs())).all()


@pytest.mark.gpu
def test_calls_at_once_and_captured_ones():
    """Two layers on two streams at a time, one of them captured and replayed, share inputs and nothing else."""
    import torch
    x = window_row()
    args = (x["q"], x["k"], x["v"], x["grad"], x["place"], x["start"], x)
    want = layer(*args)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        captured = layer(*args)
    streams = [torch.cuda.Stream() for _ in range(2)]
    got = []
    for _ in range(4):
        with torch.cuda.stream(streams[0]):
            graph.replay()
        got.append(layer(*args, stream=streams[1]))
    torch.cuda.synchronize()
    for run in (captured, *got):
        for a, b in zip((*run[0], *run[1]), (*want[0], *want[1])):
            assert (a == b).all()


@pytest.mark.gpu
def test_under_autograd():
    """The calls as a torch.autograd.Function: gradients of leaves, of a key head shared by four query heads, against autograd in 64 bits."""
    import torch

    class Local(torch.autograd.Function):
        @staticmethod
        def forward(ctx, q, k, v, start, window, sinks):
            out, lse = rp.rp_attend_window(q, k, v, start, window=window, sinks=sinks)
            ctx.save_for_backward(q, k, v, out, lse, start)
            ctx.local = dict(window=window, sinks=sinks)
            return out

        @staticmethod
        def backward(ctx, grad):
            q, k, v, out, lse, start = ctx.saved_tensors
            return (*rp.rp_attend_window_grad(grad.contiguous(), q, k, v, out, lse, start, **ctx.local), None, None, None)

    g = torch.Generator().manual_seed(4)
    T, d = 40, 16
    leaves = [torch.randn(T, n, d, generator=g).half().cuda().requires_grad_() for n in (4, 1, 1)]
    start, weight = torch.tensor([0, 13, T], device="cuda"), torch.randn(T, 4, d, generator=g).half().cuda()
    (Local.apply(*leaves, start, 5, 2) * weight).sum().backward()
    ref = [x.detach().double().requires_grad_() for x in leaves]
    loss, sizes = 0.0, [torch.zeros_like(x) for x in ref]
    for lo, hi in ((0, 13), (13, T)):
        i = torch.arange(hi - lo, device="cuda")
        hidden = (i[:, None] < i) | ((i[:, None] - i >= 5) & (i >= 2))
        for h in range(4):
            q, k, v, do = ref[0][lo:hi, h], ref[1][lo:hi, 0], ref[2][lo:hi, 0], weight[lo:hi, h].double()
            p = torch.softmax((q @ k.T * d ** -0.5).masked_fill(hidden, -float("inf")), 1)
            loss = loss + (p @ v * do).sum()
            with torch.no_grad():
                # sums of magnitudes that the roundings of weights, outputs and scores' gradients go by
                o = p @ v
                ds = p * ((do @ v.T - (do * o).sum(1, keepdim=True)).abs() + (do * o).abs().sum(1, keepdim=True))
                sizes[0][lo:hi, h] += ds @ k.abs() * d ** -0.5
                sizes[1][lo:hi, 0] += ds.T @ q.abs() * d ** -0.5
                sizes[2][lo:hi, 0] += p.T @ do.abs()
    loss.backward()
    for x, r, s in zip(leaves, ref, sizes):
        # (each rounded once to 2^-11, and the result; sums in 32 bits; float16 below 2^-14 is off by 2^-25, in up to 4 * T terms of |x| <= 5)
        assert ((x.grad.double() - r.grad).abs() <= 2.0 ** -11 * (s + r.grad.abs()) + 2e-5 * s + 2.0 ** -25 * 5 * 4 * T + 1e-7).all()
