"""The operators as a trainer runs them: routers record their choices, the record is planned, and the rows of the plan run attention and routers."""
import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp


@pytest.mark.gpu
def test_a_window_from_its_routers_to_its_rows():
    import torch
    g = torch.Generator(device="cuda").manual_seed(5)
    lengths = np.array([300, 17, 129, 1, 640, 256, 90, 33, 410, 128, 77, 5], np.int32)
    T, N, L, E, k, hq, hk, d = int(lengths.sum()), len(lengths), 2, 32, 4, 4, 2, 64
    start = torch.tensor(np.concatenate([[0], np.cumsum(lengths)]), device="cuda")
    cap, D, P = 1024, 2, 4

    # a rollout: the routers of both layers choose, and leave their choices in the record
    logits = (torch.randn(L, T, E, generator=g, device="cuda") + torch.randn(L, 1, E, generator=g, device="cuda")).bfloat16()
    record = torch.empty(T, L, k, dtype=torch.uint8, device="cuda")
    gates = []
    for l in range(L):
        _, gate, counts, _ = rp.rp_route(logits[l], k, start, routes=record[:, l], loss_coef=0.01)
        gates.append(gate)
        assert (rp.rp_count_routes(record, start, E)[:, l] == counts).all()

    # the plan of the window, from the record
    ctx = rp.rp_window_load_routes(lengths, record, E, token_cap=cap, dp_width=D, ep_width=P, pop_size=8, seed=1)
    rp.rp_place_experts(ctx)
    rows, _ = rp.rp_pack_rows(ctx)
    rp.rp_anneal(ctx, n_levels=3, steps_per_level=30, t0=1e-2, t_ratio=0.5, p_reloc=0.25, p_guide=0.8)
    cell = rp.rp_best(ctx)[0]
    assert len(set(cell.tolist())) == rows * D
    rp.rp_destroy(ctx)

    # its rows: a packed row gives each sample what it gets alone, bit for bit
    q, kk, v, grad = (torch.randn(T, h, d, generator=g, device="cuda").bfloat16() for h in (hq, hk, hk, hq))
    w = torch.rand(d, generator=g, device="cuda") + 0.5
    inv = 10000.0 ** (-torch.arange(0, d, 2, dtype=torch.float64, device="cuda") / d)

    def layer(q, kk, v, grad, st):
        qr, kr = rp.rp_rotate(q, kk, inv, st, q_weight=w, k_weight=w)
        out, lse = rp.rp_attend(qr, kr, v, st)
        dqr, dkr, dv = rp.rp_attend_grad(grad, qr, kr, v, out, lse, st)
        dq, dk, dqw, dkw = rp.rp_rotate_grad(dqr, dkr, q, kk, inv, st, q_weight=w, k_weight=w)
        return (out, lse, dq, dk, dv), (dqw, dkw)

    seen = torch.zeros(N, E, dtype=torch.int64, device="cuda")
    for c in range(rows * D):
        mine = np.flatnonzero(cell == c)
        tokens = torch.cat([torch.arange(start[i], start[i + 1], device="cuda") for i in mine])
        st = torch.tensor(np.concatenate([[0], np.cumsum(lengths[mine])]), device="cuda")
        assert len(tokens) <= cap
        row, weights = layer(q[tokens], kk[tokens], v[tokens], grad[tokens], st)
        total = [torch.zeros(d, dtype=torch.float64, device="cuda") for _ in weights]
        for x, i in enumerate(mine):
            lo, hi = int(start[i]), int(start[i + 1])
            alone, dw = layer(q[lo:hi], kk[lo:hi], v[lo:hi], grad[lo:hi], torch.tensor([0, hi - lo], device="cuda"))
            for a, b in zip(row, alone):
                assert (a[st[x]:st[x + 1]] == b).all()
            for t, s in zip(total, dw):
                t += s.double()
        for a, t in zip(weights, total):
            # sums of the same numbers in 32 bits, in another order: at most 2^10 of them a column and sample
            assert ((a.double() - t).abs() <= 2.0 ** -14 * t.abs().max()).all()
        # the routers of the row replay the record: the gates of the rollout, the counts of its samples, gradients of both
        for l in range(L):
            x = logits[l][tokens]
            _, gate, counts, loss = rp.rp_route(x, k, st, replay=record[tokens][:, l], loss_coef=0.01)
            assert (gate - gates[l][tokens]).abs().max() <= 1e-6 and torch.isfinite(loss).all()
            if l == 0:
                seen[torch.from_numpy(mine).cuda()] = counts.long()
            dx = rp.rp_route_grad(x, record[tokens][:, l], st, counts, gates_grad=torch.ones_like(gate), loss_grad=torch.ones(1, device="cuda"), loss_coef=0.01)
            # gates of one token add up to 1, and so do the shares of the loss: a row's gradient adds up to nothing
            assert dx.float().sum(1).abs().max() <= 32 * 2.0 ** -8 * dx.float().abs().max() + 1e-6
    assert (seen == rp.rp_count_routes(record, start, E)[:, 0]).all()


@pytest.mark.gpu
def test_inputs_that_need_a_gradient_are_warned_about():
    """Autograd does not see these calls: said once where it would be expected to, and not where the caller has it switched off."""
    import warnings

    import torch
    start = torch.tensor([0, 8], device="cuda")
    q, w = torch.randn(8, 2, 64, device="cuda").half(), torch.ones(64, device="cuda")
    x = torch.randn(8, 16, device="cuda")
    calls = {"rp_attend": lambda g: rp.rp_attend(q.clone().requires_grad_(g), q, q, start), "rp_rotate": lambda g: rp.rp_rotate(q, q, None, start, q_weight=w.clone().requires_grad_(g), k_weight=w),
             "rp_route": lambda g: rp.rp_route(x.clone().requires_grad_(g), 2, start)}
    for name, call in calls.items():
        with pytest.warns(UserWarning, match=name + "_grad"):
            got = call(True)
        with warnings.catch_warnings():
            warnings.simplefilter("error")
            want = call(False)
            with torch.no_grad():
                call(True)
        assert all((a == b).all() and not a.requires_grad for a, b in zip(got, want))
