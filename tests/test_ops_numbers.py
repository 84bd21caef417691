"""Numbers of a call that come as tensors or arrays: what they hold at the call is what counts."""
import numpy as np
import pytest

import paper_2608_12146_b200.binding as rp


def test_what_a_call_is_kept_by_follows_the_number():
    torch = rp._torch()
    q = torch.zeros(1, 2, 64, dtype=torch.bfloat16)
    for scale in (torch.tensor(0.25), np.array(0.25)):
        first = rp._config(q, q, np.bool_(True), scale)
        scale *= 2
        second = rp._config(q, q, True, scale)
        assert [rp._attention(*x)[0].scale for x in (first, second)] == [0.25, 0.5] and all(type(x) in (int, float) for x in first + second)
    assert rp._config(q, q, True, None)[-1] is None and rp._attention(*rp._config(q, q, True, None))[0].scale == 0.125


@pytest.mark.gpu
def test_numbers_that_change_between_calls():
    import torch
    g = torch.Generator().manual_seed(1)
    q, k, v = (torch.randn(300, n, 64, generator=g).bfloat16().cuda() for n in (4, 2, 2))
    start, freq = torch.tensor([0, 130, 300], device="cuda"), torch.logspace(0, -3, 32, dtype=torch.float64, device="cuda")
    axis, position = torch.zeros(32, dtype=torch.int32, device="cuda"), torch.arange(300, device="cuda")[None]
    logits = torch.randn(300, 16, generator=g).cuda()
    calls = [
        lambda x: rp.rp_attend(q, k, v, start, scale=x), lambda x: rp.rp_attend_window(q, k, v, start, window=50, scale=x),
        lambda x: rp.rp_attend_step(q[:2], k, v, start, scale=x), lambda x: rp.rp_rotate(q, k, freq, start, mscale=x),
        lambda x: rp.rp_rotate_axes(q, k, freq, axis, position, mscale=x), lambda x: rp.rp_rotate(q, k, None, start, q_weight=q[0, 0], k_weight=k[0, 0], eps=x),
        lambda x: rp.rp_route(logits, 4, start, scale=x), lambda x: rp.rp_route(logits, 4, start, loss_coef=x),
    ]
    for call in calls:
        x = torch.tensor(0.5)
        for value in (0.5, 2.0):
            x.fill_(value)
            for got, want in zip(call(x), call(value)):
                assert (got == want).all()
        assert any((a != b).any() for a, b in zip(call(0.5), call(2.0)))
