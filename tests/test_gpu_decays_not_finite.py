"""linear_recurrence with decays that are NaN or infinite: no state behind such a step is finite again, whatever span, warp, CTA or chunk
the step begins (needs a B200)."""
import pytest
import torch

import paper_1901_10997_b200 as pkg

pytestmark = pytest.mark.gpu

# a few steps, a cluster, many channels (vectors of four, two and one), chunks of time
SHAPES = [(3, 2, 8), (90, 1, 6), (300, 1, 32), (700, 1, 101), (200, 60, 700), (130, 40, 602), (130, 20, 301), (8200, 1, 1000), (4100, 2, 1002), (2100, 5, 801)]
PLACES = (0, 1, 4, 7, 8, 16, 48, 63, 64, 127, 128, 500, 1024, 2048, 2099)


def not_finite(t, what):
    assert not t.isfinite().any(), what


@pytest.mark.parametrize("reverse", (False, True))
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("shape", SHAPES, ids=str)
def test_a_bad_decay_is_not_lost(shape, dtype, reverse):
    T, B, D = shape
    g = torch.Generator(device="cuda").manual_seed(T + D)
    a = (0.3 + 0.6 * torch.rand(T, B, D, generator=g, device="cuda")).to(dtype)
    x, dh = (torch.randn(T, B, D, generator=g, device="cuda").to(dtype) for _ in range(2))
    h0, dhT = (1 + torch.rand(B, D, generator=g, device="cuda") for _ in range(2))
    order = (lambda t: t.flip(0)) if reverse else (lambda t: t)               # steps in the order of processing
    places = [p for p in PLACES if p < T]
    # every place in a channel of its own; NaN, and infinities of either sign
    bad = a.clone()
    for i, p in enumerate(places):
        order_p = T - 1 - p if reverse else p
        for b in range(B):
            bad[order_p, b, i % D::min(len(places) + 1, D)] = (float("nan"), float("inf"), float("-inf"))[(i + b) % 3]
    spoilt = ~order(bad).isfinite()                                             # [T, B, D] in the order of processing
    behind = spoilt.cumsum(0) > 0                                               # at a bad step and after it
    for start in (None, h0):
        want = pkg.linear_recurrence(a, x, start, gate=False, reverse=reverse, save=True)
        h, hT, states = pkg.linear_recurrence(bad, x, start, gate=False, reverse=reverse, save=True)
        not_finite(order(h)[behind], "h")
        not_finite(hT[behind[-1]], "hT")
        front = torch.cat([torch.zeros_like(behind[:1]), behind[15:-1:16]])     # in front of steps 0, 16, 32, ...
        assert front.shape == states.shape
        not_finite(states[front], "states")
        assert torch.equal(order(h)[~behind], order(want[0])[~behind]) and torch.equal(hT[~behind[-1]], want[1][~behind[-1]])
        assert torch.equal(states[~front], want[2][~front])

        da, dx, dh0 = pkg.linear_recurrence_backward(bad, x, states, dh, dhT, gate=False, reverse=reverse)
        wa, wx, w0 = pkg.linear_recurrence_backward(a, x, want[2], dh, dhT, gate=False, reverse=reverse)
        # g_t sees the decays behind t, h_{t-1} those in front of it
        before = spoilt.flip(0).cumsum(0).flip(0) - spoilt.long() > 0           # in front of a bad step
        past = torch.cat([torch.zeros_like(behind[:1]), behind[:-1]])           # h_{t-1} is spoilt
        not_finite(order(dx)[before], "dx")
        not_finite(order(da)[before | past], "da")
        not_finite(dh0[behind[-1]], "dh0")
        assert torch.equal(order(dx)[~before], order(wx)[~before]) and torch.equal(order(da)[~(before | past)], order(wa)[~(before | past)])
        assert torch.equal(dh0[~behind[-1]], w0[~behind[-1]])
