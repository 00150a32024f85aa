"""Strides by which an output of the stateless operators would overlap itself are refused, and no others (CPU: before the first CUDA call)."""
import random

import pytest

import paper_1901_10997_b200 as pkg
from test_operators_refusals import P, _built, norm, norm_backward, product, quantize, recurrence, recurrence_backward  # noqa: F401  (_built: the fixture)

OVERLAP = [
    (quantize, dict(q_ld=0)), (quantize, dict(width=100, q_ld=16)), (quantize, dict(width=100, q_ld=96, block_rows=128)), (quantize, dict(width=100, q_ld=-96)),
    (norm, dict(scales=P, y_ld=0)), (norm, dict(scales=P, width=100, y_ld=96)), (norm, dict(y_ld=0)), (norm, dict(y_ld=7)), (norm, dict(y_ld=-7)),
    (norm, dict(r=P, r_ld=0)), (norm, dict(r=P, r_ld=7)), (norm_backward, dict(dx_ld=0)), (norm_backward, dict(dx_ld=7)),
    (product, dict(y_ld=0)), (product, dict(y_ld=2)),
    (recurrence, dict(h_t=0)), (recurrence, dict(h_t=7)), (recurrence, dict(h_t=-7)), (recurrence, dict(B=2, h_b=0, h_t=16)), (recurrence, dict(B=2, h_b=8, h_t=8)),
    (recurrence, dict(B=4, h_b=16, h_t=24)), (recurrence, dict(B=2, h_b=20, h_t=8)),
    (recurrence_backward, dict(da_t=4)), (recurrence_backward, dict(dx_t=0)), (recurrence_backward, dict(B=2, dx_b=8)),
]


@pytest.mark.parametrize("call, change", OVERLAP, ids=lambda v: v.__name__ if callable(v) else "_".join(f"{k}{x}" for k, x in v.items()))
def test_outputs_that_overlap_themselves_are_refused(call, change):
    rc, why = call(**change)
    assert rc == pkg.LSTM_ERR_INVALID and "overlap" in why


def served(call, **change):
    """Not refused for its arguments (there may be no device, and the addresses are not real ones: nothing is to be launched)."""
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    return call(**change)[0] == pkg.LSTM_ERR_CUDA


def test_others_are_not():
    for call, change in ((quantize, dict(rows=1, q_ld=0)), (quantize, dict(q_ld=16)), (quantize, dict(q_ld=-16)), (norm, dict(rows=1, y_ld=0)), (norm, dict(r_ld=0)),
                         (norm, dict(y_ld=8, r=P, r_ld=-8)), (norm_backward, dict(dx_ld=8)), (norm_backward, dict(rows=1, dx_ld=0)), (product, dict(rows=1, y_ld=0)),
                         (recurrence, dict(T=1, h_t=0)), (recurrence, dict(h_b=0)), (recurrence, dict(h_t=-8)), (recurrence, dict(B=2, h_b=32, h_t=8)),
                         (recurrence, dict(B=2, h_b=8, h_t=16)), (recurrence, dict(B=2, h_b=12, h_t=24)), (recurrence_backward, dict(B=2, da_b=32, dx_t=16))):
        assert served(call, **change), (call.__name__, change)


def test_every_small_layout():
    r = random.Random(3)
    seen = [0, 0]
    for _ in range(1500):
        T, B, D = r.randint(1, 5), r.randint(1, 5), r.randint(1, 4)
        t, b = r.randint(-24, 24), r.randint(-24, 24)
        places = [i * t + j * b + d for i in range(T) for j in range(B) for d in range(D)]
        apart = len(set(places)) == len(places)
        assert served(recurrence, T=T, B=B, D=D, h_t=t, h_b=b) == apart, (T, B, D, t, b)
        seen[apart] += 1
    assert min(seen) > 300
