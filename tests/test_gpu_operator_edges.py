"""The stateless operators through their C entries at the edges of what they take: what lies beside an output is left (needs a B200)."""
import pytest
import torch

import paper_1901_10997_b200 as pkg

pytestmark = pytest.mark.gpu


def stream():
    return torch.cuda.current_stream().cuda_stream


@pytest.mark.parametrize("dtype, code", ((torch.bfloat16, pkg.LSTM_BF16), (torch.float32, pkg.LSTM_F32)))
@pytest.mark.parametrize("D", (8, 10, 7))
@pytest.mark.parametrize("T", (0, 1, 4, 5, 17))
def test_saved_states_are_as_many_as_there_are_segments(T, D, dtype, code):
    B, planes = 3, -(-T // pkg.LSTM_LINREC_SEGMENT)
    a, x = (torch.randn(max(T, 1), B, D, device="cuda").to(dtype) for _ in range(2))
    h0, h, hT = torch.randn(B, D, device="cuda"), torch.empty_like(a), torch.empty(B, D, device="cuda")
    held = torch.full((planes + 2, B, D), 5.0, device="cuda")
    rc, why = pkg.lstm_linear_recurrence(a.data_ptr(), B * D, D, x.data_ptr(), B * D, D, h0.data_ptr(), 0, T, B, D, code, pkg.LSTM_LINREC_GATE, h.data_ptr(), B * D, D,
                                         hT.data_ptr(), held[1:].data_ptr(), stream=stream())
    assert rc == pkg.LSTM_OK, why
    assert bool((held[0] == 5.0).all()) and bool((held[planes + 1:] == 5.0).all())
    if T:
        assert torch.equal(held[1], h0)
    else:
        assert torch.equal(hT, h0)
