"""Sizes that 32 bits do not hold, or whose last strip of columns they would not, are refused; no work of that size is started."""
import pytest
import torch

import paper_1901_10997_b200 as pkg
from test_operators_refusals import P, _built, product, quantize  # noqa: F401  (_built: the fixture)

MOST = 2 ** 31 - 4096


@pytest.mark.parametrize("call, change", ((quantize, dict(rows=1, width=MOST + 1, block_rows=128)), (quantize, dict(rows=1, width=2 ** 31 - 1, block_rows=128)),
                                          (quantize, dict(rows=1, width=2 ** 31 - 1)), (product, dict(rows=1, width=2 ** 31 - 1, qx_ld=2 ** 31, qw_ld=2 ** 31)),
                                          (product, dict(rows=1, outs=2 ** 31 - 1)), (product, dict(rows=1, outs=MOST + 1))))
def test_columns_beyond_the_last_strip(call, change):
    assert call(**change)[0] == pkg.LSTM_ERR_UNSUPPORTED


@pytest.mark.gpu
@pytest.mark.parametrize("n", (2 ** 31, 2 ** 32 + 1))
def test_dimensions_of_tensors(n):
    one = torch.zeros(1, 1, device="cuda", dtype=torch.bfloat16)
    w, s = torch.zeros(1, device="cuda"), torch.zeros(1, 1, device="cuda")
    q = torch.zeros(1, 16, device="cuda", dtype=torch.uint8).view(torch.float8_e4m3fn)[:, :1]
    many, steps = one.expand(n, 1), one[None].expand(n, 1, 1)
    for bad in (lambda: pkg.linear_recurrence(steps, steps), lambda: pkg.linear_recurrence(steps.transpose(0, 1), steps.transpose(0, 1)),
                lambda: pkg.linear_recurrence_backward(steps, steps, s[None], steps), lambda: pkg.rms_norm(many, w), lambda: pkg.rms_norm_fp8(many, w),
                lambda: pkg.rms_norm_backward(many, many, w), lambda: pkg.fp8_quantize(many), lambda: pkg.fp8_quantize(many, block_rows=128),
                lambda: pkg.fp8_product(q.expand(n, 1), s, q, s), lambda: pkg.fp8_product(q, s, q.expand(n, 1), s)):
        with pytest.raises(ValueError, match="2\\^31"):
            bad()
