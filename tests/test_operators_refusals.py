"""What the stateless operators refuse, on the CPU: every check of arguments comes before the first CUDA call, so the addresses
here are never read."""
import pytest

import paper_1901_10997_b200 as pkg

P = 1 << 20            # an address that is aligned to anything
F32, BF16, W = pkg.LSTM_F32, pkg.LSTM_BF16, pkg.LSTM_BF16W_F32S


@pytest.fixture(scope="module", autouse=True)
def _built():
    from paper_1901_10997_b200 import build
    build.build()


def recurrence(**k):
    v = dict(a=P, a_t=8, a_b=8, x=P, x_t=8, x_b=8, h0=0, lengths=0, T=4, B=1, D=8, dtype=F32, flags=1, h=P, h_t=8, h_b=8, hT=0, states=0)
    return pkg.lstm_linear_recurrence(*(v | k).values())


def recurrence_backward(**k):
    v = dict(a=P, a_t=8, a_b=8, x=P, x_t=8, x_b=8, states=P, dh=P, dh_t=8, dh_b=8, dhT=0, lengths=0, T=4, B=1, D=8, dtype=F32, flags=1,
             da=P, da_t=8, da_b=8, dx=P, dx_t=8, dx_b=8, dh0=0)
    return pkg.lstm_linear_recurrence_backward(*(v | k).values())


def norm(**k):
    v = dict(x=P, x_ld=8, residual=0, residual_ld=0, w=P, eps=1e-6, rows=2, width=8, dtype=BF16, y=P, y_ld=16, scales=0, r=0, r_ld=0)
    return pkg.lstm_rms_norm(*(v | k).values())


def norm_backward(**k):
    v = dict(dy=P, dy_ld=8, r=P, r_ld=8, w=P, dr=0, dr_ld=0, eps=1e-6, rows=2, width=8, dtype=BF16, dx=P, dx_ld=8, dw=P, workspace=P, floats=1 << 20)
    return pkg.lstm_rms_norm_backward(*(v | k).values())


def quantize(**k):
    v = dict(x=P, x_ld=8, rows=2, width=8, dtype=BF16, block_rows=1, q=P, q_ld=16, scales=P)
    return pkg.lstm_fp8_quantize(*(v | k).values())


def product(**k):
    v = dict(qx=P, qx_ld=16, sx=P, qw=P, qw_ld=16, sw=P, bias=0, rows=2, outs=3, width=8, dtype=BF16, y=P, y_ld=3)
    return pkg.lstm_fp8_product(*(v | k).values())


BAD = [
    (recurrence, dict(T=-1)), (recurrence, dict(B=-1)), (recurrence, dict(D=0)), (recurrence, dict(dtype=W)), (recurrence, dict(dtype=7)),
    (recurrence, dict(flags=4)), (recurrence, dict(a=0)), (recurrence, dict(x=0)), (recurrence, dict(h=0)), (recurrence, dict(a=P + 2)),
    (recurrence, dict(dtype=BF16, x=P + 1)), (recurrence, dict(h=P + 1)), (recurrence, dict(h0=P + 2)), (recurrence, dict(hT=P + 2)),
    (recurrence, dict(states=P + 2)), (recurrence, dict(lengths=P + 1)),
    (recurrence_backward, dict(T=-1)), (recurrence_backward, dict(states=0)), (recurrence_backward, dict(dh=0)), (recurrence_backward, dict(da=0)),
    (recurrence_backward, dict(dx=0)), (recurrence_backward, dict(flags=8)), (recurrence_backward, dict(dtype=1)), (recurrence_backward, dict(dh=P + 2)),
    (recurrence_backward, dict(dh0=P + 1)),
    (norm, dict(rows=-1)), (norm, dict(width=0)), (norm, dict(dtype=W)), (norm, dict(eps=-1.0)), (norm, dict(eps=float("nan"))), (norm, dict(x=0)),
    (norm, dict(w=0)), (norm, dict(y=0)), (norm, dict(x=P + 1)), (norm, dict(residual=P + 1)), (norm, dict(r=P + 1)), (norm, dict(w=P + 2)),
    (norm, dict(scales=P, y=P + 8)), (norm, dict(scales=P, y_ld=8)), (norm, dict(scales=P + 2)),
    (norm_backward, dict(rows=-1)), (norm_backward, dict(width=-3)), (norm_backward, dict(dw=0)), (norm_backward, dict(dy=0)),
    (norm_backward, dict(r=0)), (norm_backward, dict(w=0)), (norm_backward, dict(dx=0)), (norm_backward, dict(dtype=1)), (norm_backward, dict(dr=P + 1)),
    (quantize, dict(rows=-1)), (quantize, dict(width=0)), (quantize, dict(dtype=W)), (quantize, dict(block_rows=64)), (quantize, dict(block_rows=0)),
    (quantize, dict(x=0)), (quantize, dict(q=0)), (quantize, dict(scales=0)), (quantize, dict(q=P + 8)), (quantize, dict(q_ld=8)), (quantize, dict(x=P + 1)),
    (product, dict(rows=-1)), (product, dict(outs=-1)), (product, dict(width=0)), (product, dict(dtype=W)), (product, dict(qx=0)), (product, dict(sx=0)),
    (product, dict(qw=0)), (product, dict(sw=0)), (product, dict(y=0)), (product, dict(qx=P + 8)), (product, dict(qw=P + 1)), (product, dict(qx_ld=8)),
    (product, dict(qw_ld=24)), (product, dict(width=40)), (product, dict(sx=P + 2)), (product, dict(y=P + 1)), (product, dict(bias=P + 2)),
]


@pytest.mark.parametrize("call, change", BAD, ids=lambda v: v.__name__ if callable(v) else "_".join(f"{k}{x}" for k, x in v.items()))
def test_bad_arguments_are_refused_with_a_reason(call, change):
    rc, why = call(**change)
    assert rc == pkg.LSTM_ERR_INVALID and "bad argument" in why


def test_rows_too_wide_for_the_norm():
    for call in (norm, norm_backward):
        rc, why = call(width=pkg.LSTM_RMS_NORM_MAX_WIDTH + 1)
        assert rc == pkg.LSTM_ERR_UNSUPPORTED and "LSTM_RMS_NORM_MAX_WIDTH" in why


def test_sizes_beyond_the_grid():
    assert quantize(rows=65535 * 128 + 1, block_rows=128)[0] == pkg.LSTM_ERR_UNSUPPORTED
    assert product(rows=65535 * 128 + 1)[0] == pkg.LSTM_ERR_UNSUPPORTED


@pytest.mark.parametrize("call, change", [(recurrence, dict(B=0)), (recurrence, dict(T=0)), (norm, dict(rows=0, x=0, y=0)), (quantize, dict(rows=0)),
                                          (product, dict(rows=0)), (product, dict(outs=0))], ids=lambda v: v.__name__ if callable(v) else "_".join(v))
def test_nothing_to_do_is_no_error(call, change):
    assert call(**change) == (pkg.LSTM_OK, "")


def test_without_a_device_the_calls_say_so():
    import torch
    if torch.cuda.is_available():
        pytest.skip("a device is present")
    for call in (recurrence, recurrence_backward, norm, norm_backward, quantize, product):
        rc, why = call()
        assert rc == pkg.LSTM_ERR_CUDA and why
    assert pkg.lstm_rms_norm_workspace(4, 8) == -1


def test_a_reason_longer_than_its_buffer_is_cut():
    import ctypes
    lib = pkg.load_library()
    err = ctypes.create_string_buffer(b"x" * 11, 12)
    args = [P, 8, 2, 8, F32, 5, P, 16, P, None]
    assert lib.lstm_fp8_quantize(*args, err, 8) == pkg.LSTM_ERR_INVALID and err.raw == b"bad arg\0xxx\0"
    assert lib.lstm_fp8_quantize(*args, None, 0) == pkg.LSTM_ERR_INVALID


def test_tensors_of_the_host_are_refused():
    import torch
    x = torch.zeros(4, 2, 8)
    for call in (lambda: pkg.linear_recurrence(x, x), lambda: pkg.linear_recurrence_backward(x, x, x, x), lambda: pkg.rms_norm(x[0], x[0, 0]),
                 lambda: pkg.rms_norm_fp8(x[0], x[0, 0]), lambda: pkg.rms_norm_backward(x[0], x[0], x[0, 0]), lambda: pkg.fp8_quantize(x[0]),
                 lambda: pkg.fp8_product(x[0], x[0], x[0], x[0])):
        with pytest.raises(ValueError):
            call()
