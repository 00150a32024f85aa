"""rms_norm, its 8-bit output and its gradients against 64 bits (needs a B200)."""
import itertools
import random

import pytest
import torch

import operator_util as ref
import paper_1901_10997_b200 as pkg

pytestmark = pytest.mark.gpu

# widths off every vector and strip; one, 4 and 8 warps a row; rows that do not fill a CTA
SIZES = [(1, 1), (2, 2), (3, 7), (5, 8), (4, 127), (7, 128), (9, 129), (1, 255), (6, 256), (5, 260), (3, 513), (33, 1500), (4, 1502), (3, 1501), (20, 1600),
         (2, 2048), (3, 2050), (5, 2049), (2, 4100), (3, 8192), (2, 8193), (1, 16384), (2, 16383), (1000, 200), (6000, 40)]


def make(rows, width, dtype, residual, seed=0, layout="plain"):
    g = torch.Generator(device="cuda").manual_seed(rows + 7 * width + seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    dt = ref.TYPES[dtype]
    x, res, dy = 1.5 * n(rows, width), 3 * n(rows, width), n(rows, width)
    if layout == "apart":       # columns of a wider matrix, rows further apart and off their alignment
        held = torch.zeros(3, rows, width + 5, device="cuda", dtype=dt)
        for t, h in zip((x, res, dy), held):
            h[:, 3:width + 3] = t.to(dt)
        x, res, dy = (h[:, 3:width + 3] for h in held)
    else:
        x, res, dy = (t.to(dt) for t in (x, res, dy))
    return x, 1 + 0.2 * n(width), res if residual else None, dy


def terms(width):
    """Additions in a row of the sum: 64 a lane, 5 by shuffles, 8 warps; squares and a mean."""
    return min(64, -(-width // 32) + 8) + 5 + 16 + 3


def norm(x, w, residual, eps):
    r = x.double() + (0 if residual is None else residual.double())
    rstd = 1 / torch.sqrt(r.square().mean(1, keepdim=True) + eps)
    # the sum x + residual is rounded, the mean's error counts half in rstd, then a root, a quotient and two products
    loss = 0 if residual is None else ref.U * r.abs()
    return r, rstd, r * rstd * w.double(), rstd * w.double().abs() * loss, (terms(x.shape[1]) / 2 + 8) * ref.U


def cases():
    r = random.Random(4)
    for size in SIZES:
        for mode in r.sample(list(itertools.product(("bf16", "fp32"), (True, False), ("plain", "apart"))), 4):
            yield (*size, *mode)


@pytest.mark.parametrize("c", list(cases()), ids=lambda c: "_".join(str(v) for v in c))
def test_against_64_bits(c):
    rows, width, dtype, residual, layout = c
    x, w, res, dy = make(rows, width, dtype, residual, layout=layout)
    eps = 1e-5
    r, rstd, want, off, e = norm(x, w, res, eps)
    half = ref.half_step(x.dtype)
    y, stored = pkg.rms_norm(x, w, res, eps=eps)
    ref.close(y, want, half * want.abs() + off + e * want.abs(), "y")
    q, scales, stored8 = pkg.rms_norm_fp8(x, w, res, eps=eps)
    if residual:
        ref.close(stored, r, half * r.abs() + ref.U * r.abs(), "r")
        assert torch.equal(stored, stored8)
    else:
        assert stored is None and stored8 is None
    # relative error of an element that is a difference of two others may be anything; magnitudes near zero are absorbed by U of the largest
    assert q.stride(0) % 16 == 0 and q.data_ptr() % 16 == 0
    ref.check_e4m3(q, scales, want, 1, e + 2 * ref.U, "8 bits")

    at = x if stored is None else stored
    past = res if residual else None
    dx, dw = pkg.rms_norm_backward(dy, at, w, past, eps=eps)
    r = at.double()
    rstd = 1 / torch.sqrt(r.square().mean(1, keepdim=True) + eps)
    wdy = dy.double() * w.double()
    back = r * rstd ** 3 * (wdy * r).mean(1, keepdim=True)
    wx = rstd * wdy - back + (0 if past is None else past.double())
    size = (rstd * wdy).abs() + r.abs() * rstd ** 3 * (wdy * r).abs().mean(1, keepdim=True)
    ref.close(dx, wx, half * wx.abs() + 3 * (terms(width) + 8) * ref.U * size + ref.U * wx.abs(), "dx")
    each = dy.double() * r * rstd
    # a thread adds its rows one by one, then 32 threads and 5 shuffles join
    ref.close(dw, each.sum(0), (rows + 64 + terms(width)) * ref.U * each.abs().sum(0), "dw")


def test_gradients_against_differences():
    rows, width, eps = 5, 70, 1e-4
    x, w, res, dy = make(rows, width, "fp32", True, 1)
    dr = torch.randn(rows, width, device="cuda")
    r = x + res
    dx, dw = pkg.rms_norm_backward(dy, r, w, dr, eps=eps)

    def loss(r, w):
        return float((norm(r, w, None, eps)[2] * dy.double()).sum() + (r * dr.double()).sum())

    step = 1e-5
    for grad, i in ((dx, 0), (dw, 1)):
        v = torch.randn(grad.shape, device="cuda", dtype=torch.float64)
        args = [r.double(), w.double()]
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + step * v, args[i] - step * v
        slope, mine = (loss(*up) - loss(*down)) / (2 * step), float((grad.double() * v).sum())
        assert abs(slope - mine) <= 1e-6 * (float((grad.double() * v).abs().sum()) + 1), (i, slope, mine)


@pytest.mark.parametrize("width", (96, 600, 3000))
def test_zeros_infinities_and_nan(width):
    x, w, *_ = make(6, width, "fp32", False, 2)
    x[1] = 0
    x[2, 5] = float("nan")
    x[3, 90] = float("inf")
    x[4] = 1e-30
    y, _ = pkg.rms_norm(x, w, eps=0.0 + 1e-6)
    q, scales, _ = pkg.rms_norm_fp8(x, w)
    assert not y[1].any() and not q[1].float().any() and bool((scales[1] > 0).all())
    assert bool(y[2].isnan().all()) and bool(scales[2].isnan().all()) and bool(q[2].float().isnan().all())
    assert bool(y[3, 90].isnan()) and not y[3, :90].any()           # an infinite row has no length left for its other elements
    assert bool(scales[3, 0].isnan())
    assert bool(y[0].isfinite().all()) and bool(y[5].isfinite().all()) and bool(y[4].isfinite().all())
    z, _ = pkg.rms_norm(x[1:2], w, eps=0.0)                          # 0 / 0
    assert bool(z.isnan().all())


def test_bytes_between_rows_are_left_as_they_were():
    x, w, *_ = make(5, 100, "bf16", False, 3)
    held = torch.full((6, 112), 77, dtype=torch.uint8, device="cuda")
    scales = torch.full((6, 1), 9.0, device="cuda")
    rc, why = pkg.lstm_rms_norm(x.data_ptr(), 100, 0, 0, w.data_ptr(), 1e-6, 5, 100, pkg.LSTM_BF16, held.data_ptr(), 112, scales.data_ptr(), 0, 0,
                                torch.cuda.current_stream().cuda_stream)
    assert rc == pkg.LSTM_OK, why
    q, s, _ = pkg.rms_norm_fp8(x, w)
    assert torch.equal(held[:5, :100], q.contiguous().view(torch.uint8)) and torch.equal(scales[:5], s)
    assert bool((held[:, 100:] == 77).all()) and bool((held[5] == 77).all()) and float(scales[5]) == 9.0


def test_no_rows():
    w = torch.ones(24, device="cuda")
    x = torch.empty(0, 24, device="cuda", dtype=torch.bfloat16)
    assert pkg.rms_norm(x, w)[0].shape == (0, 24) and pkg.rms_norm_fp8(x, w)[1].shape == (0, 1)
    dx, dw = pkg.rms_norm_backward(x, x, w)
    assert dx.shape == (0, 24) and not dw.any()


def test_offsets_beyond_32_bits():
    far = (1 << 30) + 8
    held = torch.empty(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    x0, w, r0, dy0 = make(3, 200, "bf16", True, 4)
    put = lambda t, at: held.as_strided((3, 200), (far, 1), at).copy_(t)
    x, r, dy = put(x0, 0), put(r0, 512), put(dy0, 1024)
    for p, q in zip((*pkg.rms_norm(x, w, r), *pkg.rms_norm_fp8(x, w, r), *pkg.rms_norm_backward(dy, x, w, r)),
                    (*pkg.rms_norm(x0, w, r0), *pkg.rms_norm_fp8(x0, w, r0), *pkg.rms_norm_backward(dy0, x0, w, r0))):
        assert torch.equal(p.float(), q.float())


def test_the_same_bits_again_recorded_and_on_two_streams():
    sets = [make(3000, 1500, "bf16", True, s) for s in (5, 6)]
    run = lambda s: (*pkg.rms_norm(s[0], s[1], s[2]), *pkg.rms_norm_backward(s[3], s[0], s[1], s[2]))
    want = [run(s) for s in sets]
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(run(s))
        graphs.append(g)
    side = torch.cuda.Stream()
    for _ in range(3):
        for o in outs:
            for t in o:
                t.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graphs[0].replay()
            other = run(sets[0])
        graphs[1].replay()
        here = run(sets[1])
        torch.cuda.synchronize()
        for got, w in ((outs[0], want[0]), (outs[1], want[1]), (other, want[0]), (here, want[1])):
            assert all(torch.equal(p, q) for p, q in zip(got, w))


def test_a_workspace_that_is_too_small_is_refused():
    x, w, _, dy = make(40, 64, "fp32", False, 7)
    need = pkg.lstm_rms_norm_workspace(40, 64)
    assert need > 0 and pkg.lstm_rms_norm_workspace(0, 64) == 0 and pkg.lstm_rms_norm_workspace(4, 0) == -1
    ws, dx, dw = torch.empty(need, device="cuda"), torch.empty_like(x), torch.empty(64, device="cuda")
    call = lambda n, at: pkg.lstm_rms_norm_backward(dy.data_ptr(), 64, x.data_ptr(), 64, w.data_ptr(), 0, 0, 1e-6, 40, 64, pkg.LSTM_F32, dx.data_ptr(), 64,
                                                    dw.data_ptr(), at, n, torch.cuda.current_stream().cuda_stream)
    assert call(need - 1, ws.data_ptr())[0] == pkg.LSTM_ERR_INVALID and call(need, 0)[0] == pkg.LSTM_ERR_INVALID
    assert call(need, ws.data_ptr()) == (pkg.LSTM_OK, "")


def test_tensors_that_do_not_fit_are_refused():
    x, w, res, dy = make(4, 32, "bf16", True)
    for bad in (lambda: pkg.rms_norm(x, w[:5]), lambda: pkg.rms_norm(x, w.bfloat16()), lambda: pkg.rms_norm(x, w, res.float()), lambda: pkg.rms_norm(x.half(), w),
                lambda: pkg.rms_norm(x.t(), w[:4]), lambda: pkg.rms_norm(x, None), lambda: pkg.rms_norm_fp8(x, w, res[:2]),
                lambda: pkg.rms_norm_backward(dy[:1], x, w), lambda: pkg.rms_norm_backward(dy, x, w, res.float()), lambda: pkg.rms_norm_backward(None, x, w)):
        with pytest.raises(ValueError):
            bad()
    with pytest.raises(pkg.LstmError) as e:
        pkg.rms_norm(torch.zeros(1, 16385, device="cuda"), torch.ones(16385, device="cuda"))
    assert e.value.code == pkg.LSTM_ERR_UNSUPPORTED
