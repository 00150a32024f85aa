"""fp8_quantize and fp8_product against 64 bits (needs a B200)."""
import random

import pytest
import torch

import operator_util as ref
import paper_1901_10997_b200 as pkg

pytestmark = pytest.mark.gpu

SIZES = [(1, 1), (2, 7), (3, 16), (5, 127), (128, 128), (129, 129), (130, 256), (127, 260), (1, 1500), (257, 1501), (300, 1502), (40, 4096), (600, 33), (9, 5000)]


def make(rows, width, dtype, seed=0, apart=False):
    g = torch.Generator(device="cuda").manual_seed(rows + 3 * width + seed)
    x = torch.randn(rows, width, generator=g, device="cuda") * torch.exp(torch.randn(rows, 1, generator=g, device="cuda"))
    x = x.to(ref.TYPES[dtype])
    if apart:
        held = torch.zeros(rows, width + 3, dtype=x.dtype, device="cuda")
        held[:, 1:width + 1] = x
        x = held[:, 1:width + 1]
    return x


@pytest.mark.parametrize("block_rows", (1, 128))
@pytest.mark.parametrize("dtype", ("bf16", "fp32"))
@pytest.mark.parametrize("rows, width", SIZES)
def test_quantize(rows, width, dtype, block_rows):
    for apart in (False, True):
        x = make(rows, width, dtype, apart=apart)
        q, s = pkg.fp8_quantize(x, block_rows=block_rows)
        assert q.stride(0) % 16 == 0 and q.data_ptr() % 16 == 0 and s.is_contiguous()
        ref.check_e4m3(q, s, x.double(), block_rows, 0.0, f"apart {apart}")


def test_quantize_zeros_small_and_not_finite():
    x = torch.zeros(256, 300, device="cuda")
    x[130, 200] = 1e-44                                     # below the normal range
    x[140, 299] = float("nan")
    q, s = pkg.fp8_quantize(x, block_rows=128)
    assert not q[:, :256].float().any() and not s[:, :2].isnan().any() and bool((s[:, :2] == 2.0 ** -126).all())
    assert bool(s[1, 2].isnan()) and bool(q[128:, 256:].float().isnan().all()) and not q[:128].float().any()
    x = torch.randn(3, 140, device="cuda")
    x[1, 5] = float("-inf")
    q, s = pkg.fp8_quantize(x)
    assert float(s[1, 0]) == float("inf") and bool(q[1, 5].float().isnan()) and not q[1, :5].float().any() and not q[1, 6:128].float().any()
    for r, c in ((0, 0), (0, 1), (2, 0), (1, 1)):
        assert bool(s[r, c].isfinite())
    ref.check_e4m3(q[[0, 2]], s[[0, 2]], x[[0, 2]].double(), 1, 0.0)
    # the largest numbers there are
    big = torch.full((2, 130), torch.finfo(torch.float32).max, device="cuda")
    q, s = pkg.fp8_quantize(big)
    assert bool((q.float() == 448).all())
    assert pkg.fp8_quantize(big[:0])[0].shape == (0, 130)


def test_quantize_leaves_what_lies_between_rows():
    x = make(5, 100, "bf16")
    held = torch.full((6, 112), 77, dtype=torch.uint8, device="cuda")
    scales = torch.full((6, 1), 9.0, device="cuda")
    for block_rows in (1, 128):
        rc, why = pkg.lstm_fp8_quantize(x.data_ptr(), 100, 5, 100, pkg.LSTM_BF16, block_rows, held.data_ptr(), 112, scales.data_ptr(),
                                        torch.cuda.current_stream().cuda_stream)
        assert rc == pkg.LSTM_OK, why
        assert bool((held[:, 100:] == 77).all()) and bool((held[5] == 77).all()) and float(scales[5]) == 9.0


# ---------------------------------------------------------------- product
# every tile of rows, tiles and blocks that end anywhere, split and whole sums
PRODUCTS = [(1, 1, 1), (1, 3, 16), (2, 128, 128), (3, 129, 127), (16, 130, 129), (17, 100, 300), (32, 256, 1500), (33, 257, 1501), (50, 6000, 1500), (64, 90, 2000),
            (65, 400, 96), (100, 300, 4100), (128, 128, 640), (129, 1000, 900), (257, 511, 1313), (300, 260, 33), (700, 3000, 1500), (1000, 2050, 520),
            (2049, 1500, 200), (1, 6000, 1500), (4, 8192, 8192),
            # many tiles: pairs of CTAs, tiles, blocks and rows of the output that end anywhere, more blocks than are staged at once
            (300, 4000, 129), (1030, 1100, 260), (520, 2051, 1500), (9000, 1, 40), (8300, 3, 257), (4000, 513, 64), (1500, 900, 2200), (700, 3001, 4200)]


def operands(rows, outs, width, seed=0):
    g = torch.Generator(device="cuda").manual_seed(rows + 5 * outs + 11 * width + seed)
    x = torch.randn(rows, width, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(rows, 1, generator=g, device="cuda"))
    w = torch.randn(outs, width, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(outs, 1, generator=g, device="cuda"))
    bias = torch.randn(outs, generator=g, device="cuda")
    return (*pkg.fp8_quantize(x), *pkg.fp8_quantize(w, block_rows=128), bias)


def whole(q, s, block_rows):
    return q.double() * ref.spread(s.double(), block_rows, *q.shape)


def check_product(y, qx, sx, qw, sw, bias, what=""):
    x, w = whole(qx, sx, 1), whole(qw, sw, 128)
    want = x @ w.t() + (0 if bias is None else bias.double())
    # Products of two e4m3 values are exact.  Each of the 128 additions of a block may cut off 2 U of the magnitudes so far, each block
    # is scaled (3 roundings) and added, the parts of up to eight CTAs and the bias are added.
    blocks = sx.shape[1]
    bound = (2 * min(128, qx.shape[1]) + 3 + blocks + 8) * ref.U * (x.abs() @ w.abs().t()) + 2 * ref.U * want.abs()
    if bias is not None:
        bound = bound + ref.U * bias.double().abs()
    ref.close(y, want, bound + ref.half_step(y.dtype) * want.abs(), what)


@pytest.mark.parametrize("dtype", ("bf16", "fp32"))
@pytest.mark.parametrize("rows, outs, width", PRODUCTS)
def test_product(rows, outs, width, dtype):
    qx, sx, qw, sw, bias = operands(rows, outs, width)
    for b in (bias, None):
        y = pkg.fp8_product(qx, sx, qw, sw, b, dtype=ref.TYPES[dtype])
        check_product(y, qx, sx, qw, sw, b)
    assert torch.equal(y, pkg.fp8_product(qx, sx, qw, sw, dtype=ref.TYPES[dtype]))


def test_random_sizes():
    r = random.Random(8)
    for i in range(40):
        rows, outs, width = (int(2 ** r.uniform(0, top)) for top in (11, 11, 11.5))
        qx, sx, qw, sw, bias = operands(rows, outs, width, i)
        check_product(pkg.fp8_product(qx, sx, qw, sw, bias, dtype=torch.float32), qx, sx, qw, sw, bias, f"{rows} x {outs} x {width}")


def test_whole_numbers_are_exact():
    """Small whole numbers with scales of one: every sum is exact in 32 bits."""
    for rows, outs, width in ((7, 300, 1000), (200, 300, 1000), (1024, 1100, 777)):
        g = torch.Generator(device="cuda").manual_seed(rows)
        x = torch.randint(-4, 5, (rows, width), generator=g, device="cuda").float()
        w = torch.randint(-4, 5, (outs, width), generator=g, device="cuda").float()
        ld = (width + 15) // 16 * 16
        hold = lambda t: torch.nn.functional.pad(t, (0, ld - width), value=400.0).to(torch.float8_e4m3fn)[:, :width]     # what lies between rows is not read
        qx, qw = hold(x), hold(w)
        blocks = (width + 127) // 128
        y = pkg.fp8_product(qx, torch.ones(rows, blocks, device="cuda"), qw, torch.ones((outs + 127) // 128, blocks, device="cuda"), dtype=torch.float32)
        assert torch.equal(y.double(), x.double() @ w.double().t())


@pytest.mark.parametrize("rows", (3, 40, 300, 4100))
def test_nan_stays_in_its_row(rows):
    qx, sx, qw, sw, _ = operands(rows, 200, 300, 1)
    want = pkg.fp8_product(qx, sx, qw, sw)
    sx2 = sx.clone()
    sx2[1, 2] = float("nan")
    y = pkg.fp8_product(qx, sx2, qw, sw)
    assert bool(y[1].isnan().all())
    keep = torch.arange(rows) != 1
    assert torch.equal(y[keep], want[keep])
    sw2 = sw.clone()
    sw2[1, 0] = float("inf")
    y = pkg.fp8_product(qx, sx, qw, sw2)
    assert torch.equal(y[:, :128], want[:, :128]) and not y[:, 128:].isfinite().any()


@pytest.mark.parametrize("rows", (1, 20, 70, 500, 4400))
@pytest.mark.parametrize("dtype", ("bf16", "fp32"))
# rows that start anywhere, on 16 and on 4 bytes, and end anywhere or on 16 bytes
@pytest.mark.parametrize("at, ld, outs", ((3, 140, 131), (16, 176, 131), (2, 142, 131), (16, 176, 136)))
def test_rows_and_columns_beside_the_output_are_left(rows, dtype, at, ld, outs):
    qx, sx, qw, sw, bias = operands(rows, outs, 200, 2)
    want = pkg.fp8_product(qx, sx, qw, sw, bias, dtype=ref.TYPES[dtype])
    held = torch.full((rows + 2, ld), 5.0, dtype=ref.TYPES[dtype], device="cuda")
    out = held[1:rows + 1, at:at + outs]
    assert pkg.fp8_product(qx, sx, qw, sw, bias, dtype=held.dtype, out=out) is out
    assert torch.equal(out, want)
    out.fill_(5.0)
    assert bool((held == 5.0).all())


def test_offsets_beyond_32_bits():
    far = (1 << 30) + 16
    held = torch.empty(2 * far + 4096, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    qx0, sx, qw0, sw, bias = operands(3, 3, 200, 3)
    put = lambda t, at: held.as_strided((3, 200), (far, 1), at).copy_(t)
    qx, qw = put(qx0, 0), put(qw0, 512)
    y = torch.empty(2 * far + 64, dtype=torch.bfloat16, device="cuda").as_strided((3, 3), (far, 1), 1)
    want = pkg.fp8_product(qx0, sx, qw0, sw, bias)
    assert torch.equal(want, pkg.fp8_product(qx, sx, qw, sw, bias, out=y))


def test_recorded_and_on_two_streams():
    sets = [operands(12, 3000, 1500, 4), operands(700, 3000, 1500, 5), operands(90, 500, 2000, 6)]
    run = lambda s: (pkg.fp8_product(*s), pkg.fp8_product(*s, dtype=torch.float32))
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
            other = [run(s) for s in sets]
        for g in graphs[1:]:
            g.replay()
        here = [run(s) for s in sets]
        torch.cuda.synchronize()
        for got in (outs, other, here):
            for o, w in zip(got, want):
                assert all(torch.equal(p, q) for p, q in zip(o, w))


def test_tensors_that_do_not_fit_are_refused():
    qx, sx, qw, sw, bias = operands(4, 40, 200)
    f8 = torch.float8_e4m3fn
    for bad in (lambda: pkg.fp8_product(qx.float(), sx, qw, sw), lambda: pkg.fp8_product(qx, sx[:, :1], qw, sw), lambda: pkg.fp8_product(qx, sx, qw[:, :100], sw),
                lambda: pkg.fp8_product(qx, sx, qw, sw[:0]), lambda: pkg.fp8_product(qx, sx, qw, sw, bias[:3]), lambda: pkg.fp8_product(qx, sx, qw, sw, bias.bfloat16()),
                lambda: pkg.fp8_product(qx, sx, qw, sw, dtype=torch.float16), lambda: pkg.fp8_product(qx, sx.bfloat16(), qw, sw),
                lambda: pkg.fp8_product(qx, sx, qw, sw, out=torch.empty(4, 41, dtype=torch.bfloat16, device="cuda")),
                lambda: pkg.fp8_product(qx, sx, qw, sw, out=torch.empty(1, 40, dtype=torch.bfloat16, device="cuda").expand(4, 40)),
                lambda: pkg.fp8_quantize(torch.zeros(3, 8, device="cuda", dtype=torch.float16)), lambda: pkg.fp8_quantize(torch.zeros(8, 3, device="cuda").t())):
        with pytest.raises(ValueError):
            bad()
    for bad in (lambda: pkg.fp8_product(torch.zeros(4, 201, device="cuda").to(f8)[:, :200], sx, qw, sw), lambda: pkg.fp8_quantize(torch.zeros(3, 8, device="cuda"), block_rows=2)):
        with pytest.raises(pkg.LstmError) as e:
            bad()
        assert e.value.code == pkg.LSTM_ERR_INVALID
