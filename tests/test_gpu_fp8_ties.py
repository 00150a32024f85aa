"""fp8_quantize of values with few digits, whose quotients are often ties: q is the nearest e4m3 value of 448 x / max |x|, ties to even,
without exception (needs a B200)."""
import pytest
import torch

import paper_1901_10997_b200 as pkg

pytestmark = pytest.mark.gpu


def nearest_even(v):
    """The e4m3 value nearest to v (64 bits), ties to the one whose last bit is zero."""
    codes = torch.arange(127, dtype=torch.uint8, device=v.device)              # positive values in order: their codes are, too
    grid = codes.view(torch.float8_e4m3fn).double()
    m = v.abs()
    hi = torch.searchsorted(grid, m.contiguous()).clamp(1, 126)
    lo = hi - 1
    down, up = m - grid[lo], grid[hi] - m                                       # exact: neighbours within a factor of two, or below a step
    take = torch.where(down == up, hi % 2 == 0, up < down)
    return torch.where(take, grid[hi], grid[lo]).copysign(v)


def quotients(x, block_rows):
    """448 x / max |x| of the blocks, in 64 bits: a quotient that is a tie has few digits and is exact, and those that are none are further from one
    than 64 bits round."""
    rows, width = x.shape
    R, C = -(-rows // block_rows), -(-width // 128)
    held = torch.zeros(R * block_rows, C * 128, dtype=torch.float64, device=x.device)
    held[:rows, :width] = x.double().abs()
    top = held.reshape(R, block_rows, C, 128).amax(dim=(1, 3)).clamp_min(448 * 2.0 ** -126)
    return 448 * x.double() / top.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :width]


@pytest.mark.parametrize("block_rows", (1, 128))
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
@pytest.mark.parametrize("rows, width, first", ((500, 1312, 0), (300, 1501, 0), (300, 1502, 2), (300, 1500, 4), (300, 1000, 1)))
def test_ties_of_random_values(rows, width, first, dtype, block_rows):
    g = torch.Generator(device="cuda").manual_seed(rows + width)
    held = torch.randn(rows, width + first, generator=g, device="cuda") * torch.exp(0.5 * torch.randn(1, width + first, generator=g, device="cuda"))
    x = held.bfloat16().to(dtype)[:, first:]
    v = quotients(x, block_rows)
    q, _ = pkg.fp8_quantize(x, block_rows=block_rows)
    assert torch.equal(q.double(), nearest_even(v))


@pytest.mark.parametrize("block_rows", (1, 128))
@pytest.mark.parametrize("scale", (0, 60, -60, 118, -90))
def test_ties_of_every_largest_value(scale, block_rows):
    """Blocks whose largest value is each of the 128 of a power of two, with every odd quotient (17 .. 31) / 2^k that bf16 holds beside it."""
    tops = torch.arange(128, 256, dtype=torch.float64)
    x = torch.zeros(128, 128, dtype=torch.float64)
    seen = 0
    for i, top in enumerate(tops.tolist()):
        x[i, 0] = top
        at = 1
        for odd in range(17, 32, 2):                    # 448 x / top = odd / 2^k: halfway between two e4m3 values
            v = odd * top / 448
            for k in range(-8, 9):
                y = v * 2.0 ** k
                if at < 128 and y <= top and float(torch.tensor(y, dtype=torch.bfloat16)) == y:
                    x[i, at] = y if at % 2 else -y
                    at += 1
                    seen += 1
    assert seen > 500
    x = x.cuda() * 2.0 ** scale
    assert torch.equal(x.bfloat16().double(), x)
    if block_rows == 128:
        x = torch.cat([torch.nn.functional.pad(row[None], (0, 0, 0, 127)) for row in x])
    for dtype in (torch.bfloat16, torch.float32):
        q, _ = pkg.fp8_quantize(x.to(dtype), block_rows=block_rows)
        assert torch.equal(q.double(), nearest_even(quotients(x, block_rows)))
