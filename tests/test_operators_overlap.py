"""Outputs that the caller hands to the tensor calls may share no element with an input.  The comparison of strided tensors on the CPU, against
every element; the calls on the GPU."""
import random

import pytest
import torch

import paper_1901_10997_b200 as pkg


def elements(t):
    """The addresses of all bytes of a tensor."""
    at = {t.data_ptr()}
    for n, stride in zip(t.shape, t.stride()):
        at = {p + i * stride * t.element_size() for p in at for i in range(n)}
    return {p + k for p in at for k in range(t.element_size())}


def test_strided_tensors_against_every_element():
    from paper_1901_10997_b200.operators import _apart, _no_input
    r = random.Random(5)
    held, seen = torch.zeros(4096, dtype=torch.uint8), [0, 0]
    while min(seen) < 400:
        views = []
        for _ in range(2):
            dt = r.choice((torch.bfloat16, torch.float32))
            T, B, D = r.randint(1, 4), r.randint(1, 4), r.randint(1, 6)
            if r.random() < 0.5:
                strides = (r.randint(0, 40), r.randint(0, 40), 1)
            else:                       # parts of one matrix
                strides = (r.choice((36, 40, 48)), r.choice((12, 16)), 1)
            views.append(held.view(dt).as_strided((T, B, D), strides, r.randint(0, 120)))
        out, t = views
        try:
            _apart(out, "out")
        except ValueError:
            continue
        share = bool(elements(out) & elements(t))
        try:
            _no_input(out, "out", (None, "h0"), (t, "x"))
            assert not share, (out.shape, out.stride(), out.data_ptr() - t.data_ptr(), t.shape, t.stride())
        except ValueError as e:
            assert share and str(e) == "out overlaps x", (out.shape, out.stride(), out.data_ptr() - t.data_ptr(), t.shape, t.stride())
        seen[share] += 1


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", (torch.bfloat16, torch.float32))
def test_outputs_over_inputs_are_refused(dtype):
    T, B, D = 9, 4, 24
    z = torch.randn(T, B, 3 * D, device="cuda").to(dtype)
    a, x, out = z[..., :D], z[..., D:2 * D], z[..., 2 * D:]
    h0 = torch.randn(B, D, device="cuda")
    want = pkg.linear_recurrence(a, x, h0)
    keep = z.clone()
    more = torch.zeros(2 * B, D, device="cuda")
    lengths = torch.full((B,), T, dtype=torch.int32, device="cuda")
    for bad in (lambda: pkg.linear_recurrence(a, x, h0, out=x), lambda: pkg.linear_recurrence(a, x, h0, out=a), lambda: pkg.linear_recurrence(a, x, h0, out=z[..., D + 1:2 * D + 1]),
                lambda: pkg.linear_recurrence(a[1:], x[1:], h0, out=x[:-1]), lambda: pkg.linear_recurrence(a, x, more[:B], state=more[1:B + 1]),
                lambda: pkg.linear_recurrence(a, x, h0, lengths[:1].expand(B).contiguous(), out="h"), lambda: pkg.linear_recurrence(a, x, h0, out=None, state=more[::2])):
        with pytest.raises(ValueError):
            bad()
    assert torch.equal(z, keep)
    # beside them is well: halves of one matrix, other steps, other sequences, the initial state itself or another view of it
    got = pkg.linear_recurrence(a, x, h0, out=out)
    assert got[0] is out and torch.equal(out, want[0])
    both = torch.zeros(2 * T, B, D, device="cuda", dtype=dtype)
    both[:T] = x
    assert torch.equal(pkg.linear_recurrence(a, both[:T], h0, out=both[T:])[0], want[0])
    wide = torch.zeros(T, 2 * B, D, device="cuda", dtype=dtype)
    wide[:, ::2] = x
    assert torch.equal(pkg.linear_recurrence(a, wide[:, ::2], h0, out=wide[:, 1::2])[0], want[0])
    state = h0.clone()
    assert torch.equal(pkg.linear_recurrence(a, x, state.view(B, D), state=state)[1], want[1])
    state = torch.cat([h0, h0])
    assert torch.equal(pkg.linear_recurrence(a, x, state[:B], state=state[B:])[1], want[1]) and torch.equal(state[:B], h0)


@pytest.mark.gpu
def test_a_final_state_over_inputs_and_outputs_is_refused():
    T, B, D = 6, 3, 16
    a, x, out = (torch.randn(T, B, D, device="cuda") for _ in range(3))
    for bad in (lambda: pkg.linear_recurrence(a, x, state=x[-1]), lambda: pkg.linear_recurrence(a, x, state=a[0]), lambda: pkg.linear_recurrence(a, x, out=out, state=out[-1])):
        with pytest.raises(ValueError):
            bad()


@pytest.mark.gpu
def test_a_product_over_its_operands_is_refused():
    qx, sx = pkg.fp8_quantize(torch.randn(8, 32, device="cuda"))
    qw, sw = pkg.fp8_quantize(torch.randn(16, 32, device="cuda"), block_rows=128)
    over = qx.view(torch.uint8).view(torch.bfloat16)                # [8, 16] on the bytes of qx
    bias = torch.randn(16 * 8, device="cuda")
    for bad in (lambda: pkg.fp8_product(qx, sx, qw, sw, out=over), lambda: pkg.fp8_product(qx, sx, qw, sw, bias[:16], dtype=torch.float32, out=bias.view(8, 16)),
                lambda: pkg.fp8_product(qx, sx, qw, sw, out="y")):
        with pytest.raises(ValueError):
            bad()
    out = torch.empty(8, 16, device="cuda", dtype=torch.bfloat16)
    assert torch.equal(pkg.fp8_product(qx, sx, qw, sw, out=out), pkg.fp8_product(qx, sx, qw, sw))
