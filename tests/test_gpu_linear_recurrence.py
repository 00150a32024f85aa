"""linear_recurrence and its gradients against step-by-step evaluation in 64 bits (needs a B200)."""
import itertools
import random

import pytest
import torch

import operator_util as ref
import paper_1901_10997_b200 as pkg

pytestmark = pytest.mark.gpu

# one step, less than a segment of 16, segments and CTAs that end anywhere; channels off every vector; clusters of every size
SHAPES = [(1, 1, 1), (1, 16, 1500), (2, 3, 7), (15, 2, 33), (16, 1, 2), (17, 2, 34), (63, 3, 5), (64, 1, 64), (65, 2, 130), (129, 1, 257),
          (257, 2, 32), (400, 16, 80), (700, 1, 100), (1023, 1, 31), (1025, 2, 48), (2049, 1, 50), (4097, 1, 66), (5000, 1, 37), (35, 20, 200),
          (33, 40, 1500), (3, 700, 66)]
# many channels: vectors of four, two and one, rounds of 16, 32 and 64 steps that end anywhere
SHAPES += [(1, 100, 600), (15, 80, 500), (16, 64, 640), (17, 50, 900), (47, 100, 400), (64, 40, 1000), (65, 30, 2000), (200, 60, 700),
           (1, 80, 302), (31, 40, 602), (33, 100, 230), (129, 40, 602), (1, 30, 301), (16, 40, 151), (63, 20, 301), (65, 9, 701), (130, 20, 301)]
# few channels and many steps: chunks of time side by side
CHUNKED = [(8200, 1, 1000), (4100, 2, 1002), (2100, 5, 801)]
MODES = list(itertools.product(("bf16", "fp32"), (True, False), (False, True), (False, True), ("plain", "fused", "batch_first")))


def cases():
    r = random.Random(11)
    for shape in SHAPES:
        for mode in r.sample(MODES, 5):
            yield (*shape, *mode)
    for shape in CHUNKED:
        for mode in (("bf16", True, True, True, "fused"), ("fp32", False, False, True, "plain"), ("bf16", True, False, False, "batch_first")):
            yield (*shape, *mode)


def make(T, B, D, dtype, gate, ragged, layout, seed=0):
    g = torch.Generator(device="cuda").manual_seed(1000 * seed + T + B + D)
    dt = ref.TYPES[dtype]
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    logits = 2 + 2 * n(T, B, D)
    first = logits if gate else torch.sigmoid(logits) * torch.sign(n(T, B, D) + 1.5)
    x, dh = n(T, B, D), n(T, B, D)
    if layout == "fused":
        z = torch.cat([first, x], 2).to(dt)
        a, x = z[..., :D], z[..., D:]
    elif layout == "batch_first":
        a, x = (t.transpose(0, 1).contiguous().to(dt).transpose(0, 1) for t in (first, x))
    else:
        a, x = first.to(dt), x.to(dt)
    lengths = None
    if ragged:
        lengths = torch.randint(0, T + 1, (B,), generator=g, device="cuda", dtype=torch.int32)
        lengths[0] = T
        if B > 1:
            lengths[-1] = 0
    return a, x, n(B, D), lengths, dh.to(dt), n(B, D)


def check_forward(a, x, h0, lengths, gate, reverse, got, what=""):
    h, hT, states = got
    want, last, before, M, W, WT = ref.recurrence(a, x, h0, lengths, gate, reverse)
    e = ref.step_error(a, gate, a.dtype)
    ref.close(h, want, ref.half_step(a.dtype) * want.abs() + e * W, what + " h")
    ref.close(hT, last, e * WT, what + " hT")
    T, B, D = a.shape
    if states is not None:
        lens = torch.full((B,), T, device="cuda") if lengths is None else lengths.clamp(0, T)
        for k in range(states.shape[0]):
            for b in range(B):
                n = int(lens[b])
                if 16 * k >= n:
                    s, w = last[b], WT[b]
                else:
                    t = n - 1 - 16 * k if reverse else 16 * k
                    s, w = before[t, b], W[t, b] * 2 + before[t, b].abs() + (WT[b] if n else 0)
                ref.close(states[k, b], s, e * (w + WT[b] + s.abs()), f"{what} state {k} of {b}")
    return before, W, e


@pytest.mark.parametrize("c", list(cases()), ids=lambda c: "_".join(str(v) for v in c))
def test_against_every_step_in_64_bits(c):
    T, B, D, dtype, gate, reverse, ragged, layout = c
    a, x, h0, lengths, dh, dhT = make(T, B, D, dtype, gate, ragged, layout)
    got = pkg.linear_recurrence(a, x, h0, lengths, gate=gate, reverse=reverse, save=True)
    small = got if B * got[2].shape[0] <= 600 else (got[0], got[1], None)
    before, W, e = check_forward(a, x, h0, lengths, gate, reverse, small)
    da, dx, dh0 = pkg.linear_recurrence_backward(a, x, got[2], dh, dhT, lengths, gate=gate, reverse=reverse)
    # W of the state in front of a step: that behind it bounds it where the step does not forget all
    Wb = torch.zeros_like(W)
    run = h0.double().abs()
    lens = torch.full((B,), T, device="cuda") if lengths is None else lengths
    for t in (range(T - 1, -1, -1) if reverse else range(T)):
        Wb[t] = run
        run = torch.where((t < lens)[:, None], W[t], run)
    wa, wx, w0, ea, ex, e0 = ref.recurrence_backward(a, x, before, Wb, dh, dhT, lengths, gate, reverse, e)
    half = ref.half_step(a.dtype)
    ref.close(da, wa, half * wa.abs() + ea, "da")
    ref.close(dx, wx, half * wx.abs() + ex, "dx")
    ref.close(dh0, w0, e0, "dh0")


@pytest.mark.parametrize("gate", (True, False))
@pytest.mark.parametrize("reverse", (False, True))
def test_gradients_against_differences(gate, reverse):
    T, B, D = 37, 2, 6
    a, x, h0, lengths, dh, dhT = make(T, B, D, "fp32", gate, True, "plain", 3)
    _, _, states = pkg.linear_recurrence(a, x, h0, lengths, gate=gate, reverse=reverse, save=True)
    got = pkg.linear_recurrence_backward(a, x, states, dh, dhT, lengths, gate=gate, reverse=reverse)

    def loss(a, x, h0):
        h, hT, *_ = ref.recurrence(a, x, h0, lengths, gate, reverse)
        return float((h * dh.double()).sum() + (hT * dhT.double()).sum())

    args = [a.double(), x.double(), h0.double()]
    g = torch.Generator(device="cuda").manual_seed(5)
    step = 1e-5
    for i, grad in enumerate(got):
        v = torch.randn(args[i].shape, generator=g, device="cuda", dtype=torch.float64)
        up, down = list(args), list(args)
        up[i], down[i] = args[i] + step * v, args[i] - step * v
        slope, mine = (loss(*up) - loss(*down)) / (2 * step), float((grad.double() * v).sum())
        # the difference is off by step^2 / 6 of a third derivative of the size of the terms, and 2^-53 / step of the loss
        scale = float((grad.double() * v).abs().sum()) + 1
        assert abs(slope - mine) <= 1e-6 * scale, (i, slope, mine)


@pytest.mark.parametrize("dtype", ("bf16", "fp32"))
@pytest.mark.parametrize("reverse", (False, True))
def test_what_lies_behind_a_sequence_is_not_used(dtype, reverse):
    T, B, D = 70, 4, 24
    a, x, h0, _, dh, dhT = make(T, B, D, dtype, True, False, "plain", 4)
    lengths = torch.tensor([70, 33, 0, 16], dtype=torch.int32, device="cuda")
    behind = torch.arange(T, device="cuda")[:, None] >= lengths
    clean = pkg.linear_recurrence(a, x, h0, lengths, reverse=reverse, save=True)
    grads = pkg.linear_recurrence_backward(a, x, clean[2], dh, dhT, lengths, reverse=reverse)
    for bad in (float("nan"), float("inf"), torch.finfo(a.dtype).min):
        a2, x2, d2 = (torch.where(behind[:, :, None], torch.full_like(t, bad), t) for t in (a, x, dh))
        again = pkg.linear_recurrence(a2, x2, h0, lengths, reverse=reverse, save=True)
        assert all(torch.equal(p, q) for p, q in zip(clean, again))
        assert all(torch.equal(p, q) for p, q in zip(grads, pkg.linear_recurrence_backward(a2, x2, again[2], d2, dhT, lengths, reverse=reverse)))
    assert not clean[0][behind].any() and not grads[0][behind].any() and not grads[1][behind].any()
    assert torch.equal(clean[1][2], h0[2]) and torch.equal(grads[2][2], dhT[2])


def test_lengths_outside_the_batch_are_held_to_it():
    a, x, h0, *_ = make(20, 3, 8, "fp32", True, False, "plain", 5)
    odd = torch.tensor([-5, 1 << 30, 7], dtype=torch.int32, device="cuda")
    even = torch.tensor([0, 20, 7], dtype=torch.int32, device="cuda")
    for p, q in zip(pkg.linear_recurrence(a, x, h0, odd, save=True), pkg.linear_recurrence(a, x, h0, even, save=True)):
        assert torch.equal(p, q)


@pytest.mark.parametrize("dtype", ("bf16", "fp32"))
def test_gates_at_their_ends(dtype):
    """Gates that are shut or open altogether: a state is kept to the bit, or replaced."""
    T, B, D = 50, 1, 8
    x = torch.randn(T, B, D, device="cuda").to(ref.TYPES[dtype])
    h0 = torch.randn(B, D, device="cuda")
    low = torch.finfo(x.dtype).min
    for keep in (float("inf"), -low):
        h, hT, _ = pkg.linear_recurrence(torch.full_like(x, keep), x, h0)
        assert torch.equal(hT, h0) and torch.equal(h, h0.to(x.dtype).expand_as(h))
    for drop in (float("-inf"), low):
        h, hT, _ = pkg.linear_recurrence(torch.full_like(x, drop), x, h0)
        assert torch.equal(h, x) and torch.equal(hT, x[-1].float())
    for keep in (float("inf"), float("-inf")):
        a = torch.full_like(x, keep)
        _, _, s = pkg.linear_recurrence(a, x, h0, save=True)
        da, dx, dh0 = pkg.linear_recurrence_backward(a, x, s, torch.ones_like(x))
        assert not da.any()
        assert torch.equal(dx, torch.zeros_like(x) if keep > 0 else torch.ones_like(x))
        assert torch.equal(dh0, torch.full_like(h0, T) if keep > 0 else torch.zeros_like(h0))


def test_nan_and_infinity_reach_what_comes_after_them_only():
    T, B, D = 300, 1, 6
    a, x, h0, *_ = make(T, B, D, "fp32", True, False, "plain", 6)
    want = pkg.linear_recurrence(a, x, h0)[0]
    for bad in (float("nan"), float("inf")):
        x2 = x.clone()
        x2[150, 0, 3] = bad
        h, hT, _ = pkg.linear_recurrence(a, x2, h0)
        assert torch.equal(h[:150], want[:150]) and torch.equal(h[:, :, :3], want[:, :, :3]) and torch.equal(h[:, :, 4:], want[:, :, 4:])
        assert not h[150:, 0, 3].isfinite().any() and not hT[0, 3].isfinite()


def test_decays_of_zero_one_and_above():
    T, D = 3000, 4
    x = torch.randint(-4, 5, (T, 1, D), device="cuda").float()
    h, hT, _ = pkg.linear_recurrence(torch.ones_like(x), x, gate=False)
    assert torch.equal(h, x.cumsum(0)) and torch.equal(hT, x.sum(0))          # whole numbers: exact in any order
    h, _, _ = pkg.linear_recurrence(torch.zeros_like(x), x, torch.full((1, D), 7.0, device="cuda"), gate=False)
    assert torch.equal(h, x)
    # a state of zero stays zero under growth that passes the range of fp32 between segments
    big = torch.full((400, 1, D), 2.0, device="cuda")
    h, hT, _ = pkg.linear_recurrence(big, torch.zeros_like(big), gate=False)
    assert not h.any() and not hT.any()


@pytest.mark.parametrize("T", (0, 1, 5, 100))
def test_state_in_place_and_missing_state(T):
    B, D = 3, 10
    a, x, h0, *_ = make(max(T, 1), B, D, "bf16", True, False, "fused", 7)
    a, x = a[:T], x[:T]
    want = pkg.linear_recurrence(a, x, h0)
    state = h0.clone()
    got = pkg.linear_recurrence(a, x, state, state=state)
    assert got[1] is state and torch.equal(want[0], got[0]) and torch.equal(want[1], state)
    if T == 0:
        assert torch.equal(state, h0)
        da, dx, dh0 = pkg.linear_recurrence_backward(a, x, torch.empty(0, B, D, device="cuda"), torch.empty_like(a), h0)
        assert da.shape == a.shape and torch.equal(dh0, h0)
    zero = pkg.linear_recurrence(a, x, torch.zeros_like(h0))
    assert all(torch.equal(p, q) for p, q in zip(zero[:2], pkg.linear_recurrence(a, x)[:2]))


@pytest.mark.parametrize("T, B, D", ((4100, 2, 1000), (300, 40, 602), (600, 1, 64)))
def test_states_and_their_gradients_in_place(T, B, D):
    """The final state over the initial one where many CTAs read it: chunks of time, many channels, a cluster."""
    a, x, h0, _, dh, dhT = make(T, B, D, "bf16", True, False, "fused", 13)
    want = pkg.linear_recurrence(a, x, h0, save=True)
    grads = pkg.linear_recurrence_backward(a, x, want[2], dh, dhT)
    for _ in range(5):
        state = h0.clone()
        h, _, _ = pkg.linear_recurrence(a, x, state, state=state)
        assert torch.equal(h, want[0]) and torch.equal(state, want[1])
        need = pkg.lstm_linear_recurrence_workspace(T, B, D)
        work, g, da, dx = torch.empty(max(need, 1), device="cuda"), dhT.clone(), torch.empty_like(h), torch.empty_like(h)
        rc, why = pkg.lstm_linear_recurrence_backward(a.data_ptr(), a.stride(0), a.stride(1), x.data_ptr(), x.stride(0), x.stride(1), want[2].data_ptr(),
                                                      dh.data_ptr(), dh.stride(0), dh.stride(1), g.data_ptr(), 0, T, B, D, pkg.LSTM_BF16, pkg.LSTM_LINREC_GATE,
                                                      da.data_ptr(), B * D, D, dx.data_ptr(), B * D, D, g.data_ptr(), work.data_ptr(), need,
                                                      torch.cuda.current_stream().cuda_stream)
        assert rc == pkg.LSTM_OK, why
        assert all(torch.equal(p, q) for p, q in zip((da, dx, g), grads))


def test_chunks_carry_the_state():
    T, B, D = 500, 2, 40
    a, x, h0, *_ = make(T, B, D, "fp32", True, False, "fused", 8)
    want, last, *_, M, W, WT = ref.recurrence(a, x, h0, None, True, False)
    e = ref.step_error(a, True, a.dtype)
    state, at = h0.clone(), 0
    for n in (1, 16, 17, 200, 266):
        h, _, _ = pkg.linear_recurrence(a[at:at + n], x[at:at + n], state, state=state)
        ref.close(h, want[at:at + n], ref.U * want[at:at + n].abs() + e * W[at:at + n], f"chunk at {at}")
        at += n
    ref.close(state, last, e * WT, "state")


def test_outputs_of_other_layouts_and_rows_beside_them():
    T, B, D = 40, 3, 18
    a, x, h0, *_ = make(T, B, D, "bf16", True, False, "plain", 9)
    want = pkg.linear_recurrence(a, x, h0)[0]
    held = torch.full((B + 1, T + 2, D + 6), 5.0, dtype=torch.bfloat16, device="cuda")
    out = held[:B, 1:T + 1, 3:D + 3].transpose(0, 1)
    pkg.linear_recurrence(a, x, h0, out=out)
    assert torch.equal(out, want)
    out.fill_(5.0)
    assert bool((held == 5.0).all())


@pytest.mark.parametrize("T, B, D", ((30, 4, 24), (40, 40, 600), (4100, 2, 1000)))
def test_broadcast_inputs(T, B, D):
    """Decays of a channel for all steps and sequences, inputs of one sequence for all: strides of zero."""
    a = torch.rand(D, device="cuda").expand(T, B, D)
    x = torch.randn(T, 1, D, device="cuda").expand(T, B, D)
    dh = torch.randn(D, device="cuda").expand(T, B, D)
    got = pkg.linear_recurrence(a, x, gate=False, save=True)
    want = pkg.linear_recurrence(a.contiguous(), x.contiguous(), gate=False, save=True)
    assert all(torch.equal(p, q) for p, q in zip(got, want))
    for p, q in zip(pkg.linear_recurrence_backward(a, x, got[2], dh, gate=False), pkg.linear_recurrence_backward(a.contiguous(), x.contiguous(), want[2], dh.contiguous(), gate=False)):
        assert torch.equal(p, q)


def test_offsets_beyond_32_bits():
    """Steps a gigabyte apart: element offsets pass 2^31."""
    D, far = 64, (1 << 30) + 8
    held = torch.empty(2 * far + 4096, dtype=torch.bfloat16, device="cuda")
    a0, x0, h0, _, dh0, dhT = make(3, 1, D, "bf16", True, False, "plain", 10)
    put = lambda t, at: held.as_strided((3, 1, D), (far, D, 1), at).copy_(t)
    a, x, dh, out = put(a0, 0), put(x0, 512), put(dh0, 1024), held.as_strided((3, 1, D), (far, D, 1), 2048)
    want = pkg.linear_recurrence(a0, x0, h0, save=True)
    got = pkg.linear_recurrence(a, x, h0, save=True, out=out)
    assert all(torch.equal(p, q) for p, q in zip(want, got))
    for p, q in zip(pkg.linear_recurrence_backward(a0, x0, want[2], dh0, dhT), pkg.linear_recurrence_backward(a, x, got[2], dh, dhT)):
        assert torch.equal(p, q)


@pytest.mark.parametrize("shape", ((900, 2, 64), (40, 40, 600), (4100, 2, 1000)), ids=str)
def test_recorded_and_on_two_streams(shape):
    """Calls keep nothing: recorded twice, replayed beside ordinary calls on another stream, all give the same bits."""
    sets = [make(*shape, "bf16", True, True, "fused", s) for s in (11, 12)]

    def both(s):
        a, x, h0, lengths, dh, dhT = s
        h, hT, states = pkg.linear_recurrence(a, x, h0, lengths, save=True)
        return (h, hT, states, *pkg.linear_recurrence_backward(a, x, states, dh, dhT, lengths))

    want = [both(s) for s in sets]
    graphs, outs = [], []
    for s in sets:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            outs.append(both(s))
        graphs.append(g)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    for _ in range(3):
        for g, o in zip(graphs, outs):
            for t in o:
                t.zero_()
        side.wait_stream(torch.cuda.current_stream())
        with torch.cuda.stream(side):
            graphs[0].replay()
            other = both(sets[0])
        graphs[1].replay()
        here = both(sets[1])
        torch.cuda.synchronize()
        for got, w in ((outs[0], want[0]), (outs[1], want[1]), (other, want[0]), (here, want[1])):
            assert all(torch.equal(p, q) for p, q in zip(got, w))


def test_a_workspace_that_is_too_small_is_refused():
    assert all(pkg.lstm_linear_recurrence_workspace(*shape) > 0 for shape in CHUNKED)
    T, B, D = CHUNKED[0]
    need = pkg.lstm_linear_recurrence_workspace(T, B, D)
    assert pkg.lstm_linear_recurrence_workspace(1, 4, 100) == 0 and pkg.lstm_linear_recurrence_workspace(-1, 4, 100) == -1
    t = torch.zeros(T, B, D, device="cuda")
    work, h = torch.empty(need, device="cuda"), torch.empty_like(t)
    call = lambda at, n: pkg.lstm_linear_recurrence(t.data_ptr(), D, D, t.data_ptr(), D, D, 0, 0, T, B, D, pkg.LSTM_F32, 1, h.data_ptr(), D, D, 0, 0, at, n,
                                                    torch.cuda.current_stream().cuda_stream)
    assert call(0, need)[0] == pkg.LSTM_ERR_INVALID and call(work.data_ptr(), need - 1)[0] == pkg.LSTM_ERR_INVALID
    assert call(work.data_ptr(), need) == (pkg.LSTM_OK, "")


def test_tensors_that_do_not_fit_are_refused():
    a, x, h0, *_ = make(4, 2, 8, "bf16", True, False, "plain")
    L = torch.tensor([1, 2], device="cuda")
    s = torch.empty(1, 2, 8, device="cuda")
    for bad in (lambda: pkg.linear_recurrence(a, x.float(), h0), lambda: pkg.linear_recurrence(a, x[:3], h0), lambda: pkg.linear_recurrence(a, None, h0),
                lambda: pkg.linear_recurrence(a.half(), x.half(), h0), lambda: pkg.linear_recurrence(a, x, h0.bfloat16()), lambda: pkg.linear_recurrence(a, x, h0, L),
                lambda: pkg.linear_recurrence(a, x, h0[:1]), lambda: pkg.linear_recurrence(a, x, h0, out=a[:1].expand(4, 2, 8)),
                lambda: pkg.linear_recurrence(a, x, h0, out=torch.empty(64, device="cuda", dtype=a.dtype).as_strided((4, 2, 8), (8, 8, 1))),
                lambda: pkg.linear_recurrence(a, x.transpose(1, 2).contiguous().transpose(1, 2), h0), lambda: pkg.linear_recurrence(a, x.cpu(), h0),
                lambda: pkg.linear_recurrence_backward(a, x, s[:, :1], a), lambda: pkg.linear_recurrence_backward(a, x, s, a[:2])):
        with pytest.raises(ValueError):
            bad()
