"""The operators as they are used together: a stack of layers norm -> 8-bit projection -> linear recurrence -> residual, whole sequences and
step by step, and a layer's training step (needs a B200)."""
import math

import pytest
import torch

import operator_util as ref
import paper_1901_10997_b200 as pkg

pytestmark = pytest.mark.gpu


def weights(D, layers, seed=0):
    g = torch.Generator(device="cuda").manual_seed(seed)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    out = []
    for _ in range(layers):
        w = n(2 * D, D) / math.sqrt(D)
        bias = torch.cat([torch.full((D,), 2.0, device="cuda"), torch.zeros(D, device="cuda")])
        out.append((1 + 0.1 * n(D), *pkg.fp8_quantize(w, block_rows=128), bias))
    return out


def layer(x, residual, p, state, lengths=None):
    """x, residual [T, B, D] -> (h, the sum that goes on); the state is updated in place."""
    T, B, D = x.shape
    w, qw, sw, bias = p
    q, s, r = pkg.rms_norm_fp8(x.view(T * B, D), w, residual.view(T * B, D))
    z = pkg.fp8_product(q, s, qw, sw, bias, dtype=x.dtype).view(T, B, 2 * D)
    h, _, _ = pkg.linear_recurrence(z[..., :D], z[..., D:], state, lengths, state=state)
    return (q, s, r, z, h), r.view(T, B, D)


def stack(x, params, states, lengths=None):
    residual, seen = torch.zeros_like(x), []
    for p, state in zip(params, states):
        parts, residual = layer(x, residual, p, state, lengths)
        seen.append(parts)
        x = parts[-1]
    return x, residual, seen


@pytest.mark.parametrize("dtype", ("bf16", "fp32"))
@pytest.mark.parametrize("T, B, D", ((1, 4, 200), (35, 20, 200), (90, 3, 333)))
def test_a_stack_each_operator_on_what_the_last_one_made(T, B, D, dtype):
    params = weights(D, 2)
    x = torch.randn(T, B, D, device="cuda").to(ref.TYPES[dtype])
    lengths = torch.arange(T, T - B, -1, device="cuda", dtype=torch.int32).clamp(min=0)
    states = [torch.randn(B, D, device="cuda") for _ in params]
    before = [s.clone() for s in states]
    _, _, seen = stack(x, params, states, lengths)
    residual = torch.zeros_like(x)
    for (w, qw, sw, bias), (q, s, r, z, h), h0, hT in zip(params, seen, before, states):
        total = (x.double() + residual.double()).view(T * B, D)
        ref.close(r, total, (ref.half_step(x.dtype) + ref.U) * total.abs(), "r")
        y = total / torch.sqrt(total.square().mean(1, keepdim=True) + 1e-6) * w.double()
        ref.check_e4m3(q, s, y, 1, 64 * ref.U, "q")
        big = q.double() * ref.spread(s.double(), 1, T * B, D)
        m = qw.double() * ref.spread(sw.double(), 128, 2 * D, D)
        want = (big @ m.t() + bias.double()).view(T, B, 2 * D)
        ref.close(z, want, ref.half_step(x.dtype) * want.abs() + 300 * ref.U * (big.abs() @ m.abs().t() + bias.abs()).view(T, B, 2 * D), "z")
        hw, last, _, _, W, WT = ref.recurrence(z[..., :D], z[..., D:], h0, lengths, True, False)
        e = ref.step_error(z, True, z.dtype)
        ref.close(h, hw, ref.half_step(x.dtype) * hw.abs() + e * W, "h")
        ref.close(hT, last, e * WT, "hT")
        x, residual = h, r.view(T, B, D)


def test_generation_in_a_graph_follows_the_whole_sequence():
    """One step recorded into a graph and replayed: states go on from replay to replay and give the bits of ordinary steps."""
    T, B, D = 12, 4, 200
    params = weights(D, 2, 1)
    xs = torch.randn(T, B, D, device="cuda").bfloat16()
    ordinary = [torch.zeros(B, D, device="cuda") for _ in params]
    want = [stack(xs[t:t + 1], params, ordinary)[0].clone() for t in range(T)]
    states = [torch.zeros(B, D, device="cuda") for _ in params]
    x = torch.zeros(1, B, D, device="cuda", dtype=torch.bfloat16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, _, _ = stack(x, params, states)
    for t in range(T):
        x.copy_(xs[t:t + 1])
        graph.replay()
        assert torch.equal(y, want[t]), t
    assert all(torch.equal(p, q) for p, q in zip(states, ordinary))


def test_a_training_step():
    """norm -> projection (fp32 weights) -> recurrence, its gradients against differentiation of the formulas in 64 bits."""
    T, B, D = 45, 3, 64
    g = torch.Generator(device="cuda").manual_seed(2)
    n = lambda *s: torch.randn(s, generator=g, device="cuda")
    x, residual, w, W, h0 = n(T * B, D), n(T * B, D), 1 + 0.1 * n(D), n(2 * D, D) / math.sqrt(D), n(B, D)
    dh, dr = n(T, B, D), n(T * B, D)
    lengths = torch.tensor([45, 20, 1], dtype=torch.int32, device="cuda")
    y, r = pkg.rms_norm(x, w, residual)
    z = (y @ W.t()).view(T, B, 2 * D)
    h, _, states = pkg.linear_recurrence(z[..., :D], z[..., D:], h0, lengths, save=True)
    da, dz, dh0 = pkg.linear_recurrence_backward(z[..., :D], z[..., D:], states, dh, None, lengths)
    dzz = torch.cat([da, dz], 2).view(T * B, 2 * D)
    dx, dw = pkg.rms_norm_backward(dzz @ W, r, w, dr)
    dW = dzz.t() @ y

    leaves = [t.double().requires_grad_() for t in (x, w, W, h0)]
    r64 = leaves[0] + residual.double()
    y64 = r64 * torch.rsqrt(r64.square().mean(1, keepdim=True) + 1e-6) * leaves[1]
    z64 = (y64 @ leaves[2].t()).view(T, B, 2 * D)
    state, loss = leaves[3], (r64 * dr.double()).sum()
    for t in range(T):
        f = torch.sigmoid(z64[t, :, :D])
        state = torch.where((t < lengths)[:, None], f * state + (1 - f) * z64[t, :, D:], state)
        loss = loss + (torch.where((t < lengths)[:, None], state, 0.0) * dh[t].double()).sum()
    want = torch.autograd.grad(loss, leaves)
    # sums of up to 135 rows and 128 columns and of the recurrence's memory, all in 32 bits: some 1000 roundings of U against the whole
    for got, wanted in zip((dx, dw, dW, dh0), want):
        assert float((got.double() - wanted).norm() / wanted.norm()) <= 1000 * ref.U


FIRST = """
import torch, paper_1901_10997_b200 as pkg
n = lambda *s: torch.randn(s, device="cuda")
x, w, z, z2, dh = n(30, 200).bfloat16(), n(200), n(90, 2, 96).bfloat16(), n(9000, 1, 1000), n(90, 2, 96).bfloat16()
wide, m, states = n(40, 30, 900).bfloat16(), n(400, 200).bfloat16(), n(6, 2, 96)
many = n(9000, 200).bfloat16()
torch.cuda.synchronize()
g = torch.cuda.CUDAGraph()
def run():
    q, s, r = pkg.rms_norm_fp8(x, w, x)
    qw, sw = pkg.fp8_quantize(m, block_rows=128)
    return [pkg.fp8_product(q, s, qw, sw), pkg.fp8_product(*pkg.fp8_quantize(many), qw, sw), *pkg.rms_norm_backward(x, x, w), pkg.linear_recurrence(z, z)[0],
            pkg.linear_recurrence(z2, z2)[0], pkg.linear_recurrence(wide, wide)[0], *pkg.linear_recurrence_backward(z, z, states, dh), s, r]
with torch.cuda.graph(g):
    out = run()
g.replay()
torch.cuda.synchronize()
assert all(torch.equal(p, q) for p, q in zip(out, run()))
print("same")
"""


def test_the_first_call_of_a_process_may_be_a_recorded_one():
    import os
    import subprocess
    import sys
    from pathlib import Path
    root = Path(__file__).resolve().parent.parent
    r = subprocess.run([sys.executable, "-c", FIRST], capture_output=True, text=True, timeout=300, cwd=str(root), env=dict(os.environ, PYTHONPATH=str(root)))
    assert r.returncode == 0 and "same" in r.stdout, r.stderr[-2000:]
