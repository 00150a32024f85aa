"""The tensor calls record no graph, and say so instead of losing a gradient (needs a B200)."""
import pytest
import torch

import paper_1901_10997_b200 as pkg

pytestmark = pytest.mark.gpu


def calls():
    n = lambda *s: torch.randn(s, device="cuda")
    a, x, h0, w, m = n(5, 2, 16), n(5, 2, 16), n(2, 16), n(16), n(10, 16)
    _, _, states = pkg.linear_recurrence(a, x, h0, save=True)
    qx, sx = pkg.fp8_quantize(m)
    qw, sw = pkg.fp8_quantize(n(24, 16), block_rows=128)
    bias = n(24)
    yield pkg.linear_recurrence, (a, x, h0), (0, 1, 2)
    yield pkg.linear_recurrence_backward, (a, x, states, x, h0), (0, 1, 3, 4)
    yield pkg.rms_norm, (m, w, m.clone()), (0, 1, 2)
    yield pkg.rms_norm_fp8, (m, w, m.clone()), (0, 1, 2)
    yield pkg.rms_norm_backward, (m, m.clone(), w, m.clone()), (0, 1, 2, 3)
    yield pkg.fp8_quantize, (m,), (0,)
    yield pkg.fp8_product, (qx, sx, qw, sw, bias), (1, 3, 4)


def test_tensors_that_require_gradients_are_refused_while_they_are_recorded():
    for call, args, places in calls():
        want = call(*args)
        for i in places:
            with_grad = list(args)
            with_grad[i] = args[i].detach().requires_grad_()
            with pytest.raises(ValueError, match="no graph"):
                call(*with_grad)
            with torch.no_grad():
                got = call(*with_grad)
            with_grad[i] = with_grad[i].detach()
            for again in (got, call(*with_grad)):
                for p, q in zip(*((v if isinstance(v, tuple) else (v,)) for v in (again, want))):
                    assert p is None and q is None or torch.equal(p.float(), q.float()) and not p.requires_grad


def test_outputs_that_require_gradients_are_refused():
    a, x = torch.randn(5, 2, 16, device="cuda"), torch.randn(5, 2, 16, device="cuda")
    with pytest.raises(ValueError, match="no graph"):
        pkg.linear_recurrence(a, x, out=torch.empty_like(a).requires_grad_())
    with pytest.raises(ValueError, match="no graph"):
        pkg.linear_recurrence(a, x, state=torch.zeros(2, 16, device="cuda").requires_grad_())


def test_other_objects_are_refused_as_before():
    n = lambda *s: torch.randn(s, device="cuda")
    a, m, w = n(5, 2, 16), n(4, 16), n(16)
    _, _, states = pkg.linear_recurrence(a, a, save=True)
    q, s = pkg.fp8_quantize(m)
    for bad in (lambda: pkg.linear_recurrence(a, 3), lambda: pkg.linear_recurrence(a, a, "h0"), lambda: pkg.linear_recurrence(a, a, state=3), lambda: pkg.linear_recurrence(a, a, out=3),
                lambda: pkg.linear_recurrence_backward(a, a, states, 3), lambda: pkg.linear_recurrence_backward(a, a, states, a, "dhT"), lambda: pkg.rms_norm(m, 3),
                lambda: pkg.rms_norm(m, w, 3), lambda: pkg.rms_norm_fp8(m, 3), lambda: pkg.rms_norm_backward(m, m, 3), lambda: pkg.rms_norm_backward(m, m, w, 3),
                lambda: pkg.fp8_quantize(3), lambda: pkg.fp8_product(q, 3, q, s), lambda: pkg.fp8_product(q, s, q, s, 3)):
        with pytest.raises(ValueError):
            bad()
