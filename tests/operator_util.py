"""References in 64 bits for the stateless operators, written step by step, with the error that arithmetic in 32 bits may have.

U = 2^-24 is half a step of fp32 relative to the value; a result rounded to type t adds torch.finfo(t).eps / 2 of itself."""
import torch

U = 2.0 ** -24
TYPES = {"bf16": torch.bfloat16, "fp32": torch.float32}
TINY = 1e-36          # what falls below the normal range of fp32


def half_step(dtype):
    return torch.finfo(dtype).eps / 2


def close(got, want, bound, what=""):
    """|got - want| <= bound element by element, non-finite values equal."""
    got, want = got.double(), want.double()
    assert got.shape == want.shape, (what, got.shape, want.shape)
    fine = want.isfinite()
    assert torch.equal(got.isfinite(), fine), f"{what}: finite where it should not be, or not where it should"
    assert torch.equal(got.isnan(), want.isnan()), f"{what}: NaN"
    off = torch.where(fine, (got - want).abs(), 0.0)
    allowed = torch.where(fine, bound + TINY, 1.0).expand_as(off)
    worst = (off / allowed).max() if off.numel() else torch.tensor(0.0)
    at = tuple(int(i) for i in torch.unravel_index((off / allowed).argmax(), off.shape)) if off.numel() else ()
    assert worst <= 1, f"{what}: off by {float(worst):.3g} times what may be, at {at}: {float(got[at]):.9g} for {float(want[at]):.9g}"


# ---------------------------------------------------------------- recurrence
def step_error(a, gate, dtype):
    """Relative error of one step's f and b in 32 bits.  expf is off by 2 units in the last place (4 U), the fast exponential of bf16
    data by 2 (and 2^-22 of rounding inside) and by the rounding of its argument |u| log2(e), 2 |u| U; then a sum, a quotient of 2 units, two
    products, the fma of a pass and the product of decays."""
    if not gate:
        return 4 * U
    largest = float(a.abs().clamp(max=90).max()) if a.numel() else 0.0
    return (4 + 1 + 4 + 1 + 1 + 1 + 1 + 1 + (8 + 2 * largest if dtype == torch.bfloat16 else 0)) * U


def recurrence(a, x, h0, lengths, gate, reverse):
    """(h, hT, before, M, W): every step in 64 bits, time in the order of the tensors; M the sum of the terms' magnitudes, W that sum with each term
    as often as it has passed a step (an error of e a step makes an error of e W)."""
    T, B, D = a.shape
    dev = a.device
    a, x = a.double(), x.double()
    f = torch.sigmoid(a) if gate else a
    b = torch.sigmoid(-a) * x if gate else x
    lens = torch.full((B,), T, device=dev) if lengths is None else lengths.clamp(0, T)
    h = torch.zeros(B, D, dtype=torch.float64, device=dev) if h0 is None else h0.double()
    M, W = h.abs(), h.abs()
    out = {k: torch.zeros(T, B, D, dtype=torch.float64, device=dev) for k in ("h", "before", "M", "W")}
    for t in (range(T - 1, -1, -1) if reverse else range(T)):
        live = (t < lens)[:, None]
        out["before"][t] = h
        M2 = f[t].abs() * M + b[t].abs()
        h, W, M = (torch.where(live, new, old) for new, old in ((f[t] * h + b[t], h), (f[t].abs() * W + M2, W), (M2, M)))
        for k, v in (("h", h), ("M", M), ("W", W)):
            out[k][t] = torch.where(live, v, 0.0)
    return out["h"], h, out["before"], out["M"], out["W"], W


def recurrence_backward(a, x, before, W, dh, dhT, lengths, gate, reverse, e):
    """(da, dx, dh0) and the error each may have, with e the relative error of a step."""
    T, B, D = a.shape
    dev = a.device
    a, x, dh = a.double(), x.double(), dh.double()
    f, w = (torch.sigmoid(a), torch.sigmoid(-a)) if gate else (a, torch.ones_like(a))
    lens = torch.full((B,), T, device=dev) if lengths is None else lengths.clamp(0, T)
    q = torch.zeros(B, D, dtype=torch.float64, device=dev) if dhT is None else dhT.double()
    Mq, Wq = q.abs(), q.abs()
    da, dx, eda, edx = (torch.zeros(T, B, D, dtype=torch.float64, device=dev) for _ in range(4))
    for t in (range(T) if reverse else range(T - 1, -1, -1)):
        live = (t < lens)[:, None]
        g, Mg = dh[t] + q, dh[t].abs() + Mq
        eg = e * Wq + 2 * U * Mg                    # the error of g
        u = (before[t] - x[t]) * f[t] * w[t] if gate else before[t]
        # W holds |h| and more; the error of h - x is that of h and one rounding
        eu = (e * W[t] + U * (before[t].abs() + x[t].abs()) + 3 * e * (before[t] - x[t]).abs()) * (f[t] * w[t]) if gate else e * W[t]
        for o, v in ((da, g * u), (dx, g * w[t]), (eda, eg * u.abs() + g.abs() * eu + eg * eu + 2 * U * (g * u).abs()),
                     (edx, (eg + (e + 2 * U) * g.abs()) * w[t])):
            o[t] = torch.where(live, v, 0.0)
        q, Wq, Mq = (torch.where(live, new, old) for new, old in
                     ((f[t] * g, q), (f[t].abs() * (Wq + dh[t].abs() + Mg), Wq), (f[t].abs() * Mg, Mq)))
    return da, dx, q, eda, edx, 2 * e * Wq + 2 * U * Mq


# ---------------------------------------------------------------- 8 bits
def e4m3_values():
    v = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double()
    return v[v.isfinite()].unique()


def spread(scales, block_rows, rows, width):
    """Each element's scale."""
    return scales.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :width]


def check_e4m3(q, scales, y, block_rows, e, what=""):
    """q, scales stand for y (64 bits), of which the library had a version with relative error e: scales from the largest magnitudes, q the
    nearest of the values of e4m3."""
    rows, width = y.shape
    assert q.shape == y.shape and q.dtype == torch.float8_e4m3fn
    R, C = -(-rows // block_rows), -(-width // 128)
    held = torch.zeros(R * block_rows, C * 128, dtype=torch.float64, device=y.device)
    held[:rows, :width] = y.abs()
    top = held.reshape(R, block_rows, C, 128).amax(dim=(1, 3)).clamp_min(448 * 2.0 ** -126) / 448
    close(scales, top, top * (e + 2 * U), what + " scales")
    v = y / spread(scales.double(), block_rows, rows, width)
    grid = e4m3_values().to(y.device)
    at = torch.searchsorted(grid, v.contiguous()).clamp(1, len(grid) - 1)
    nearest = torch.minimum((v - grid[at - 1]).abs(), (v - grid[at]).abs())
    # a reciprocal, a product and the error of y lie between v and what was rounded
    fuzz = v.abs() * (e + 4 * U)
    off = (q.double() - v).abs()
    assert bool((off <= nearest + 2 * fuzz + TINY).all()), f"{what}: q is not the nearest value"
