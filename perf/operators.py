"""Operators of stacks of gated linear recurrences with 8-bit projections, as cases that can be timed and compared.

A layer of such a stack normalises its input (with the residual's addition), multiplies it by 8-bit weights and runs the
two halves of the product, gate logits and candidates, through a recurrence that is linear in its state:

  recurrence      f_t = sigmoid(a_t) (gate) or a_t (decay);  h_t = f_t h_{t-1} + (1 - f_t) x_t  or  + x_t; backward too
  norm            r = x + residual;  y = r / sqrt(mean(r^2) + eps) * w, in the inputs' type or in 8 bits with a scale for each
                  128 columns of a row; backward too
  quantize        8-bit values with a scale for each 128 columns of a row, or for each 128 x 128 block
  product         y = x w^T + b of such 8-bit matrices

``own`` false: the definitions in elementary torch operations; true: the library's calls.  Sizes are those of this
repository's language model (widths 1500, 200; 35 steps, 20 sequences) and speech model (800 units a direction, inputs
of 1312 and 1600, 400 steps), and ragged ones between and around them.
"""
import math

import torch

own = False

EPS = 1e-6
E4M3_MAX = 448.0
FLT_MIN = 2.0 ** -126
SEGMENT = 16          # steps between two saved states


def _recur(name, T, B, D, *, dtype="bf16", gate=True, reverse=False, ragged=False, fused=True, save=False, back=False):
    c = {"op": "recurrence_backward" if back else "recurrence", "T": T, "B": B, "D": D, "dtype": dtype, "gate": gate,
         "reverse": reverse, "ragged": ragged, "fused": fused, "save": save}
    return c | ({"name": name} if name else {})


def _norm(name, rows, width, *, dtype="bf16", residual=True, bits8=False, back=False):
    c = {"op": "norm_backward" if back else "norm", "rows": rows, "width": width, "dtype": dtype, "residual": residual, "bits8": bits8}
    return c | ({"name": name} if name else {})


def _quant(name, rows, width, *, dtype="bf16", block_rows=1):
    c = {"op": "quantize", "rows": rows, "width": width, "dtype": dtype, "block_rows": block_rows}
    return c | ({"name": name} if name else {})


def _product(name, rows, outs, width, *, dtype="bf16", bias=True):
    c = {"op": "product", "rows": rows, "outs": outs, "width": width, "dtype": dtype, "bias": bias}
    return c | ({"name": name} if name else {})


def listed():
    return [
        # generation: one step of 16 sequences, the state carried; gates and candidates are halves of one projection
        _recur("recurrence_step", 1, 16, 1500),
        # the backward direction of a speech layer on utterances of different lengths, in full fp32
        _recur("recurrence_speech", 400, 16, 800, dtype="fp32", reverse=True, ragged=True),
        # one document of 65536 tokens read at once
        _recur("recurrence_long", 65536, 1, 1500),
        # a training batch of utterances: gradients from the saved states
        _recur("recurrence_back", 400, 64, 800, ragged=True, back=True),
        # generation: the norm of 16 rows, in 8 bits for the projection behind it
        _norm("norm_step", 16, 1500, bits8=True),
        # 64 utterances of 400 frames, both directions' outputs side by side
        _norm("norm_bulk", 25600, 1600, bits8=True),
        # the norm's gradients in a training batch
        _norm("norm_back", 25600, 1500, back=True),
        # a layer's weights, laid out when a model is loaded
        _quant("quantize_weights", 6000, 1500, dtype="fp32", block_rows=128),
        # spectrogram frames on their way into the first projection
        _quant("quantize_frames", 25600, 1312),
        # generation: four gates of 1500 units for one sequence
        _product("product_step", 1, 6000, 1500),
        # the language model at its usual batch: 20 sentences of 35 words
        _product("product_batch", 700, 6000, 1500, dtype="fp32"),
        # 64 utterances of 400 frames through a bidirectional layer's gates
        _product("product_bulk", 25600, 6400, 1600),
    ]


def draw(rng):
    def log_int(lo, hi):
        return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))

    kind = rng.choice(["recurrence", "recurrence", "recurrence_backward", "norm", "norm_backward", "quantize", "product", "product"])
    dtype = rng.choice(["bf16", "bf16", "fp32"])
    if kind.startswith("recurrence"):
        back = kind == "recurrence_backward"
        T, D = log_int(1, 65536), log_int(100, 2048)
        most = 98_000_000 // (2 if dtype == "fp32" or back else 1)
        B = max(1, min(log_int(1, 64), most // (T * D)))
        T = min(T, most // D)
        return _recur("", T, B, D, dtype=dtype, gate=rng.random() < 0.7, reverse=rng.random() < 0.4, ragged=rng.random() < 0.4,
                      fused=rng.random() < 0.6, save=rng.random() < 0.3, back=back)
    if kind == "product":
        outs, width = log_int(200, 8192), log_int(100, 8192)
        rows = max(1, min(log_int(1, 25600), 25600 * 6400 * 1600 // (outs * width)))
        return _product("", rows, outs, width, dtype=dtype, bias=rng.random() < 0.5)
    width = log_int(100, 8192)
    rows = max(1, min(log_int(1, 25600), 40_000_000 // width // (2 if dtype == "fp32" else 1)))
    if kind == "quantize":
        return _quant("", rows, width, dtype=dtype, block_rows=rng.choice([1, 128]))
    return _norm("", rows, width, dtype=dtype, residual=rng.random() < 0.6, bits8=kind == "norm" and rng.random() < 0.6, back=kind == "norm_backward")


def _type(c):
    return {"bf16": torch.bfloat16, "fp32": torch.float32}[c["dtype"]]


def _lengths(c):
    """Lengths of a ragged batch: from T down to about half of it."""
    T, B = c["T"], c["B"]
    return [T - (b * T) // (2 * B) for b in range(B)] if c["ragged"] else [T] * B


# ---------------------------------------------------------------- inputs
def _pad16(q):
    """8-bit rows as the product takes them: a multiple of 16 bytes apart."""
    rows, width = q.shape
    held = torch.zeros((rows, -(-width // 16) * 16), dtype=torch.uint8, device=q.device).view(torch.float8_e4m3fn)
    held[:, :width] = q
    return held[:, :width]


def prepare(case, seed):
    c = case
    dev = torch.device("cuda")
    g = torch.Generator(device=dev).manual_seed(seed)
    dt = _type(c)

    def normal(*shape, scale=1.0):
        return torch.randn(shape, generator=g, device=dev) * scale

    s = {"case": c}
    if c["op"].startswith("recurrence"):
        T, B, D = c["T"], c["B"], c["D"]
        # gates that forget within a few steps up to within some hundred
        logits = 2.0 + 1.5 * normal(T, B, D)
        first = logits if c["gate"] else torch.sigmoid(logits)
        x = normal(T, B, D)
        if c["fused"]:
            z = torch.cat([first, x], dim=2).to(dt)
            s["a"], s["x"] = z[..., :D], z[..., D:]
        else:
            s["a"], s["x"] = first.to(dt), x.to(dt)
        s["h0"] = normal(B, D)
        s["lengths"] = None
        if c["ragged"]:
            at = torch.randperm(B, generator=g, device=dev)
            s["lengths"] = torch.tensor(_lengths(c), dtype=torch.int32, device=dev)[at].contiguous()
        if c["op"] == "recurrence_backward":
            h, _, s["states"] = _recurrence(s["a"], s["x"], s["h0"], s["lengths"], c["gate"], c["reverse"], torch.float32)
            s["dh"] = normal(T, B, D).to(dt)
            s["dhT"] = normal(B, D)
        return s
    if c["op"] == "product":
        m, n, k = c["rows"], c["outs"], c["width"]
        # activations of a norm, some channels larger than the rest
        x = normal(m, k) * (1 + 3 * (torch.rand(k, generator=g, device=dev) < 0.02).float())
        w = (torch.rand((n, k), generator=g, device=dev) * 2 - 1) / math.sqrt(k)
        qx, s["sx"] = _quantize(x, 1)
        qw, s["sw"] = _quantize(w, 128)
        s["qx"], s["qw"] = _pad16(qx), _pad16(qw)
        s["bias"] = normal(n, scale=0.1) if c["bias"] else None
        return s
    rows, width = c["rows"], c["width"]
    if c["op"] == "quantize":
        s["x"] = (normal(rows, width) * torch.exp(normal(1, width, scale=0.5))).to(dt)
        return s
    s["w"] = 1 + normal(width, scale=0.2)
    s["x"] = (1.5 * normal(rows, width)).to(dt)
    s["residual"] = (3 * normal(rows, width)).to(dt) if c["residual"] else None
    if c["op"] == "norm_backward":
        s["dy"] = normal(rows, width).to(dt)
    return s


# ---------------------------------------------------------------- plain forms
def _scan(f, b, h0):
    """h_t = f_t h_{t-1} + b_t over the first axis, every step at once: spans of 1, 2, 4 ... steps joined pairwise."""
    A, H = f, torch.cat([b[:1] + f[:1] * h0, b[1:]])
    span, T = 1, f.shape[0]
    while span < T:
        H = torch.cat([H[:span], H[span:] + A[span:] * H[:-span]])
        A = torch.cat([A[:span], A[span:] * A[:-span]])
        span *= 2
    return H


def _in_order(t, lengths, reverse):
    """Steps in the order of processing (its own inverse): a reversed sequence begins at its own last step."""
    if not reverse:
        return t
    if lengths is None:
        return t.flip(0)
    i = torch.arange(t.shape[0], device=t.device).reshape(-1, 1)
    at = torch.where(i < lengths, lengths - 1 - i, i)
    return torch.take_along_dim(t, at[:, :, None], 0)


def _steps(a, x, lengths, gate, reverse):
    """Decay, addend and the steps that count, in the order of processing."""
    a, x = (_in_order(t.float(), lengths, reverse) for t in (a, x))
    f = torch.sigmoid(a) if gate else a
    b = torch.sigmoid(-a) * x if gate else x
    if lengths is None:
        return a, x, f, b, None
    valid = (torch.arange(a.shape[0], device=a.device).reshape(-1, 1) < lengths)[:, :, None]
    return a, x, torch.where(valid, f, 1.0), torch.where(valid, b, 0.0), valid


def _recurrence(a, x, h0, lengths, gate, reverse, dt):
    _, _, f, b, valid = _steps(a, x, lengths, gate, reverse)
    H = _scan(f, b, h0)
    states = torch.cat([h0[None], H[SEGMENT - 1:-1:SEGMENT]])
    h = H if valid is None else torch.where(valid, H, 0.0)
    return _in_order(h, lengths, reverse).to(dt), H[-1].clone(), states


def _recurrence_backward(a, x, h0, dh, dhT, lengths, gate, reverse, dt):
    a, x, f, b, valid = _steps(a, x, lengths, gate, reverse)
    before = torch.cat([h0[None], _scan(f, b, h0)[:-1]])
    d = _in_order(dh.float(), lengths, reverse)
    if valid is not None:
        d = torch.where(valid, d, 0.0)
    # g_t = dh_t + f_{t+1} g_{t+1}, from the last step to the first
    g = _scan(torch.cat([torch.ones_like(f[:1]), f[1:].flip(0)]), d.flip(0), dhT).flip(0)
    if gate:
        da, dx = g * (before - x) * torch.sigmoid(a) * torch.sigmoid(-a), g * torch.sigmoid(-a)
    else:
        da, dx = g * before, g
    if valid is not None:
        da, dx = torch.where(valid, da, 0.0), torch.where(valid, dx, 0.0)
    return _in_order(da, lengths, reverse).to(dt), _in_order(dx, lengths, reverse).to(dt), f[0] * g[0]


def _quantize(x, block_rows):
    """8-bit values and the scales that they are multiples of: the largest magnitude of a block becomes 448."""
    rows, width = x.shape
    x = x.float()
    R, C = -(-rows // block_rows), -(-width // 128)
    held = torch.zeros((R * block_rows, C * 128), device=x.device)
    held[:rows, :width] = x
    scales = held.reshape(R, block_rows, C, 128).abs().amax(dim=(1, 3)).clamp_min(E4M3_MAX * FLT_MIN) / E4M3_MAX
    return (x / _spread(scales, block_rows, rows, width)).to(torch.float8_e4m3fn), scales


def _spread(scales, block_rows, rows, width):
    return scales.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(128, 1)[:, :width]


def _plain(s):
    c = s["case"]
    dt = _type(c)
    if c["op"] == "recurrence":
        h, hT, states = _recurrence(s["a"], s["x"], s["h0"], s["lengths"], c["gate"], c["reverse"], dt)
        return [h, hT, states] if c["save"] else [h, hT]
    if c["op"] == "recurrence_backward":
        return list(_recurrence_backward(s["a"], s["x"], s["h0"], s["dh"], s["dhT"], s["lengths"], c["gate"], c["reverse"], dt))
    if c["op"] == "product":
        x = s["qx"].float() * _spread(s["sx"], 1, c["rows"], c["width"])
        w = s["qw"].float() * _spread(s["sw"], 128, c["outs"], c["width"])
        y = x @ w.t()
        return (y if s["bias"] is None else y + s["bias"]).to(dt)
    if c["op"] == "quantize":
        return list(_quantize(s["x"], c["block_rows"]))
    r = s["x"].float()
    if c["op"] == "norm":
        if s["residual"] is not None:
            r = r + s["residual"].float()
        y = r * torch.rsqrt(r.square().mean(1, keepdim=True) + EPS) * s["w"]
        out = list(_quantize(y, 1)) if c["bits8"] else [y.to(dt)]
        return out + [r.to(dt)] if s["residual"] is not None else out
    # r is the stored sum; the gradient that reaches it past the norm is added
    rstd = torch.rsqrt(r.square().mean(1, keepdim=True) + EPS)
    dy = s["dy"].float()
    wdy = dy * s["w"]
    dr = rstd * (wdy - r * rstd.square() * (wdy * r).mean(1, keepdim=True))
    if s["residual"] is not None:
        dr = dr + s["residual"].float()
    return [dr.to(dt), (dy * r * rstd).sum(0)]


def _library(s):
    import paper_1901_10997_b200 as lib
    c = s["case"]
    if c["op"] == "recurrence":
        h, hT, states = lib.linear_recurrence(s["a"], s["x"], s["h0"], s["lengths"], gate=c["gate"], reverse=c["reverse"], save=c["save"])
        return [h, hT, states] if c["save"] else [h, hT]
    if c["op"] == "recurrence_backward":
        return list(lib.linear_recurrence_backward(s["a"], s["x"], s["states"], s["dh"], s["dhT"], s["lengths"], gate=c["gate"],
                                                   reverse=c["reverse"]))
    if c["op"] == "product":
        return lib.fp8_product(s["qx"], s["sx"], s["qw"], s["sw"], s["bias"], dtype=_type(c))
    if c["op"] == "quantize":
        return list(lib.fp8_quantize(s["x"], block_rows=c["block_rows"]))
    if c["op"] == "norm_backward":
        return list(lib.rms_norm_backward(s["dy"], s["x"], s["w"], s["residual"], eps=EPS))
    if c["bits8"]:
        q, scales, r = lib.rms_norm_fp8(s["x"], s["w"], s["residual"], eps=EPS)
        return [q, scales] if r is None else [q, scales, r]
    y, r = lib.rms_norm(s["x"], s["w"], s["residual"], eps=EPS)
    return [y] if r is None else [y, r]


def run(state):
    return _library(state) if own else _plain(state)


# ---------------------------------------------------------------- what a pass cannot do without
def work(case):
    c = case
    es = 4 if c["dtype"] == "fp32" else 2
    if c["op"].startswith("recurrence"):
        n, rows = c["T"] * c["B"] * c["D"], c["B"] * c["D"]
        valid = sum(_lengths(c)) * c["D"]
        states = -(-c["T"] // SEGMENT) * rows
        if c["op"] == "recurrence":
            return {"bytes": es * (2 * valid + n) + 8 * rows + (4 * states if c["save"] else 0), "flops": 8.0 * valid}
        return {"bytes": es * (3 * valid + 2 * n) + 8 * rows + 4 * states, "flops": 18.0 * valid}
    if c["op"] == "product":
        m, n, k = c["rows"], c["outs"], c["width"]
        blocks = -(-k // 128)
        return {"bytes": m * k + n * k + 4 * blocks * (m + -(-n // 128)) + es * m * n + (4 * n if c["bias"] else 0), "flops": 2.0 * m * n * k}
    n, blocks = c["rows"] * c["width"], -(-c["width"] // 128)
    if c["op"] == "quantize":
        return {"bytes": (es + 1) * n + 4 * blocks * -(-c["rows"] // c["block_rows"]), "flops": 3.0 * n}
    if c["op"] == "norm":
        held = n + 4 * blocks * c["rows"] if c["bits8"] else es * n
        return {"bytes": es * n * (3 if c["residual"] else 1) + held + 4 * c["width"], "flops": 6.0 * n}
    return {"bytes": es * n * (4 if c["residual"] else 3) + 8 * c["width"], "flops": 12.0 * n}


# ---------------------------------------------------------------- the definitions in 64 bits, step by step
def exact(case, seed):
    c, s = case, prepare(case, seed)
    if c["op"].startswith("recurrence"):
        T, B, D = c["T"], c["B"], c["D"]
        a, x, h0 = s["a"].double(), s["x"].double(), s["h0"].double()
        f = 1 / (1 + torch.exp(-a)) if c["gate"] else a
        add = x / (1 + torch.exp(a)) if c["gate"] else x
        lens = s["lengths"] if c["ragged"] else torch.full((B,), T, dtype=torch.int32, device=a.device)
        live = torch.arange(T, device=a.device)[:, None, None] < lens[:, None].long()
        f.masked_fill_(~live, 1.0)
        add.masked_fill_(~live, 0.0)
        times = range(T - 1, -1, -1) if c["reverse"] else range(T)
        h, before, after = h0, torch.empty_like(a), torch.empty_like(a)
        for t in times:
            before[t] = h
            h = torch.addcmul(add[t], f[t], h, out=after[t])
        if c["op"] == "recurrence":
            out = [torch.where(live, after, 0.0), h.clone()]
            if c["save"]:
                k = torch.arange(0, T, SEGMENT, device=a.device)[:, None]
                at = lens.long() - k if c["reverse"] else k - 1
                held = torch.take_along_dim(after, at.clamp(0, T - 1)[:, :, None].expand(-1, B, D), 0)
                held[0] = h0
                out.append(held)
            return out
        d = torch.where(live, s["dh"].double(), 0.0)
        g, gs = s["dhT"].double(), torch.empty_like(a)
        for t in reversed(times):
            g = torch.add(g, d[t], out=gs[t]) * f[t]
        if c["gate"]:
            da, dx = gs * (before - x) * f * (1 - f), gs * (1 - f)
        else:
            da, dx = gs * before, gs
        return [torch.where(live, da, 0.0), torch.where(live, dx, 0.0), g]
    if c["op"] == "product":
        def whole(q, scales, block_rows):
            out = q.double()
            for j in range(scales.shape[1]):
                out[:, 128 * j:128 * (j + 1)] *= scales[:, j].double().repeat_interleave(block_rows)[:q.shape[0], None]
            return out
        y = whole(s["qx"], s["sx"], 1) @ whole(s["qw"], s["sw"], 128).t()
        return y if s["bias"] is None else y + s["bias"].double()

    def held(y, block_rows):
        q, scales = torch.empty_like(y, dtype=torch.float32), []
        for j in range(0, y.shape[1], 128):
            top = y[:, j:j + 128].abs().amax(1)
            if block_rows > 1:
                top = torch.stack([p.amax() for p in top.split(block_rows)])
            scales.append(top.clamp_min(E4M3_MAX * FLT_MIN) / E4M3_MAX)
            q[:, j:j + 128] = y[:, j:j + 128] / scales[-1].repeat_interleave(block_rows)[:y.shape[0], None]
        return [q.to(torch.float8_e4m3fn).double(), torch.stack(scales, 1)]

    x = s["x"].double()
    if c["op"] == "quantize":
        return held(x, c["block_rows"])
    w, res = s["w"].double(), None if s["residual"] is None else s["residual"].double()
    if c["op"] == "norm":
        r = x if res is None else x + res
        y = r / torch.sqrt((r * r).sum(1) / c["width"] + EPS)[:, None] * w
        return (held(y, 1) if c["bits8"] else [y]) + ([] if res is None else [r])
    dy = s["dy"].double()
    norm = torch.sqrt((x * x).sum(1) / c["width"] + EPS)[:, None]
    unit = x / norm
    part = dy * w
    dr = (part - unit * ((part * unit).sum(1) / c["width"])[:, None]) / norm
    return [dr if res is None else dr + res, (dy * unit).sum(0)]
