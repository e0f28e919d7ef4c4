"""Timed operators of encoder training and of encoders outside an index: the
layers of a network in fp32, bf16 and fp16, whose latents the search takes as
logits, and whose gradients start from the L_sim loss.

  linear        y = act(x W^T + bias) + residual (NR.nr_linear).  One row is an
                interactive query's pass through a layer, some tens a serving
                batch, 10,000 the benchmark's batch, 65,536 a chunk of the base.
  linear_train  the same with its backward pass (NR.nr_linear with the
                pre-activation kept, NR.nr_linear_grad): gradients of the input,
                the weights and the bias.  4096 rows is the trainer's batch.
  norm          layer norm of rows (NR.nr_layer_norm).
  norm_train    the same with its backward pass (NR.nr_layer_norm_grad), whose
                input gradient is joined with the residual path's.
  hold          activations put into 8 bits and read back (NR.nr_act_hold,
                NR.nr_act_read): groups of 32 along a row share a power of two.
  block_train   a pre-norm residual block, x + act(norm(x) W^T + bias), forward
                and backward, its three activations held in 8 bits in between.

Widths are those of the framework's encoders (96, 128, 1536 -> 512, 256, 128,
64 -> 16 to 24) and wider generic ones up to its limit of 4096.
"""
from __future__ import annotations

import math

import torch

own = False
DEV = "cuda"
TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
EPS = 1e-5
GROUP = 32


# --------------------------------------------------------------------------
# the cases
# --------------------------------------------------------------------------

def listed():
    return [
        # one interactive query through the first layer of the 1M and 1B encoders
        dict(name="linear_f32_1q", kind="linear", dtype="f32", m=1, k=128, n=256, act="relu",
             res=False, bias=True, pad=0),
        # a serving batch through a wide layer: reading the weights decides
        dict(name="linear_bf16_48q", kind="linear", dtype="bf16", m=48, k=4096, n=4096, act="silu",
             res=True, bias=True, pad=0),
        # the benchmark's batch through the first layer of the 1536-d encoder
        dict(name="linear_f32_10k", kind="linear", dtype="f32", m=10_000, k=1536, n=512,
             act="relu", res=False, bias=True, pad=0),
        # a chunk of the base through a wide hidden layer, the largest products
        dict(name="linear_bf16_64k", kind="linear", dtype="bf16", m=65_536, k=1024, n=4096,
             act="gelu", res=False, bias=True, pad=0),
        # the trainer's batch through its first layer
        dict(name="linear_train_f32_4k", kind="linear_train", dtype="f32", m=4096, k=128, n=256,
             act="relu", res=False, bias=True, pad=0),
        # a residual layer of a wider encoder in half the memory
        dict(name="linear_train_bf16_16k", kind="linear_train", dtype="bf16", m=16_384, k=1024,
             n=1024, act="gelu", res=True, bias=True, pad=0),
        # odd widths, a ragged batch, rows cut out of a wider array
        dict(name="linear_train_f16_odd", kind="linear_train", dtype="f16", m=5003, k=333, n=777,
             act="silu", res=True, bias=True, pad=7),
        # a serving batch's norm
        dict(name="norm_bf16_48q", kind="norm", dtype="bf16", m=48, d=1536, pad=0),
        # norms of a large batch of embeddings, forward and backward
        dict(name="norm_train_bf16_64k", kind="norm_train", dtype="bf16", m=65_536, d=1536,
             add=True, pad=0),
        # an odd width in fp32
        dict(name="norm_train_f32_odd", kind="norm_train", dtype="f32", m=4097, d=257, add=False,
             pad=3),
        # the activations of a large batch into 8 bits and back
        dict(name="hold_bf16_i8", kind="hold", dtype="bf16", m=65_536, d=1536, fmt="i8", pad=0),
        # a residual block whose activations are held in 8 bits
        dict(name="block_train_bf16_e4m3", kind="block_train", dtype="bf16", m=16_384, d=1024,
             act="gelu", fmt="e4m3", pad=0),
    ]


def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _width(rng, lo, hi):
    """Widths over [lo, hi]: half of them whole vectors, the others any number."""
    w = _log_int(rng, lo, hi)
    return max(16, w // 16 * 16) if rng.random() < 0.5 else w


def draw(rng):
    kind = rng.choice(["linear", "linear", "linear_train", "linear_train", "norm", "norm_train",
                       "hold", "block_train"])
    c = dict(kind=kind, dtype=rng.choice(["f32", "bf16", "f16"]), pad=rng.choice([0, 0, 0, 5, 16]))
    rows = _log_int(rng, 1 if kind in ("linear", "norm", "hold") else 100, 65_536)
    if kind in ("linear", "linear_train"):
        c.update(m=rows, k=_width(rng, 16, 4096), n=_width(rng, 16, 4096),
                 act=rng.choice(["none", "relu", "gelu", "silu"]), res=rng.random() < 0.4,
                 bias=rng.random() < 0.8)
        per_row = (2 if kind == "linear" else 6) * c["k"] * c["n"]
        c["m"] = min(c["m"], int((5e11 if c["dtype"] != "f32" else 2e11) // per_row))
    elif kind == "block_train":
        c.update(m=rows, d=_width(rng, 64, 2048), act=rng.choice(["relu", "gelu", "silu"]),
                 fmt=rng.choice(["i8", "e4m3"]))
        c["m"] = min(c["m"], int(2e11 // (6 * c["d"] ** 2)))
    else:
        c.update(m=rows, d=_width(rng, 16, 4096))
        if kind == "norm_train":
            c["add"] = rng.random() < 0.5
        if kind == "hold":
            c["fmt"] = rng.choice(["i8", "e4m3"])
    return c


# --------------------------------------------------------------------------
# inputs
# --------------------------------------------------------------------------

def _rows(g, m, d, dtype, pad, scale=1.0, wide=True):
    """[m, d] activations: normal, a few columns of large ones (`wide`), the
    last rows of a batch zero as padding leaves them; with `pad` a cut out of
    rows that are longer."""
    x = torch.randn((m, d + pad), generator=g, device=DEV) * scale
    if wide:
        x[:, 7::97] *= 8.0
    if m >= 50:
        x[m - m // 50:] = 0.0
    return x.to(TYPES[dtype])[:, :d]


def prepare(case, seed):
    g = torch.Generator(device=DEV).manual_seed(seed * 8 + 5)
    t, m, pad = TYPES[case["dtype"]], case["m"], case["pad"]
    s = dict(case=case)
    if case["kind"] in ("linear", "linear_train", "block_train"):
        block = case["kind"] == "block_train"
        k = case["d"] if block else case["k"]
        n = case["d"] if block else case["n"]
        s["x"] = _rows(g, m, k, case["dtype"], pad)
        s["w"] = (torch.randn((n, k), generator=g, device=DEV) / math.sqrt(k)).to(t)
        s["b"] = ((torch.randn(n, generator=g, device=DEV) * 0.1).to(t)
                  if block or case["bias"] else None)
        s["r"] = (_rows(g, m, n, case["dtype"], pad)
                  if not block and case["res"] else None)
        if case["kind"] != "linear":
            s["dy"] = _rows(g, m, n, case["dtype"], pad, scale=0.05, wide=False)
        if block:
            s["g"] = (1.0 + 0.1 * torch.randn(k, generator=g, device=DEV)).to(t)
            s["gb"] = (0.1 * torch.randn(k, generator=g, device=DEV)).to(t)
    else:
        d = case["d"]
        s["x"] = _rows(g, m, d, case["dtype"], pad)
        if case["kind"] != "hold":
            s["x"] = s["x"] + 0.5 if pad == 0 else s["x"]
            s["g"] = (1.0 + 0.1 * torch.randn(d, generator=g, device=DEV)).to(t)
            s["gb"] = (0.1 * torch.randn(d, generator=g, device=DEV)).to(t)
        if case["kind"] == "norm_train":
            s["dy"] = _rows(g, m, d, case["dtype"], pad, scale=0.05, wide=False)
            s["add"] = (_rows(g, m, d, case["dtype"], pad, scale=0.05, wide=False)
                        if case["add"] else None)
    return s


# --------------------------------------------------------------------------
# the operators, plainly: elementary operations in 32 bits
# --------------------------------------------------------------------------

def _act(z, act):
    if act == "relu":
        return torch.clamp_min(z, 0.0)
    if act == "gelu":
        return 0.5 * z * torch.erfc(z * -math.sqrt(0.5))
    if act == "silu":
        return z / (1.0 + torch.exp(-z))
    return z


def _act_slope(z, act):
    if act == "relu":
        return (z > 0).to(z.dtype)
    if act == "gelu":
        return (0.5 * torch.erfc(z * -math.sqrt(0.5))
                + z * torch.exp(-0.5 * z * z) * (1.0 / math.sqrt(2.0 * math.pi)))
    if act == "silu":
        p = 1.0 / (1.0 + torch.exp(-z))
        return p * (1.0 + z * (1.0 - p))
    return torch.ones_like(z)


def _linear(x, w, b, r, act):
    z = x @ w.T
    if b is not None:
        z = z + b
    y = _act(z, act)
    return (y if r is None else y + r), z


def _linear_grad(dy, x, w, z, act):
    dz = dy * _act_slope(z, act) if act != "none" else dy
    return dz @ w, dz.T @ x, dz.sum(0)


def _norm(x, g, b):
    mean = x.mean(1, keepdim=True)
    c = x - mean
    rstd = torch.rsqrt((c * c).mean(1, keepdim=True) + EPS)
    return c * rstd * g + b, mean, rstd


def _norm_grad(dy, x, mean, rstd, g):
    xh = (x - mean) * rstd
    dg = dy * g
    dx = rstd * (dg - dg.mean(1, keepdim=True) - xh * (dg * xh).mean(1, keepdim=True))
    return dx, (dy * xh).sum(0), dy.sum(0)


def _pow2(e):
    """2^e in 32 bits for -126 <= e <= 127, from its bits."""
    return ((e + 127) << 23).to(torch.int32).view(torch.float32)


def _held(x, fmt, dtype):
    """The values that 8 bits stand for: per group of 32 along a row q 2^e,
    with the smallest e at which the largest magnitude fits (int8: it rounds to
    at most 127; e4m3: it is at most 448)."""
    m, d = x.shape
    p = torch.nn.functional.pad(x, (0, -d % GROUP)).view(m, -1, GROUP)
    amax = p.abs().amax(2, keepdim=True)
    top = 6 if fmt == "i8" else 8
    e = torch.frexp(amax)[1].to(torch.int64) - 1 - top
    e = torch.where(amax > 0, e, -126).clamp(-126, 121)
    v = amax * _pow2(-e)
    e = e + (v >= 127.5 if fmt == "i8" else v > 448.0).to(torch.int64)
    half = dtype == torch.float16
    e = e.clamp(-126, (9 if half else 121) if fmt == "i8" else (7 if half else 119))
    v = p * _pow2(-e)
    if fmt == "i8":
        q = torch.round(v).clamp(-127.0, 127.0)
    else:
        v = v.clamp(-448.0, 448.0)
        step = _pow2((torch.frexp(v)[1].to(torch.int64) - 1).clamp_min(-6) - 3)
        q = torch.round(v / step) * step
    return (q * _pow2(e)).view(m, -1)[:, :d]


def _plain(s):
    c = s["case"]
    t, kind = TYPES[c["dtype"]], c["kind"]
    f = {k: (v.float() if isinstance(v, torch.Tensor) else v) for k, v in s.items()}
    if kind == "linear":
        return _linear(f["x"], f["w"], f["b"], f["r"], c["act"])[0].to(t)
    if kind == "linear_train":
        y, z = _linear(f["x"], f["w"], f["b"], f["r"], c["act"])
        out = (y,) + _linear_grad(f["dy"], f["x"], f["w"], z, c["act"])
        return [v.to(t) for v in (out if c["bias"] else out[:3])]
    if kind == "norm":
        return _norm(f["x"], f["g"], f["gb"])[0].to(t)
    if kind == "norm_train":
        y, mean, rstd = _norm(f["x"], f["g"], f["gb"])
        dx, dg, db = _norm_grad(f["dy"], f["x"], mean, rstd, f["g"])
        if f["add"] is not None:
            dx = dx + f["add"]
        return [v.to(t) for v in (y, dx, dg, db)]
    if kind == "hold":
        return _held(f["x"], c["fmt"], t).to(t)
    # the block: what is held is held of the tensors between the operators, in their type
    y1, mean, rstd = _norm(f["x"], f["g"], f["gb"])
    y1 = y1.to(t).float()
    out, z = _linear(y1, f["w"], f["b"], f["x"], c["act"])
    hx, hy, hz = (_held(v.to(t).float(), c["fmt"], t) for v in (f["x"], y1, z))
    d1, dw, db = _linear_grad(f["dy"], hy, f["w"], hz, c["act"])
    dx, dg, dgb = _norm_grad(d1, hx, mean, rstd, f["g"])
    return [v.to(t) for v in (out, dx + f["dy"], dw, db, dg, dgb)]


# --------------------------------------------------------------------------
# the framework's calls
# --------------------------------------------------------------------------

def _calls(s):
    from paper_2608_15438_amd import neuroute as NR
    c = s["case"]
    kind = c["kind"]
    if kind == "linear":
        return NR.nr_linear(s["x"], s["w"], s["b"], act=c["act"], residual=s["r"])
    if kind == "linear_train":
        y, z = NR.nr_linear(s["x"], s["w"], s["b"], act=c["act"], residual=s["r"], pre=True)
        dx, dw, db = NR.nr_linear_grad(s["dy"], s["x"], s["w"], act=c["act"], pre=z, db=c["bias"])
        return [y, dx, dw, db] if c["bias"] else [y, dx, dw]
    if kind == "norm":
        return NR.nr_layer_norm(s["x"], s["g"], s["gb"], eps=EPS)
    if kind == "norm_train":
        y, stats = NR.nr_layer_norm(s["x"], s["g"], s["gb"], eps=EPS, stats=True)
        dx, dg, db = NR.nr_layer_norm_grad(s["dy"], s["x"], stats, s["g"], add=s["add"])
        return [y, dx, dg, db]
    if kind == "hold":
        return NR.nr_act_read(NR.nr_act_hold(s["x"], c["fmt"]))
    fmt = c["fmt"]
    y1, stats, hx, hy = NR.nr_layer_norm(s["x"], s["g"], s["gb"], eps=EPS, stats=True, hold_x=fmt,
                                         hold_y=fmt)
    out, hz = NR.nr_linear(y1, s["w"], s["b"], act=c["act"], residual=s["x"], pre=fmt)
    d1, dw, db = NR.nr_linear_grad(s["dy"], hy, s["w"], act=c["act"], pre=hz)
    dx, dg, dgb = NR.nr_layer_norm_grad(d1, hx, stats, s["g"], add=s["dy"])
    return [out, dx, dw, db, dg, dgb]


def run(state):
    return _calls(state) if own else _plain(state)


# --------------------------------------------------------------------------
# work and exact results
# --------------------------------------------------------------------------

def work(case):
    e = 4 if case["dtype"] == "f32" else 2
    m, kind = case["m"], case["kind"]
    if kind in ("linear", "linear_train"):
        k, n = case["k"], case["n"]
        io = m * k + n * k + m * n + (m * n if case["res"] else 0) + (n if case["bias"] else 0)
        if kind == "linear":
            return dict(bytes=e * io, flops=2 * m * n * k)
        io += m * n + m * k + n * k + (n if case["bias"] else 0)
        return dict(bytes=e * io, flops=6 * m * n * k)
    d = case["d"]
    if kind == "norm":
        return dict(bytes=e * (2 * m * d + 2 * d), flops=8 * m * d)
    if kind == "norm_train":
        io = 4 * m * d + (m * d if case["add"] else 0) + 4 * d
        return dict(bytes=e * io, flops=24 * m * d)
    if kind == "hold":
        return dict(bytes=2 * m * d * e, flops=4 * m * d)
    return dict(bytes=e * (4 * m * d + 2 * d * d + 6 * d), flops=6 * m * d * d)


def exact(case, seed):
    """From the definitions, in 64 bits."""
    s = prepare(case, seed)
    kind, t = case["kind"], TYPES[case["dtype"]]

    def dbl(name):
        return s[name].double() if s.get(name) is not None else None

    def typed(v):       # a tensor that one operator hands to the next, in its type
        return v.to(t).double()

    def phi(z):         # the normal distribution function
        return 0.5 * torch.special.erfc(-z / math.sqrt(2.0))

    def layer(x, w, b, act):
        z = torch.mm(x, w.t().contiguous())
        z = z if b is None else z + b[None, :]
        if act == "relu":
            return z, torch.where(z > 0, z, torch.zeros_like(z))
        if act == "gelu":
            return z, z * phi(z)
        if act == "silu":
            return z, z * torch.sigmoid(z)
        return z, z

    def slope(z, act):
        if act == "relu":
            return torch.where(z > 0, 1.0, 0.0).double()
        if act == "gelu":
            return phi(z) + z * torch.exp(-z * z / 2) / math.sqrt(2 * math.pi)
        if act == "silu":
            p = torch.sigmoid(z)
            return p + z * p * torch.sigmoid(-z)
        return torch.ones_like(z)

    def layer_back(dy, x, w, z, act):
        dz = dy * slope(z, act)
        return torch.mm(dz, w), torch.mm(dz.t().contiguous(), x), dz.sum(dim=0)

    def whiten(x):
        mu = x.mean(dim=1, keepdim=True)
        sd = torch.sqrt(((x - mu) ** 2).mean(dim=1, keepdim=True) + EPS)
        return mu, sd

    def whiten_back(dy, xh, sd, g):
        u = dy * g
        proj = u - u.mean(dim=1, keepdim=True) - xh * (u * xh).mean(dim=1, keepdim=True)
        return proj / sd, (dy * xh).sum(dim=0), dy.sum(dim=0)

    def eight(x, fmt):
        m, d = x.shape
        out = torch.empty_like(x)
        small = t == torch.float16
        for c0 in range(0, d, GROUP):
            v = x[:, c0:c0 + GROUP]
            big = v.abs().max(dim=1, keepdim=True).values
            lim = 127.5 if fmt == "i8" else 448.0
            # the smallest power at which the largest magnitude fits
            e = torch.floor(torch.log2(big.clamp_min(2.0 ** -1000) / lim)) - 1
            fits = (lambda a: a < lim) if fmt == "i8" else (lambda a: a <= lim)
            for _ in range(3):
                e = torch.where(fits(big * torch.exp2(-e)), e, e + 1)
            hi = (9 if small else 121) if fmt == "i8" else (7 if small else 119)
            e = e.clamp(-126, hi)
            u = v * torch.exp2(-e)
            if fmt == "i8":
                q = torch.round(u).clamp(-127, 127)
            else:
                u = u.clamp(-448, 448)
                b = torch.floor(torch.log2(u.abs().clamp_min(2.0 ** -20))).clamp_min(-6)
                b = torch.where(torch.exp2(b) > u.abs(), (b - 1).clamp_min(-6), b)
                q = torch.round(u * torch.exp2(3 - b)) * torch.exp2(b - 3)
            out[:, c0:c0 + GROUP] = q * torch.exp2(e)
        return out

    x = dbl("x")
    if kind in ("linear", "linear_train"):
        w, r = dbl("w"), dbl("r")
        z, y = layer(x, w, dbl("b"), case["act"])
        y = y if r is None else y + r
        if kind == "linear":
            return y
        dx, dw, db = layer_back(dbl("dy"), x, w, z, case["act"])
        return [y, dx, dw, db] if case["bias"] else [y, dx, dw]
    if kind == "hold":
        return eight(x, case["fmt"])
    g, gb = dbl("g"), dbl("gb")
    mu, sd = whiten(x)
    y = (x - mu) / sd * g + gb
    if kind == "norm":
        return y
    if kind == "norm_train":
        dx, dg, db = whiten_back(dbl("dy"), (x - mu) / sd, sd, g)
        return [y, dx if s["add"] is None else dx + dbl("add"), dg, db]
    fmt, dy, w = case["fmt"], dbl("dy"), dbl("w")
    y = typed(y)
    z, out = layer(y, w, dbl("b"), case["act"])
    d1, dw, db = layer_back(dy, eight(y, fmt), w, eight(typed(z), fmt), case["act"])
    dx, dg, dgb = whiten_back(d1, (eight(x, fmt) - mu) / sd, sd, g)
    return [out + x, dx + dy, dw, db, dg, dgb]
