"""The layers' kernels (linear with its epilogue, layer norm, activations in 8
bits, and their gradients) against plain forms in 64 bits, at the sizes, types,
strides and values where they can go wrong.

Tolerances count roundings.  A sum of n products in fp32 is off by at most
n 2^-24 of the sum of their magnitudes, whatever its order; a rounding to the
type by half a step.  Slopes of the activations are at most 1.13, and the
activation and its slope are evaluated to 2e-6 (1 + |z|) (fp32: a few steps of
2^-24; the 16-bit types: an approximation good to 1.5e-7 and fast exponentials)."""
import math
import zlib

import pytest
import torch

from paper_2608_15438_amd import neuroute as NR
from tests import layers_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
U = R.U


def gen(*key):
    return torch.Generator(device=DEV).manual_seed(zlib.crc32(repr(key).encode()))


def rows(g, m, d, dtype, pad=0, scale=1.0):
    """[m, d]; with pad the rows lie `pad` elements further apart, one element in."""
    x = (torch.randn((m, d + pad), generator=g, device=DEV) * scale).to(dtype)
    return x[:, 1:d + 1] if pad else x


def close(got, want, tol, what):
    err = (got.double() - want).abs()
    bad = ~(err <= tol)
    assert not bool(bad.any()), (what, int(bad.sum()), float(err.max()),
                                 float((err / tol.clamp_min(1e-300)).max()))


SIZES = [(1, 1, 1), (1, 128, 256), (2, 4096, 40), (3, 17, 5), (7, 1536, 512), (16, 40, 16),
         (33, 31, 33), (64, 64, 64), (65, 100, 130), (130, 96, 20), (257, 333, 129),
         (1000, 256, 24), (300, 2048, 96), (4096, 128, 256), (515, 1030, 777)]


def linear_case(m, k, n, t, pad=0):
    g = gen(m, k, n, t)
    dt = R.TYPES[t]
    x = rows(g, m, k, dt, pad)
    w = rows(g, n, k, dt, pad, 1.0 / math.sqrt(k))
    b = rows(g, 1, n, dt, scale=0.5)[0]
    r = rows(g, m, n, dt, pad)
    return g, dt, x, w, b, r


def check_linear(x, w, b, r, act, y, z):
    dt = y.dtype
    X, W = x.double(), w.double()
    mag = X.abs() @ W.abs().T
    Z = X @ W.T
    if b is not None:
        Z, mag = Z + b.double(), mag + b.double().abs()
    Y = R.act(Z, act) + (0 if r is None else r.double())
    tz = (x.shape[1] + 2) * U * mag
    if z is not None:
        close(z, Z, tz + R.half_step(Z.abs() + tz, dt), "pre")
    ty = 1.13 * tz + 2e-6 * (1 + Z.abs()) * (act in ("gelu", "silu")) + 2 * U * Y.abs()
    if r is not None:
        ty = ty + U * r.double().abs()
    close(y, Y, ty + R.half_step(Y.abs() + ty, dt), "y")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_linear(m, k, n, t):
    g, dt, x, w, b, r = linear_case(m, k, n, t)
    for act, bias, res in (("none", None, None), ("relu", b, None), ("gelu", b, r),
                           ("silu", None, r)):
        y, z = NR.nr_linear(x, w, bias, act=act, residual=res, pre=True)
        check_linear(x, w, bias, res, act, y, z)
        # without the pre-activation, and again: the same bits
        assert torch.equal(NR.nr_linear(x, w, bias, act=act, residual=res), y)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad", [1, 8, 13])
def test_linear_strides(pad, t):
    # rows off the 16-byte boundaries, and cut out of longer ones
    for m, k, n in ((70, 64, 96), (5, 200, 33), (200, 65, 66)):
        g, dt, x, w, b, r = linear_case(m, k, n, t, pad)
        y, z = NR.nr_linear(x, w, b, act="silu", residual=r, pre=True)
        check_linear(x, w, b, r, "silu", y, z)
        c = NR.nr_linear(x.contiguous(), w.contiguous(), b, act="silu", residual=r.contiguous())
        assert torch.equal(c, y)


def grad_check(dy, x, w, act, pre, got, rounded):
    """got = (dx, dw, db) against the formulas; `rounded`: dz was rounded to the type"""
    dt = dy.dtype
    DY, X, W = dy.double(), x.double(), w.double()
    m, n = dy.shape
    Z = pre.double() if pre is not None else None
    S = R.slope(Z, act) if act != "none" else torch.ones_like(DY)
    DZ = DY * S
    tz = torch.zeros_like(DZ)
    if act != "none":
        tz = 2e-6 * (1 + Z.abs()) * DY.abs() * (act != "relu") + U * DZ.abs()
    td = tz + (R.half_step(DZ.abs() + tz, dt) if rounded else 0)
    AZ = DZ.abs() + td
    dx, dw, db = got
    if dx is not None:
        t = td @ W.abs() + (n + 2) * U * (AZ @ W.abs())
        close(dx, DZ @ W, t + R.half_step((DZ @ W).abs() + t, dt), "dx")
    if dw is not None:
        t = td.T @ X.abs() + (m + 2) * U * (AZ.T @ X.abs())
        want = DZ.T @ X
        close(dw, want, t + R.half_step(want.abs() + t, dt), "dw")
    if db is not None:
        t = tz.sum(0) + (m + 2) * U * AZ.sum(0)
        want = DZ.sum(0)
        close(db, want, t + R.half_step(want.abs() + t, dt), "db")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_linear_grad(m, k, n, t):
    g, dt, x, w, b, r = linear_case(m, k, n, t)
    dy = rows(g, m, n, dt, scale=0.1)
    pre = rows(g, m, n, dt)
    for act in ("none", "relu", "gelu", "silu"):
        got = NR.nr_linear_grad(dy, x, w, act=act, pre=pre)
        grad_check(dy, x, w, act, pre, got, act != "none" and t != "f32")
        again = NR.nr_linear_grad(dy, x, w, act=act, pre=pre)
        assert all(torch.equal(a, c) for a, c in zip(got, again))
    # each alone: the same bits
    dx, dw, db = got
    assert torch.equal(NR.nr_linear_grad(dy, None, w, "silu", pre, dw=False, db=False)[0], dx)
    assert torch.equal(NR.nr_linear_grad(dy, x, None, "silu", pre, dx=False, db=False)[1], dw)
    assert torch.equal(NR.nr_linear_grad(dy, x, None, "silu", pre, dx=False, dw=False)[2], db)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n", [(4200, 200, 4104), (200, 4200, 4104), (4200, 4104, 200),
                                   (4097, 72, 4099), (16_400, 1030, 264), (9000, 520, 48),
                                   (16_384, 1024, 1024), (300, 40, 8192), (20_000, 33, 100)])
def test_linear_many_tiles(m, k, n, t):
    # each product with more outputs than the chip takes at once, its ends inside tiles
    g, dt, x, w, b, r = linear_case(m, k, n, t)
    y, z = NR.nr_linear(x, w, b, act="gelu", residual=r, pre=True)
    check_linear(x, w, b, r, "gelu", y, z)
    dy = rows(g, m, n, dt, scale=0.1)
    got = NR.nr_linear_grad(dy, x, w, act="gelu", pre=z)
    grad_check(dy, x, w, "gelu", z, got, t != "f32")
    for fmt in ("i8", "e4m3"):
        h, hx = NR.nr_act_hold(z, fmt), NR.nr_act_hold(x, fmt)
        y2, hz = NR.nr_linear(x, w, b, act="gelu", residual=r, pre=fmt)
        assert torch.equal(y, y2) and torch.equal(h.scale, hz.scale)
        assert torch.equal(h.q.view(torch.uint8), hz.q.view(torch.uint8))
        got = NR.nr_linear_grad(dy, hx, w, act="gelu", pre=hz)
        want = NR.nr_linear_grad(dy, NR.nr_act_read(hx), w, act="gelu", pre=NR.nr_act_read(hz))
        # one held: another path for dw, the same products in the same order
        grad_check(dy, NR.nr_act_read(hx), w, "gelu", NR.nr_act_read(hz), got, t != "f32")
        assert torch.equal(got[0], want[0]) and torch.equal(got[2], want[2])


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad", [1, 8, 13])
def test_linear_grad_strides(pad, t):
    for m, k, n in ((70, 64, 96), (5, 200, 33), (200, 65, 66)):
        g, dt, x, w, b, r = linear_case(m, k, n, t, pad)
        dy, pre = rows(g, m, n, dt, pad, 0.1), rows(g, m, n, dt, pad)
        for act in ("none", "gelu"):
            got = NR.nr_linear_grad(dy, x, w, act=act, pre=pre)
            grad_check(dy, x, w, act, pre, got, act != "none" and t != "f32")


def test_linear_gradient_against_differences():
    # fp32 gradients against central differences of the 64-bit forward pass: the
    # step's square (1e-8) times the third derivative, and fp32's own roundings
    m, k, n = 20, 12, 9
    for act in ("none", "gelu", "silu"):
        g, dt, x, w, b, r = linear_case(m, k, n, "f32")
        dy = rows(g, m, n, dt)
        y, z = NR.nr_linear(x, w, b, act=act, residual=r, pre=True)
        dx, dw, db = NR.nr_linear_grad(dy, x, w, act=act, pre=z)
        f = lambda X, W, B: (R.act(X @ W.T + B, act) * dy.double()).sum()
        X, W, B = x.double(), w.double(), b.double()
        for grad, i in ((dx, 0), (dw, 1), (db, 2)):
            v = torch.randn(grad.shape, generator=g, device=DEV).double()
            h = 1e-4
            args = [[X, W, B], [X, W, B]]
            args[0][i], args[1][i] = args[0][i] + h * v, args[1][i] - h * v
            want = float((f(*args[0]) - f(*args[1])) / (2 * h))
            size = float((grad.double() * v).abs().sum())
            assert abs(float((grad.double() * v).sum()) - want) <= 1e-5 * size + 1e-6, (act, i)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_linear_no_rows(t):
    g, dt, x, w, b, r = linear_case(4, 6, 5, t)
    y, z = NR.nr_linear(x[:0], w, b, act="gelu", residual=r[:0], pre=True)
    assert y.shape == z.shape == (0, 5)
    y, z = NR.nr_linear(x[:0], w, b, act="gelu", pre="i8")
    assert z.shape == (0, 5)
    dx, dw, db = NR.nr_linear_grad(y, x[:0], w, act="gelu", pre=z)
    assert dx.shape == (0, 6) and not dw.any() and not db.any()
    assert dw.shape == (5, 6) and db.shape == (5,)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_linear_rows_apart(t):
    # a row's infinities and NaN stay in its own outputs; rows behind the
    # outputs' ends are left as they were
    g, dt, x, w, b, r = linear_case(70, 96, 40, t)
    y0, z0 = NR.nr_linear(x, w, b, act="relu", pre=True)
    x2 = x.clone()
    x2[3, 5], x2[40, 0], x2[64, 95] = math.nan, math.inf, -math.inf
    y, z = NR.nr_linear(x2, w, b, act="relu", pre=True)
    keep = torch.ones(70, dtype=torch.bool, device=DEV)
    keep[[3, 40, 64]] = False
    assert torch.equal(y[keep], y0[keep]) and torch.equal(z[keep], z0[keep])
    assert bool(z[3].isnan().all()) and bool(y[3].isnan().all())
    want = x2[[40, 64]].double() @ w.double().T + b.double()
    assert torch.equal(z[[40, 64]].double(), want)                # infinities of w's sign
    # and a weight of zero times infinity is no number
    w2 = w.clone()
    w2[7] = 0.0
    assert bool(NR.nr_linear(x2, w2)[40, 7].isnan())


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_linear_large_values(t):
    # the type's largest finite values, where partial results must not overflow
    dt = R.TYPES[t]
    big = torch.finfo(dt).max
    x = torch.zeros((5, 70), device=DEV, dtype=dt)
    w = torch.zeros((66, 70), device=DEV, dtype=dt)
    x[2, 9], w[4, 9], w[65, 9] = big, 1.0, -0.5
    x[1, 69], w[3, 69] = torch.finfo(dt).smallest_normal, 1.0
    y = NR.nr_linear(x, w)
    want = x.double() @ w.double().T
    assert torch.equal(y.double(), want)


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("m,k,n", [(5, 70, 66), (300, 512, 512), (4200, 256, 4104)])
def test_linear_small_values(m, k, n, t):
    # subnormal elements count as they are
    g = gen(m, k, n, t, "sub")
    dt = R.TYPES[t]
    f = torch.finfo(dt)
    x = (torch.randint(-200, 200, (m, k), generator=g, device=DEV).double()
         * (f.smallest_normal * f.eps)).to(dt)
    w = torch.randn((n, k), generator=g, device=DEV).to(dt) * 64
    check_linear(x, w, None, None, "none", *NR.nr_linear(x, w, pre=True))
    dy = rows(g, m, n, dt)
    dx, dw, db = NR.nr_linear_grad(dy, x, w)
    grad_check(dy, x, w, "none", None, (dx, dw, db), False)


def test_linear_small_values_fp32():
    # a float's parts are bf16: below 2^-110 the lowest of them are subnormal, and
    # what they lose is at most 2^-126 for an element
    g = gen("sub32")
    for e in (-100, -112, -125, -135):
        x = torch.randn((70, 96), generator=g, device=DEV) * 2.0 ** e
        w = torch.randn((40, 96), generator=g, device=DEV)
        y = NR.nr_linear(x, w)
        want = x.double() @ w.double().T
        tol = 98 * U * (x.double().abs() @ w.double().abs().T) + 2.0 ** -126 * w.double().abs().sum(1)
        close(y, want, tol + R.half_step(want, torch.float32), e)


# ---------------------------------------------------------------- 8 bits

def hold_values(t):
    g = gen(t, "hold")
    dt = R.TYPES[t]
    f = torch.finfo(dt)
    x = torch.randn((40, 77), generator=g, device=DEV)
    x[1] *= 1e3
    x[2] *= 1e-3
    x[3] = 0.0
    x[4, 33:] = 0.0
    x[5] = torch.linspace(-127.5, 127.5, 77, device=DEV)
    x[6] = torch.arange(77, device=DEV) - 38.5                    # ties
    x[7, 0], x[7, 1:] = 127.0, 0.5
    x[8, 0], x[8, 1:] = 448.0, 1.0 / 512
    x[9, 0], x[9, 1:32] = 464.0, torch.arange(31, device=DEV) * 2.0 ** -9
    x = x.to(dt)
    x[10] = f.max
    x[11, 40] = -f.max
    x[12] = f.smallest_normal
    x[13] = f.smallest_normal * f.eps * 3                         # subnormals
    x[14, 5] = math.nan
    x[15, 70] = math.inf
    x[16, 32], x[16, 33] = -math.inf, math.nan
    x[17] = torch.tensor(127.5, dtype=dt)
    x[18] = torch.nextafter(torch.tensor(127.5, device=DEV).to(dt), torch.tensor(0.0, device=DEV).to(dt))
    return x


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_hold(t, fmt):
    x = hold_values(t)
    for v in (x, x[:, 1:], x[:, :32], x[:, 3:4], x[:, ::1][:7], x[:1]):
        h = NR.nr_act_hold(v, fmt)
        val, byte = R.hold(v, fmt, v.dtype)
        assert torch.equal(h.scale.cpu().long(), byte)
        got = NR.nr_act_read(h)
        want = val.to(v.dtype)                                   # rounds fp16's subnormals only
        assert torch.equal(got.cpu().isnan(), want.isnan())
        assert torch.equal(got.cpu().nan_to_num(0.0), want.nan_to_num(0.0))
        # the bytes stand for the values, zeros behind the width
        q = h.q.float().cpu().double()
        s = torch.exp2(h.scale.cpu().double() - 127).repeat_interleave(32, 1)
        ok = (h.scale.cpu() != 255).repeat_interleave(32, 1)
        d = v.shape[1]
        assert torch.equal((q * s)[:, :d][ok[:, :d]], val[ok[:, :d]])
        assert not q[:, d:].any()
        for other in (torch.float32, torch.bfloat16):
            o = NR.nr_act_read(h, other)
            assert o.dtype == other and torch.equal(o.cpu().nan_to_num(0.0),
                                                    val.to(other).nan_to_num(0.0))


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_hold_error(t, fmt):
    # int8: off by at most half of 2^e; e4m3: by 2^-4 of the value, or half of
    # its smallest step 2^-9 of 2^e
    x = rows(gen(t, fmt), 200, 320, R.TYPES[t])
    h = NR.nr_act_hold(x, fmt)
    y = NR.nr_act_read(h, torch.float32).double()
    s = torch.exp2(h.scale.double() - 127).repeat_interleave(32, 1)
    tol = 0.5 * s if fmt == "i8" else torch.maximum(x.double().abs() * 2.0 ** -4, s * 2.0 ** -10)
    assert bool(((y - x.double()).abs() <= tol).all())


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n", [(1, 7, 5), (70, 65, 96), (300, 333, 129), (2000, 128, 256)])
def test_linear_held(m, k, n, t, fmt):
    g, dt, x, w, b, r = linear_case(m, k, n, t)
    dy = rows(g, m, n, dt, scale=0.1)
    for act in ("relu", "gelu"):
        y, z = NR.nr_linear(x, w, b, act=act, residual=r, pre=True)
        y2, hz = NR.nr_linear(x, w, b, act=act, residual=r, pre=fmt)
        assert torch.equal(y, y2)
        h = NR.nr_act_hold(z, fmt)                               # what the epilogue wrote
        assert torch.equal(h.scale, hz.scale)
        assert torch.equal(h.q.view(torch.uint8), hz.q.view(torch.uint8))
        # gradients from what is held are those of its values
        hx = NR.nr_act_hold(x, fmt)
        got = NR.nr_linear_grad(dy, hx, w, act=act, pre=hz)
        want = NR.nr_linear_grad(dy, NR.nr_act_read(hx), w, act=act, pre=NR.nr_act_read(hz))
        assert all(torch.equal(a, c) for a, c in zip(got, want))


# ---------------------------------------------------------------- layer norm

NORMS = [(1, 1), (1, 8), (3, 2), (5, 33), (64, 64), (70, 100), (33, 257), (130, 1536), (17, 1000),
         (9, 2049), (3, 4096), (2, 8200), (2, 16384), (3000, 128)]


def norm_case(m, d, t, pad=0, shift=0.5):
    g = gen(m, d, t, "n")
    dt = R.TYPES[t]
    x = rows(g, m, d, dt, pad) + 0
    if pad:
        x = torch.cat([x, x], 1)[:, :d]
    x += shift
    w = (1 + 0.3 * torch.randn(d, generator=g, device=DEV)).to(dt)
    b = (0.3 * torch.randn(d, generator=g, device=DEV)).to(dt)
    return g, dt, x, w, b


def check_norm(x, w, b, eps, y, stats):
    dt, d = y.dtype, x.shape[1]
    X = x.double()
    mu = X.mean(1, keepdim=True)
    var = ((X - mu) ** 2).mean(1, keepdim=True)
    rs = 1 / torch.sqrt(var + eps)
    tmu = (d + 2) * U * X.abs().mean(1, keepdim=True)
    # the variance: its own sum, and the mean's error squared plus roundings of x - mu
    trs = ((d + 8) * U / 2 + 2 * U) * rs + (tmu ** 2 + 4 * U * (X - mu).abs().mean(1, keepdim=True)
                                           * (tmu + U * X.abs().amax(1, keepdim=True))) * rs ** 3
    close(stats[0], mu[:, 0], tmu[:, 0] + 1e-300, "mean")
    close(stats[1], rs[:, 0], trs[:, 0], "rstd")
    c = X - mu
    W = w.double() if w is not None else torch.ones(d, device=DEV).double()
    Y = c * rs * W + (b.double() if b is not None else 0)
    t = W.abs() * ((tmu + U * X.abs()) * rs + c.abs() * trs + 3 * U * c.abs() * rs) + 2 * U * Y.abs()
    if b is not None:
        t = t + U * b.double().abs()
    close(y, Y, t + R.half_step(Y.abs() + t, dt), "y")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,d", NORMS)
def test_norm(m, d, t):
    g, dt, x, w, b = norm_case(m, d, t)
    for W, B in ((w, b), (None, None), (w, None)):
        y, stats = NR.nr_layer_norm(x, W, B, eps=1e-5, stats=True)
        check_norm(x, W, B, 1e-5, y, stats)
        assert torch.equal(NR.nr_layer_norm(x, W, B), y)
    for fx, fy in (("i8", None), (None, "e4m3"), ("e4m3", "i8")):
        out = NR.nr_layer_norm(x, w, None, hold_x=fx, hold_y=fy)
        held = list(out[1:])
        assert torch.equal(out[0], y)
        for f, src in ((fx, x), (fy, y)):
            if f is None:
                continue
            h, want = held.pop(0), NR.nr_act_hold(src, f)
            assert torch.equal(h.scale, want.scale)
            assert torch.equal(h.q.view(torch.uint8), want.q.view(torch.uint8))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("pad", [1, 5, 8])
def test_norm_strides(pad, t):
    for m, d in ((40, 96), (7, 333)):
        g = gen(m, d, pad)
        x = rows(g, m, d, R.TYPES[t], pad)
        w = rows(g, 1, d, R.TYPES[t])[0]
        y, stats = NR.nr_layer_norm(x, w, None, stats=True)
        check_norm(x, w, None, 1e-5, y, stats)
        c, cs = NR.nr_layer_norm(x.contiguous(), w, None, stats=True)
        assert torch.equal(c, y) and torch.equal(cs, stats)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_norm_values(t):
    # constant rows, a row far from zero, one with an infinity, eps of zero
    dt = R.TYPES[t]
    g, _, x, w, b = norm_case(40, 128, t)
    x[1] = 3.0
    x[2] = 0.0
    x[3] = 1000 + x[3]
    y, stats = NR.nr_layer_norm(x, w, b, stats=True)
    check_norm(x, w, b, 1e-5, y, stats)
    assert torch.equal(y[1], b) and torch.equal(y[2], b)
    x2 = x.clone()
    x2[4, 7], x2[5, 0] = math.inf, math.nan
    y2 = NR.nr_layer_norm(x2, w, b)
    keep = torch.ones(40, dtype=torch.bool, device=DEV)
    keep[[4, 5]] = False
    assert torch.equal(y2[keep], y[keep]) and bool(y2[4:6].isnan().all())
    y3, s3 = NR.nr_layer_norm(x[4:], w, b, eps=0.0, stats=True)
    check_norm(x[4:], w, b, 0.0, y3, s3)
    assert NR.nr_layer_norm(x[:0], w, b).shape == (0, 128)


def norm_grad_check(dy, x, stats, w, add, got):
    dt, d, m = dy.dtype, x.shape[1], x.shape[0]
    X, DY = x.double(), dy.double()
    mu, rs = stats[0].double()[:, None], stats[1].double()[:, None]
    W = w.double() if w is not None else torch.ones(d, device=DEV).double()
    xh = (X - mu) * rs
    txh = 3 * U * (xh.abs() + X.abs() * rs * 0)
    u = DY * W
    dx, dw, db = got
    if dx is not None:
        m1, m2 = u.mean(1, keepdim=True), (u * xh).mean(1, keepdim=True)
        a1, a2 = u.abs().mean(1, keepdim=True), (u * xh).abs().mean(1, keepdim=True)
        want = rs * (u - m1 - xh * m2)
        t = rs * (4 * U * u.abs() + (d + 4) * U * a1 + xh.abs() * (d + 10) * U * a2 + txh * a2
                  + 4 * U * (m1.abs() + (xh * m2).abs()))
        if add is not None:
            want = want + add.double()
            t = t + U * want.abs()
        close(dx, want, t + R.half_step(want.abs() + t, dt), "dx")
    if dw is not None:
        want, t = (DY * xh).sum(0), (m + 6) * U * (DY * xh).abs().sum(0)
        close(dw, want, t + R.half_step(want.abs() + t, dt), "dweight")
    if db is not None:
        want, t = DY.sum(0), (m + 2) * U * DY.abs().sum(0)
        close(db, want, t + R.half_step(want.abs() + t, dt), "dbias")


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,d", NORMS)
def test_norm_grad(m, d, t):
    g, dt, x, w, b = norm_case(m, d, t)
    dy, add = rows(g, m, d, dt, scale=0.1), rows(g, m, d, dt)
    y, stats = NR.nr_layer_norm(x, w, b, stats=True)
    for W, A in ((w, None), (None, add), (w, add)):
        got = NR.nr_layer_norm_grad(dy, x, stats, W, add=A)
        norm_grad_check(dy, x, stats, W, A, got)
        again = NR.nr_layer_norm_grad(dy, x, stats, W, add=A)
        assert all(torch.equal(a, c) for a, c in zip(got, again))
    for i in range(3):                                            # each alone: the same bits
        want = [False] * 3
        want[i] = True
        one = NR.nr_layer_norm_grad(dy, x, stats, w, add=add, dx=want[0], dweight=want[1],
                                    dbias=want[2])
        assert torch.equal(one[i], got[i]) and sum(v is not None for v in one) == 1
    for f in ("i8", "e4m3"):
        h = NR.nr_act_hold(x, f)
        a = NR.nr_layer_norm_grad(dy, h, stats, w, add=add)
        c = NR.nr_layer_norm_grad(dy, NR.nr_act_read(h), stats, w, add=add)
        assert all(torch.equal(p, q) for p, q in zip(a, c))


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
def test_norm_grad_strides_and_no_rows(t):
    for pad in (1, 5, 8):
        g = gen(pad)
        dt = R.TYPES[t]
        x, dy, add = rows(g, 40, 96, dt, pad), rows(g, 40, 96, dt, pad), rows(g, 40, 96, dt, pad)
        w = rows(g, 1, 96, dt)[0]
        y, stats = NR.nr_layer_norm(x, w, None, stats=True)
        norm_grad_check(dy, x, stats, w, add, NR.nr_layer_norm_grad(dy, x, stats, w, add=add))
    dx, dw, db = NR.nr_layer_norm_grad(dy[:0], x[:0], stats[:, :0].contiguous(), w)
    assert dx.shape == (0, 96) and not dw.any() and not db.any()


def test_norm_gradient_against_differences():
    g, dt, x, w, b = norm_case(12, 20, "f32")
    dy = rows(g, 12, 20, dt)
    y, stats = NR.nr_layer_norm(x, w, b, stats=True)
    dx, dw, db = NR.nr_layer_norm_grad(dy, x, stats, w)

    def f(X, W, B):
        c = X - X.mean(1, keepdim=True)
        return ((c / torch.sqrt((c * c).mean(1, keepdim=True) + 1e-5) * W + B) * dy.double()).sum()
    X, W, B = x.double(), w.double(), b.double()
    for grad, i in ((dx, 0), (dw, 1), (db, 2)):
        v = torch.randn(grad.shape, generator=g, device=DEV).double()
        h = 1e-4
        args = [[X, W, B], [X, W, B]]
        args[0][i], args[1][i] = args[0][i] + h * v, args[1][i] - h * v
        want = float((f(*args[0]) - f(*args[1])) / (2 * h))
        size = float((grad.double() * v).abs().sum())
        assert abs(float((grad.double() * v).sum()) - want) <= 1e-5 * size + 1e-6, i


# ---------------------------------------------------------------- streams, graphs

def block(x, w, b, gw, gb, dy, fmt, stream=None):
    """A residual block, forward and backward, its activations in 8 bits."""
    y1, st, hx, hy = NR.nr_layer_norm(x, gw, gb, stats=True, hold_x=fmt, hold_y=fmt, stream=stream)
    out, hz = NR.nr_linear(y1, w, b, act="gelu", residual=x, pre=fmt, stream=stream)
    d1, dw, db = NR.nr_linear_grad(dy, hy, w, act="gelu", pre=hz, stream=stream)
    dx, dg, dgb = NR.nr_layer_norm_grad(d1, hx, st, gw, add=dy, stream=stream)
    return [out, dx, dw, db, dg, dgb]


def block_inputs(m, d, t):
    g, dt, x, gw, gb = norm_case(m, d, t)
    return (x, rows(g, d, d, dt, scale=1 / math.sqrt(d)), rows(g, 1, d, dt)[0], gw, gb,
            rows(g, m, d, dt, scale=0.1))


@pytest.mark.parametrize("t,fmt", [("f32", "i8"), ("bf16", "e4m3"), ("f16", "i8")])
def test_block_on_another_stream(t, fmt):
    a = block_inputs(600, 160, t)
    want = block(*a, fmt)
    side = torch.cuda.Stream()
    for _ in range(3):
        torch.cuda.synchronize()
        with torch.cuda.stream(side):
            torch.cuda._sleep(20_000_000)
        got = block(*a, fmt, stream=side)
        junk = [torch.full((n,), 1e9, device="cuda") for n in (1 << 13, 1 << 16, 1 << 18, 1 << 20)]
        torch.cuda.synchronize()
        del junk
        assert all(torch.equal(p, q) for p, q in zip(got, want))


@pytest.mark.parametrize("t,fmt", [("f32", "e4m3"), ("bf16", "i8")])
@pytest.mark.parametrize("m", [1, 300])
def test_block_captured(m, t, fmt):
    # two graphs of the same calls, replayed between eager work on other inputs
    a = [v.clone() for v in block_inputs(m, 160, t)]
    want1 = [v.clone() for v in block(*a, fmt)]
    side = torch.cuda.Stream()
    graphs = []
    for _ in range(2):
        gr = torch.cuda.CUDAGraph()
        torch.cuda.synchronize()
        with torch.cuda.graph(gr, stream=side):
            out = block(*a, fmt)
        graphs.append((gr, out))
    x1 = a[0].clone()
    for rep in range(4):
        a[0].copy_(x1 if rep % 2 == 0 else x1 * 0.5)
        want = want1 if rep % 2 == 0 else block(*a, fmt)
        for gr, out in graphs:
            gr.replay()
        for gr, out in graphs:
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(out, want)), rep


def test_two_streams_at_once():
    a, c = block_inputs(900, 256, "bf16"), block_inputs(500, 192, "bf16")
    wa, wc = block(*a, "i8"), block(*c, "i8")
    s1, s2 = torch.cuda.Stream(), torch.cuda.Stream()
    torch.cuda.synchronize()
    for _ in range(4):
        ga, gc = block(*a, "i8", stream=s1), block(*c, "i8", stream=s2)
    torch.cuda.synchronize()
    assert all(torch.equal(p, q) for p, q in zip(ga + gc, wa + wc))


# ---------------------------------------------------------------- refusals

def test_wrong_tensors_are_refused():
    x, w = torch.rand((8, 6), device=DEV), torch.rand((5, 6), device=DEV)
    b, r, dy = torch.rand(5, device=DEV), torch.rand((8, 5), device=DEV), torch.rand((8, 5), device=DEV)
    NR.nr_linear(x, w, b, residual=r)
    bad = [dict(x=x.cpu()), dict(x=x.double()), dict(x=x[0]), dict(x=x.T), dict(x=x.int()),
           dict(x=x[:, :5]), dict(w=w.half()), dict(w=w.T), dict(w=w.cpu()), dict(w=w[0]),
           dict(bias=b[:4]), dict(bias=b.half()), dict(bias=b[None]), dict(bias=b.cpu()),
           dict(residual=r[:7]), dict(residual=r.half()), dict(residual=r[:1].expand(8, 5)),
           dict(x=x[:1].expand(8, 6)), dict(act="tanh"), dict(pre="fp8"), dict(pre=1)]
    for kw in bad:
        args = dict(x=x, w=w, bias=b, residual=r)
        args.update(kw)
        with pytest.raises(ValueError):
            NR.nr_linear(**args)
    z = torch.rand((8, 5), device=DEV)
    hx, hz = NR.nr_act_hold(x), NR.nr_act_hold(z)
    NR.nr_linear_grad(dy, hx, w, "gelu", hz)
    for a in ((dy, hz, w, "gelu", z), (dy, x, w, "gelu", None), (dy, x, w, "gelu", hx),
              (dy, None, w, "none", None), (dy, x, None, "none", None), (dy, x.half(), w, "none"),
              (dy, NR.nr_act_hold(x.half()), w, "none"), (dy[:7], x, w, "none"),
              (dy, x, w.T, "none"), (dy, x, w, "gelu", z[:, :4])):
        with pytest.raises(ValueError):
            NR.nr_linear_grad(*a)
    st = torch.rand((2, 8), device=DEV)
    NR.nr_layer_norm_grad(x, x, st)
    for a in ((x, x, st[:, :7]), (x, x, st.double()), (x, x, st.T), (x, hz, st), (x, w, st),
              (x, x, st, b), (x, x.half(), st)):
        with pytest.raises(ValueError):
            NR.nr_layer_norm_grad(*a)
    with pytest.raises(ValueError):
        NR.nr_layer_norm_grad(x, x, st, add=r)
    for kw in (dict(hold_x="i4"), dict(hold_y="e5m2"), dict(weight=b), dict(bias=b)):
        with pytest.raises(ValueError):
            NR.nr_layer_norm(x, **kw)
    for eps in (-1.0, math.nan, math.inf):
        with pytest.raises(NR.NRError):
            NR.nr_layer_norm(x, eps=eps)
    with pytest.raises(ValueError):
        NR.nr_act_hold(x, "i4")
    with pytest.raises(ValueError):
        NR.nr_act_read(hx, torch.float64)
    wide = torch.zeros((2, 16385), device=DEV)
    for call in (lambda: NR.nr_layer_norm(wide), lambda: NR.nr_act_hold(wide),
                 lambda: NR.nr_linear(wide, wide[:1])):
        with pytest.raises(NR.NRError) as e:
            call()
        assert e.value.status == NR.NR_EUNSUPPORTED
