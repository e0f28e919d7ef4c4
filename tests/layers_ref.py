"""Plain 64-bit forms of the layers (CPU or GPU tensors), for the tests."""
import math

import torch

TYPES = {"f32": torch.float32, "bf16": torch.bfloat16, "f16": torch.float16}
U = 2.0 ** -24                       # half a step of fp32, relative


def act(z, name):
    if name == "relu":
        return torch.where(z > 0, z, torch.zeros_like(z))
    if name == "gelu":
        return 0.5 * z * torch.special.erfc(-z / math.sqrt(2.0))
    if name == "silu":
        return z * torch.sigmoid(z)
    return z


def slope(z, name):
    if name == "relu":
        return (z > 0).double()
    if name == "gelu":
        return (0.5 * torch.special.erfc(-z / math.sqrt(2.0))
                + z * torch.exp(-0.5 * z * z) / math.sqrt(2 * math.pi))
    if name == "silu":
        p = torch.sigmoid(z)
        return p + z * p * torch.sigmoid(-z)
    return torch.ones_like(z)


def half_step(v, dtype):
    """What rounding v to the type can change it by: half a step, and half the
    type's smallest number near zero."""
    f = torch.finfo(dtype)
    return v.abs() * (f.eps / 2) + f.smallest_normal * f.eps / 2


def hold(x, fmt, dtype):
    """(values, q, scale byte) of x [m, d] (any float type) in 8 bits, element by
    element from the definition; all arithmetic is exact in 64 bits."""
    m, d = x.shape
    ldq = (d + 31) // 32 * 32
    v = torch.zeros((m, ldq), dtype=torch.float64)
    v[:, :d] = x.detach().cpu().double()
    val = torch.zeros_like(v)
    byte = torch.zeros((m, ldq // 32), dtype=torch.int64)
    half = dtype == torch.float16
    lo, hi = -126, {("i8", False): 121, ("e4m3", False): 119, ("i8", True): 9,
                    ("e4m3", True): 7}[(fmt, half)]
    for r in range(m):
        for g in range(ldq // 32):
            s = v[r, 32 * g:32 * g + 32]
            if not bool(torch.isfinite(s).all()):
                byte[r, g] = 255
                val[r, 32 * g:32 * g + 32] = math.nan
                continue
            big = float(s.abs().max())
            e = lo
            while e < hi and not (big * 2.0 ** -e < 127.5 if fmt == "i8" else big * 2.0 ** -e <= 448):
                e += 1
            byte[r, g] = e + 127
            u = s * 2.0 ** -e
            if fmt == "i8":
                q = torch.round(u).clamp(-127, 127)           # ties to even
            else:
                u = u.clamp(-448, 448)
                ex = torch.frexp(u)[1].double() - 1           # floor(log2 |u|)
                st = 2.0 ** (ex.clamp_min(-6) - 3)
                q = torch.round(u / st) * st
            val[r, 32 * g:32 * g + 32] = q * 2.0 ** e
    return val[:, :d], byte
