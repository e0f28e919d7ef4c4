"""16-bit operands of large products that start off a 16-byte boundary, their rows'
stride a multiple of it: each alone and all of them, against 64 bits, and the same
bits on every call laid out the same (another layout may take another path)."""
import pytest
import torch

from paper_2608_15438_amd import neuroute as NR
from tests import layers_ref as R
from tests.test_gpu_layers import check_linear, gen, grad_check, rows

pytestmark = pytest.mark.gpu
DEV = "cuda"


def shifted(t, at):
    """t's values in a wider array, `at` elements in."""
    wide = torch.zeros((t.shape[0], t.shape[1] + 16), dtype=t.dtype, device=DEV)
    v = wide[:, at:at + t.shape[1]]
    v.copy_(t)
    return v


@pytest.mark.parametrize("t", ["bf16", "f16"])
@pytest.mark.parametrize("m,k,n", [(16_384, 512, 512), (4200, 200, 4104), (2000, 1000, 2000)])
@pytest.mark.parametrize("at", [1, 4])
def test_starts(m, k, n, t, at):
    dt = R.TYPES[t]
    g = gen(m, k, n, t, "at")
    x, w, dy = rows(g, m, k, dt), rows(g, n, k, dt, scale=k ** -0.5), rows(g, m, n, dt, scale=0.1)
    b = rows(g, 1, n, dt)[0]
    sx, sw, sd = shifted(x, at), shifted(w, at), shifted(dy, at)
    assert all(v.data_ptr() % 16 and v.stride(0) % 8 == 0 for v in (sx, sw, sd))
    z = NR.nr_linear(x, w, b, act="gelu", pre=True)[1]
    for a, c in ((sx, w), (x, sw), (sx, sw)):
        y, u = NR.nr_linear(a, c, b, act="gelu", pre=True)
        check_linear(x, w, b, None, "gelu", y, u)
        assert all(torch.equal(p, q)
                   for p, q in zip(NR.nr_linear(a, c, b, act="gelu", pre=True), (y, u)))
    for act, pre in (("none", None), ("gelu", z)):
        for a, c, d in ((sd, x, w), (dy, sx, w), (dy, x, sw), (sd, sx, sw)):
            got = NR.nr_linear_grad(a, c, d, act=act, pre=pre)
            grad_check(dy, x, w, act, pre, got, act != "none")
            again = NR.nr_linear_grad(a, c, d, act=act, pre=pre)
            assert all(torch.equal(p, q) for p, q in zip(got, again))
