"""fp32 products next to infinities: an output that is not finite is made again by
a chain of fp32, the finite ones beside it in its row keep their bits."""
import math

import pytest
import torch

from paper_2608_15438_amd import neuroute as NR

pytestmark = pytest.mark.gpu
DEV = "cuda"


def rnd(seed, *shape):
    g = torch.Generator(device=DEV).manual_seed(seed)
    return torch.randn(shape, generator=g, device=DEV)


@pytest.mark.parametrize("m,k,n", [(5, 70, 66), (300, 333, 129), (7, 4096, 96), (4200, 520, 1032)])
def test_neighbours_keep_their_bits(m, k, n):
    x, w, dy = rnd(1, m, k), rnd(2, n, k), rnd(3, m, n)
    w2, x2, dy2 = w.clone(), x.clone(), dy.clone()
    cols = torch.arange(3, n, 11, device=DEV)
    w2[cols, 1] = math.inf                    # these columns of y, for every row
    y, y2 = NR.nr_linear(x, w), NR.nr_linear(x, w2)
    keep = torch.ones(n, dtype=torch.bool, device=DEV)
    keep[cols] = False
    assert torch.equal(y2[:, keep], y[:, keep])
    want = x[:, 1:2].double().expand(m, len(cols)) * math.inf
    assert torch.equal(y2[:, cols].double(), want)
    some = torch.arange(2, k, 13, device=DEV)
    x2[m // 2, some] = -math.inf              # these columns of dw
    dw, dw2 = NR.nr_linear_grad(dy, x, w, db=False)[1], NR.nr_linear_grad(dy, x2, w, db=False)[1]
    keep = torch.ones(k, dtype=torch.bool, device=DEV)
    keep[some] = False
    assert torch.equal(dw2[:, keep], dw[:, keep])
    want = (dy[m // 2].double() * -math.inf)[:, None].expand(n, len(some))
    assert torch.equal(dw2[:, some].double(), want)


@pytest.mark.parametrize("fmt", ["i8", "e4m3"])
@pytest.mark.parametrize("m,k,n", [(9, 37, 21), (300, 333, 129), (4200, 520, 1032)])
def test_chain_of_held_rows_and_large_sums(m, k, n, fmt):
    # sums that leave the range: an infinity of the terms' sign; rows held in 8
    # bits beside a group that is NaN
    dy = torch.zeros((m, n), device=DEV)
    x = rnd(4, m, k).abs() + 1
    dy[:, 2] = 3e38 if m < 100 else 3e36
    dy[:, n - 1] = -dy[:, 2]
    x[m - 1, 0] = math.nan                    # the group of the first 32 columns of its row
    dx, dw, db = NR.nr_linear_grad(dy, NR.nr_act_hold(x, fmt), rnd(5, n, k))
    assert bool(dw[:, :32].isnan().all())
    want = torch.zeros_like(dw[:, 32:])
    want[2], want[n - 1] = math.inf, -math.inf
    assert torch.equal(dw[:, 32:], want)
