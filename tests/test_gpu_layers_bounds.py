"""The layers' C entry points write their outputs and nothing else: strided
outputs inside larger buffers, work space of just the size asked for, at sizes
that reach each way of taking the products (small tiles, large ones, parts of k,
copied rows)."""
import ctypes as C

import pytest
import torch

from paper_2608_15438_amd import neuroute as NR
from tests import layers_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"
MARK = 0x5A


class Guard:
    """Outputs [m, w] with a row stride of w + gap in a buffer of marks."""

    def __init__(self):
        self.items = []

    def out(self, m, w, dtype, gap=3, front=16):
        e = torch.empty(0, dtype=dtype).element_size()
        n = front * e + m * (w + gap) * e + 64
        raw = torch.full((n,), MARK, dtype=torch.uint8, device=DEV)
        body = raw[front * e:front * e + m * (w + gap) * e].view(dtype).view(m, w + gap)
        self.items.append((raw, body, front * e, w))
        return body

    def work(self, nbytes):
        raw = torch.full((nbytes + 1024,), MARK, dtype=torch.uint8, device=DEV)
        self.items.append((raw, None, nbytes, 0))
        return raw.data_ptr()

    def check(self):
        torch.cuda.synchronize()
        for raw, body, at, w in self.items:
            if body is None:
                assert bool((raw[at:] == MARK).all()), "work space overrun"
                continue
            assert bool((raw[:at] == MARK).all()) and bool((raw[-64:] == MARK).all())
            gaps = body[:, w:].contiguous().view(torch.uint8)
            assert bool((gaps == MARK).all()), "between the rows"


def ptr(t):
    return t.data_ptr()


def run(name, desc, guard):
    L = NR.lib()
    need = getattr(L, name + "_ws")(C.byref(desc))
    ws = guard.work(need) if need else None
    assert getattr(L, name)(C.byref(desc), ws, need, torch.cuda.current_stream().cuda_stream) == 0


SIZES = [(1, 40, 24), (7, 4096, 96), (65, 33, 70), (300, 300, 300), (5000, 72, 136),
         (4200, 200, 4104), (3000, 601, 515), (40_000, 64, 40)]


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,k,n", SIZES)
def test_linear_writes_its_outputs_only(m, k, n, t):
    dt = R.TYPES[t]
    g = torch.Generator(device=DEV).manual_seed(m + k + n)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).to(dt)
    x, w, b, dy = r(m, k), r(n, k), r(n), r(m, n)
    want_y, want_z = NR.nr_linear(x, w, b, act="gelu", pre=True)
    G = Guard()
    y, z = G.out(m, n, dt), G.out(m, n, dt, gap=5)
    d = NR.nr_linear_desc(m, n, k, NR.LAYER_DTYPES[dt], 2, ptr(x), k, ptr(w), k, ptr(b), None, 0,
                          ptr(y), n + 3, ptr(z), n + 5, 0, None)
    run("nr_linear", d, G)
    G.check()
    assert torch.equal(y[:, :n], want_y) and torch.equal(z[:, :n], want_z)
    want = NR.nr_linear_grad(dy, x, w, "gelu", want_z)
    G = Guard()
    dx, dw, db = G.out(m, k, dt), G.out(n, k, dt, gap=1), G.out(1, n, dt)
    e = NR.nr_linear_grad_desc(m, n, k, NR.LAYER_DTYPES[dt], 2, ptr(dy), n, ptr(x), k, 0, None,
                               ptr(w), k, ptr(want_z), n, 0, None, ptr(dx), k + 3, ptr(dw), k + 1,
                               ptr(db))
    run("nr_linear_grad", e, G)
    G.check()
    for got, exp, c in ((dx, want[0], k), (dw, want[1], k), (db, want[2][None], n)):
        assert torch.equal(got[:, :c], exp)


@pytest.mark.parametrize("t", ["f32", "bf16", "f16"])
@pytest.mark.parametrize("m,d", [(1, 5), (70, 33), (300, 257), (33, 1537), (9, 5000), (3, 16384)])
def test_norm_writes_its_outputs_only(m, d, t):
    dt = R.TYPES[t]
    g = torch.Generator(device=DEV).manual_seed(m + d)
    r = lambda *s: torch.randn(s, generator=g, device=DEV).to(dt)
    x, w, b, dy = r(m, d), r(d), r(d), r(m, d)
    want_y, st, hx, hy = NR.nr_layer_norm(x, w, b, stats=True, hold_x="i8", hold_y="e4m3")
    G = Guard()
    y, stats = G.out(m, d, dt), G.out(1, 2 * m, torch.float32, gap=0)
    ldq = (d + 31) // 32 * 32
    xq, yq = (G.out(m, ldq, torch.uint8, gap=0, front=16) for _ in range(2))
    xs, ys = (G.out(m, ldq // 32, torch.uint8, gap=0) for _ in range(2))
    e = NR.nr_layer_norm_desc(m, d, NR.LAYER_DTYPES[dt], 1e-5, ptr(x), d, ptr(w), ptr(b), ptr(y),
                              d + 3, ptr(stats), 1, 2, ptr(xq), ptr(xs), ptr(yq), ptr(ys))
    assert NR.lib().nr_layer_norm(C.byref(e), torch.cuda.current_stream().cuda_stream) == 0
    G.check()
    assert torch.equal(y[:, :d], want_y) and torch.equal(stats.view(2, m), st)
    assert torch.equal(xq, hx.q.view(torch.uint8)) and torch.equal(ys, hy.scale)
    want = NR.nr_layer_norm_grad(dy, x, st, w)
    G = Guard()
    dx, dg, db = G.out(m, d, dt), G.out(1, d, dt), G.out(1, d, dt)
    e = NR.nr_layer_norm_grad_desc(m, d, NR.LAYER_DTYPES[dt], ptr(dy), d, ptr(x), d, 0, None,
                                   ptr(st), ptr(w), None, 0, ptr(dx), d + 3, ptr(dg), ptr(db))
    run("nr_layer_norm_grad", e, G)
    G.check()
    for got, exp in ((dx, want[0]), (dg, want[1][None]), (db, want[2][None])):
        assert torch.equal(got[:, :d], exp)


@pytest.mark.parametrize("fmt", [1, 2])
@pytest.mark.parametrize("m,d", [(1, 1), (65, 31), (300, 100), (1000, 64)])
def test_hold_writes_its_outputs_only(m, d, fmt):
    x = torch.randn((m, d), device=DEV)
    G = Guard()
    ldq = (d + 31) // 32 * 32
    q, s = G.out(m, ldq, torch.uint8, gap=0), G.out(m, ldq // 32, torch.uint8, gap=0)
    stream = torch.cuda.current_stream().cuda_stream
    assert NR.lib().nr_act_hold(ptr(x), d, m, d, NR.NR_F32, fmt, ptr(q), ptr(s), stream) == 0
    y = G.out(m, d, torch.bfloat16, gap=7)
    assert NR.lib().nr_act_read(ptr(q), ptr(s), m, d, fmt, NR.NR_BF16, ptr(y), d + 7, stream) == 0
    G.check()
    h = NR.nr_act_hold(x, {1: "i8", 2: "e4m3"}[fmt])
    assert torch.equal(h.scale, s) and torch.equal(NR.nr_act_read(h, torch.bfloat16), y[:, :d])
