"""The differentiable layers and encoder training on them: gradients against
torch's own autograd in 64 bits, what is kept for the backward pass, layouts."""
import math

import numpy as np
import pytest
import torch

from paper_2608_15438_amd import layers as LY
from paper_2608_15438_amd import neuroute as NR
from paper_2608_15438_amd import train as TR
from paper_2608_15438_amd.index_build import Encoder
from tests import layers_ref as R

pytestmark = pytest.mark.gpu
DEV = "cuda"


def near(got, want, rel, what):
    err, size = (got.double() - want).norm(), want.norm()
    err, size = float(err.detach()), float(size.detach())
    assert err <= rel * size + 1e-30, (what, err / max(size, 1e-300))


# How far a whole gradient may be off, in the 2-norm: fp32 sums of up to some
# hundred terms, a few layers deep, 1e-5; with bf16 (half a step 2^-9 relative on
# the mean) a rounding per tensor handed on, at most eight of them in a row and
# their effects added, 8 x 2^-8
REL = {torch.float32: 1e-5, torch.bfloat16: 2.0 ** -5}


def net(x, p, lin, norm):
    h = lin(x, p["w0"], p["b0"], "gelu", None)
    for i in (1, 2):
        h = lin(norm(h, p[f"g{i}"], p[f"n{i}"]), p[f"w{i}"], p[f"b{i}"], "silu", h)
    return lin(h, p["w3"], None, "none", None)


def params(dtype, k=24, d=40, out=12):
    g = torch.Generator(device=DEV).manual_seed(5)
    r = lambda *s: torch.randn(s, generator=g, device=DEV)
    p = dict(w0=r(d, k) / math.sqrt(k), b0=r(d) * 0.1, w3=r(out, d) / math.sqrt(d))
    for i in (1, 2):
        p.update({f"w{i}": r(d, d) / math.sqrt(d), f"b{i}": r(d) * 0.1,
                  f"g{i}": 1 + 0.1 * r(d), f"n{i}": 0.1 * r(d)})
    x = r(6, 50, k)
    return ({n: v.to(dtype).requires_grad_(True) for n, v in p.items()},
            x.to(dtype).requires_grad_(True), r(6, 50, out).to(dtype))


def wide(p, x):
    q = {n: v.detach().double().requires_grad_(True) for n, v in p.items()}
    return q, x.detach().double().requires_grad_(True)


def plain_linear(x, w, b, act, r):
    z = x @ w.T
    y = R.act(z if b is None else z + b, act)
    return y if r is None else y + r


def plain_norm(x, g, b):
    c = x - x.mean(-1, keepdim=True)
    return c / torch.sqrt((c * c).mean(-1, keepdim=True) + 1e-5) * g + b


@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
def test_network_gradients(dtype):
    p, x, dy = params(dtype)
    out = net(x, p, lambda x, w, b, act, r: LY.linear(x, w, b, act, r), LY.layer_norm)
    out.backward(dy)
    q, xd = wide(p, x)
    want = net(xd, q, plain_linear, plain_norm)
    want.backward(dy.double())
    near(out, want, REL[dtype], "out")
    near(x.grad, xd.grad, REL[dtype], "x")
    for n in p:
        assert p[n].grad.dtype == dtype and p[n].grad.shape == p[n].shape
        near(p[n].grad, q[n].grad, REL[dtype], n)


# int8: off by up to 1/127 of a group's largest, about 1/40 of its typical
# magnitude; e4m3 by up to 2^-4 of the value: with the roundings' spread below a
# half of that, and a few of them met in a gradient
@pytest.mark.parametrize("hold,rel", [("i8", 0.05), ("e4m3", 0.125)])
def test_network_gradients_held(hold, rel):
    p, x, dy = params(torch.float32)
    net(x, p, lambda x, w, b, act, r: LY.linear(x, w, b, act, r, hold=hold),
        lambda x, g, b: LY.layer_norm(x, g, b, hold=hold)).backward(dy)
    held = {n: v.grad.clone() for n, v in p.items()}
    q, xd = wide(p, x)
    net(xd, q, plain_linear, plain_norm).backward(dy.double())
    for n in p:
        near(held[n], q[n].grad, rel, n)
    near(x.grad, xd.grad, rel, "x")


def test_each_input_alone_and_frozen_ones():
    p, x, dy = params(torch.float32)
    r = torch.randn((6, 50, 40), device=DEV, requires_grad=True)
    ins = dict(x=x, w=p["w0"], b=p["b0"], r=r)
    full = LY.linear(x, p["w0"], p["b0"], "gelu", r)
    d = torch.randn_like(full)
    full.backward(d)
    want = {n: v.grad.clone() for n, v in ins.items()}
    for only in ins:
        a = {n: v.detach().requires_grad_(n == only) for n, v in ins.items()}
        LY.linear(a["x"], a["w"], a["b"], "gelu", a["r"]).backward(d)
        for n, v in a.items():
            assert (v.grad is not None) == (n == only)
        assert torch.equal(a[only].grad, want[only])
    with torch.no_grad():
        assert torch.equal(LY.linear(x, p["w0"], p["b0"], "gelu", r), full)


def test_layouts():
    # transposed, expanded and broadcast inputs and gradients
    w = torch.randn((16, 24), device=DEV, requires_grad=True)
    base = torch.randn((24, 30), device=DEV)
    x = base.T.requires_grad_(True)
    y = LY.linear(x, w, act="relu")
    y.sum().backward()                                  # dy: an expanded scalar
    xd, wd = x.detach().double().requires_grad_(True), w.detach().double().requires_grad_(True)
    (xd @ wd.T).clamp_min(0).sum().backward()
    near(x.grad, xd.grad, 1e-6, "x")
    near(w.grad, wd.grad, 1e-6, "w")
    e = torch.randn((1, 24), device=DEV).expand(5, 24)
    assert torch.equal(LY.linear(e, w)[0], LY.linear(e.contiguous(), w)[0])
    v = torch.randn(24, device=DEV)
    assert LY.linear(v, w).shape == (16,) and LY.layer_norm(v).shape == (24,)
    n = LY.layer_norm(x.detach())
    near(n, torch.nn.functional.layer_norm(x.detach().double(), (24,)), 1e-6, "norm")
    assert LY.linear(x[:0], w).shape == (0, 16)
    LY.linear(x[:0], w, act="gelu").sum().backward()


def test_what_is_kept():
    x = torch.randn((512, 256), device=DEV, requires_grad=True)
    w = torch.randn((256, 256), device=DEV, requires_grad=True)
    saved = lambda y: sum(t.numel() * t.element_size() for t in y.grad_fn.saved_tensors
                          if t is not None and t.data_ptr() != w.data_ptr())
    whole, held = LY.linear(x, w, act="gelu"), LY.linear(x, w, act="gelu", hold="i8")
    assert torch.equal(whole, held)
    assert saved(whole) == 2 * 512 * 256 * 4
    assert saved(held) == 2 * 512 * 256 * 33 // 32
    y = LY.linear(x, w, act="relu")                      # its own output serves
    assert any(t.data_ptr() == y.data_ptr() for t in y.grad_fn.saved_tensors)
    assert saved(LY.layer_norm(x, hold="e4m3")) == 512 * 256 * 33 // 32 + 2 * 512 * 4
    y.backward(torch.ones_like(y))
    y = LY.linear(x, w, act="relu")
    y.data_ptr()
    with torch.no_grad():
        y += 1                                           # what the backward pass needs
    with pytest.raises(RuntimeError):
        y.sum().backward()


def test_refusals():
    x, w = torch.randn((4, 8), device=DEV), torch.randn((5, 8), device=DEV)
    for call in (lambda: LY.linear(x, w, hold="i4"), lambda: LY.layer_norm(x, hold="f8"),
                 lambda: LY.linear(x, w, residual=torch.randn(5, device=DEV)),
                 lambda: LY.linear(x, w, act="tanh"), lambda: LY.linear(x.cpu(), w),
                 lambda: LY.linear(x, w.half()), lambda: LY.linear(x[0, 0], w)):
        with pytest.raises(ValueError):
            call()
    y = LY.linear(x.requires_grad_(True), w, act="gelu")
    g, = torch.autograd.grad(y.sum(), x, create_graph=True)
    with pytest.raises(RuntimeError):
        g.sum().backward()


def encoder(widths, seed=1):
    r = np.random.default_rng(seed)
    ws = [r.standard_normal((n, k)).astype(np.float32) / math.sqrt(k)
          for k, n in zip(widths, widths[1:])]
    return Encoder(weights=ws, biases=[0.1 * r.standard_normal(len(w)).astype(np.float32) for w in ws],
                   input_scale=1 / 255)


def loss_grads(layers, dtype, hold, x, enc):
    m = TR._Mlp(enc, DEV, layers, dtype, hold)
    lat = m(x)
    lat.retain_grad()
    loss, tau, _ = TR.lsim_loss_gpu(x * enc.input_scale, lat, 0.6, 1.5)
    loss.backward()
    return float(loss.detach()), [q.grad for q in m.parameters()], lat.grad


@pytest.mark.parametrize("widths", [(128, 256, 24), (96, 200, 64, 20)])
def test_training_step_on_the_kernels(widths):
    # one step's gradients of the encoder: fp32 layers like torch's (both sum in
    # fp32; the loss is the same kernel on latents some 1e-6 apart, at whose mask's
    # border a pair in some thousand may change sides: 1e-3)
    enc = encoder(widths)
    g = torch.Generator(device=DEV).manual_seed(2)
    x = torch.randint(0, 256, (1000, widths[0]), generator=g, device=DEV).float()
    l0, g0, d0 = loss_grads("torch", torch.float32, None, x, enc)
    l1, g1, d1 = loss_grads("hip", torch.float32, None, x, enc)
    assert abs(l0 - l1) <= 1e-3 * abs(l0)
    for a, b in zip(g0[:-1], g1[:-1]):
        near(b, a.double(), 1e-3, "grad")
    # the loss sees differences of latents only, so adding one vector to them all
    # leaves it: the last bias's gradient, the sum of the latents' gradients, is
    # zero, and what is there are roundings.  A latent's own gradient is a sum of up
    # to m terms (and each term stands in two latents' sums with opposite signs), so
    # m 2^-24 of the magnitudes from there and as much from the column sum
    for b, d in ((g0[-1], d0), (g1[-1], d1)):
        assert bool((b.double().abs() <= 2 * 1000 * R.U * d.double().abs().sum(0)).all())
    for dtype, hold in ((torch.float32, "i8"), (torch.bfloat16, None), (torch.bfloat16, "e4m3")):
        l2, g2, _ = loss_grads("hip", dtype, hold, x, enc)
        assert math.isfinite(l2) and all(bool(t.isfinite().all()) for t in g2)


@pytest.mark.parametrize("dtype,hold", [(torch.float32, None), (torch.bfloat16, "i8")])
def test_train_encoder_on_the_kernels(dtype, hold):
    enc = encoder((64, 96, 12))
    g = torch.Generator(device=DEV).manual_seed(3)
    base = torch.randint(0, 256, (4000, 64), generator=g, device=DEV).to(torch.uint8)
    kw = dict(n=4000, steps=3, batch=512, layers="hip", dtype=dtype, hold=hold)
    a = TR.train_encoder(enc, lambda ids: base[ids], **kw)
    b = TR.train_encoder(enc, lambda ids: base[ids], **kw)
    for u, v in zip(a.weights + a.biases, b.weights + b.biases):
        assert u.dtype == np.float32 and np.array_equal(u, v)     # reproducible
    assert not np.array_equal(a.weights[0], enc.weights[0])
