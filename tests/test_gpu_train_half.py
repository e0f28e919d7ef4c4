"""Encoder training in fp16: the gradients that the optimizer is handed, beside
those of fp32, for losses from ordinary to small ones, whose gradients are below
fp16's range."""
import math

import numpy as np
import pytest
import torch

from paper_2608_15438_amd import train as TR
from paper_2608_15438_amd.index_build import Encoder

pytestmark = pytest.mark.gpu
DEV = "cuda"


def encoder(widths, shrink):
    r = np.random.default_rng(1)
    ws = [r.standard_normal((n, k)).astype(np.float32) / math.sqrt(k)
          for k, n in zip(widths, widths[1:])]
    return Encoder(weights=ws, input_scale=shrink / 255,
                   biases=[(0.1 * shrink * r.standard_normal(len(w))).astype(np.float32) for w in ws])


def grads(monkeypatch, enc, steps=1, **kw):
    """What Adam is handed, step by step, and the trained encoder."""
    seen = []

    class Adam(torch.optim.Adam):
        def step(self, *a, **k):
            seen.append([p.grad.detach().double().clone() for g in self.param_groups
                         for p in g["params"]])
            return super().step(*a, **k)
    monkeypatch.setattr(TR.torch.optim, "Adam", Adam)
    g = torch.Generator(device=DEV).manual_seed(3)
    base = torch.randint(0, 256, (1000, enc.weights[0].shape[1]), generator=g, device=DEV)
    out = TR.train_encoder(enc, lambda ids: base[ids], n=1000, steps=steps, batch=1000, device=DEV,
                           layers="hip", **kw)
    monkeypatch.undo()
    return seen, out


# fp16 rounds each tensor handed on, at most eight in a row, by 2^-11, together
# 2^-8; the loss's residuals S_lat - gamma rho S_emb are some times smaller than the
# latents' distances and magnify a latent's rounding by as much: 2^-6.  The last
# bias's gradient is zero up to roundings (adding a vector to all latents changes no
# difference) and is left out
@pytest.mark.parametrize("shrink", [1.0, 1e-2, 1e-3])
@pytest.mark.parametrize("widths", [(128, 256, 24), (96, 200, 64, 20)])
def test_gradients(monkeypatch, widths, shrink):
    enc = encoder(widths, shrink)
    (want,), _ = grads(monkeypatch, enc)
    (got,), _ = grads(monkeypatch, enc, dtype=torch.float16)
    for a, b in list(zip(got, want))[:-1]:
        assert float((a - b).norm()) <= 2.0 ** -6 * float(b.norm()), (shrink, a.shape)


def test_a_step_that_overflows_is_left_out(monkeypatch):
    # gradients past fp16's range: the parameters wait until the scale fits
    enc = encoder((64, 96, 12), 1.0)
    enc.weights[1] *= 30
    seen, out = grads(monkeypatch, enc, steps=16, dtype=torch.float16)
    assert 0 < len(seen) < 16
    assert all(bool(v.isfinite().all()) for s in seen for v in s)
    assert all(np.isfinite(v).all() for v in out.weights + out.biases)
    assert not np.array_equal(out.weights[0], enc.weights[0])


def test_wider_types_are_not_scaled(monkeypatch):
    # one backward pass and one step, as before, in fp32 and bf16
    enc = encoder((64, 96, 12), 1.0)
    for dtype in (torch.float32, torch.bfloat16):
        seen, _ = grads(monkeypatch, enc, steps=3, dtype=dtype)
        assert len(seen) == 3
