"""Differentiable layers on the library's kernels (nr_linear, nr_layer_norm and
their gradients): what an encoder is trained with, or one that no index holds is
run with (its latents go to Index.nr_search as `logits`).

Tensors are device tensors [..., width] of float32, bfloat16 or float16, all of
a call's of one type.  `hold` ("i8" or "e4m3") keeps what the backward pass needs
of the activations in 8 bits (nr_act_hold: a power of two per 32 elements): half
of bfloat16's memory, a quarter of float32's.  A linear layer's gradients are then
those at the held values; a layer norm's take the held row with the mean and the
deviation of the row itself, which it keeps in fp32.  Under torch.no_grad() nothing
is kept or put into 8 bits (needs_input_grad says which inputs want gradients there
too, so the layers pass the grad mode on).

Gradients have the tensors' type: in float16, whose smallest number is 6e-8, scale
the loss (torch.amp.GradScaler).  Double backward is not supported.
"""
from __future__ import annotations

import math
from typing import Optional

import torch
from torch.autograd.function import once_differentiable

from . import neuroute as NR


def _rows(t: torch.Tensor, name: str) -> torch.Tensor:
    """t [..., d] as a matrix with neighbouring elements in its rows (a copy only
    where it is laid out otherwise)."""
    if t.dim() == 0:
        raise ValueError(f"{name} must have a last dimension")
    m = t.reshape(math.prod(t.shape[:-1]), t.shape[-1])
    plain = m.stride(1) == 1 or m.shape[1] == 1
    return m if plain and (m.shape[0] <= 1 or m.stride(0) >= m.shape[1]) else m.contiguous()


def _keep(ctx, *items):
    """Saves tensors and Held activations, each once, for _kept."""
    tensors, how = [], []
    for v in items:
        if isinstance(v, NR.Held):
            how.append((v.d, v.fmt, v.dtype))
            tensors += [v.q, v.scale]
        else:
            how.append(None)
            tensors.append(v)
    ctx.save_for_backward(*tensors)
    ctx.how = how


def _kept(ctx):
    tensors, out = list(ctx.saved_tensors), []
    for h in ctx.how:
        if h is None:
            out.append(tensors.pop(0))
        else:
            out.append(NR.Held(tensors.pop(0), tensors.pop(0), *h))
    return out


class _Linear(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, w, bias, residual, act, hold, grad):
        need_x, need_w, need_b = (need and grad for need in ctx.needs_input_grad[:3])
        x2 = _rows(x, "x")
        r2 = None if residual is None else _rows(residual, "residual")
        slope = act != "none" and (need_x or need_w or need_b)
        # a relu's own output has the pre-activation's sign
        own = slope and act == "relu" and residual is None and hold is None
        y = NR.nr_linear(x2, w, bias, act=act, residual=r2,
                         pre=(hold or True) if slope and not own else False)
        y, pre = y if slope and not own else (y, None)
        out = y.view(*x.shape[:-1], w.shape[0])
        keep_x = None
        if need_w:
            keep_x = NR.nr_act_hold(x2, hold) if hold else x2
        _keep(ctx, keep_x, w if need_x or need_w else None, out if own else pre)
        ctx.act, ctx.shape, ctx.own = act, x.shape, own
        return out

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        need_x, need_w, need_b, need_r = ctx.needs_input_grad[:4]
        dx = dw = db = None
        if need_x or need_w or need_b:
            x2, w, pre = _kept(ctx)
            if ctx.own:
                pre = _rows(pre, "y")
            d2 = _rows(dy, "dy")
            if x2 is None and w is None:   # only the bias's: the width does not matter
                x2 = d2
            dx, dw, db = NR.nr_linear_grad(d2, x2, w, act=ctx.act, pre=pre, dx=need_x, dw=need_w,
                                           db=need_b)
            dx = None if dx is None else dx.view(ctx.shape)
        return dx, dw, db, dy if need_r else None, None, None, None


class _LayerNorm(torch.autograd.Function):
    @staticmethod
    def forward(ctx, x, weight, bias, eps, hold, grad):
        x2 = _rows(x, "x")
        if grad and any(ctx.needs_input_grad[:3]):
            y, stats, *held = NR.nr_layer_norm(x2, weight, bias, eps, stats=True, hold_x=hold)
            _keep(ctx, held[0] if held else x2, stats, weight)
        else:
            y = NR.nr_layer_norm(x2, weight, bias, eps)
        ctx.shape = x.shape
        return y.view(x.shape)

    @staticmethod
    @once_differentiable
    def backward(ctx, dy):
        x2, stats, weight = _kept(ctx)
        need_x, need_w, need_b = ctx.needs_input_grad[:3]
        dx, dw, db = NR.nr_layer_norm_grad(_rows(dy, "dy"), x2, stats, weight, dx=need_x,
                                           dweight=need_w, dbias=need_b)
        return None if dx is None else dx.view(ctx.shape), dw, db, None, None, None


def linear(x: torch.Tensor, w: torch.Tensor, bias: Optional[torch.Tensor] = None,
           act: str = "none", residual: Optional[torch.Tensor] = None,
           hold: Optional[str] = None) -> torch.Tensor:
    """act(x w^T + bias) + residual, x [..., k], w [n, k], residual [..., n]; act one
    of "none", "relu", "gelu" (erf) and "silu"."""
    if residual is not None and residual.shape != (*x.shape[:-1], w.shape[0]):
        raise ValueError(f"residual must be {[*x.shape[:-1], w.shape[0]]}, "
                         f"got {list(residual.shape)}")
    if hold is not None and hold not in NR.HOLDS:
        raise ValueError(f"hold must be one of {sorted(NR.HOLDS)}, got {hold!r}")
    return _Linear.apply(x, w, bias, residual, act, hold, torch.is_grad_enabled())


def layer_norm(x: torch.Tensor, weight: Optional[torch.Tensor] = None,
               bias: Optional[torch.Tensor] = None, eps: float = 1e-5,
               hold: Optional[str] = None) -> torch.Tensor:
    """Layer norm over the last dimension of x."""
    if hold is not None and hold not in NR.HOLDS:
        raise ValueError(f"hold must be one of {sorted(NR.HOLDS)}, got {hold!r}")
    return _LayerNorm.apply(x, weight, bias, eps, hold, torch.is_grad_enabled())
