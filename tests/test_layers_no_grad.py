"""What the differentiable layers ask of the kernels where no gradient is wanted:
the output, and nothing that only a backward pass reads.  The kernels' calls are
stood in for by plain forms, so no GPU is needed."""
import pytest
import torch

from paper_2608_15438_amd import layers as LY
from paper_2608_15438_amd import neuroute as NR


@pytest.fixture
def calls(monkeypatch):
    seen = []

    def linear(x, w, bias=None, act="none", residual=None, pre=False, stream=None):
        seen.append(("linear", pre))
        z = x @ w.T + (0 if bias is None else bias)
        y = z.clamp_min(0) if act == "relu" else z
        y = y if residual is None else y + residual
        return y if pre is False else (y, z)

    def norm(x, weight=None, bias=None, eps=1e-5, stats=False, hold_x=None, hold_y=None,
             stream=None):
        seen.append(("norm", stats, hold_x))
        y = torch.nn.functional.layer_norm(x, x.shape[-1:], weight, bias, eps)
        out = [y] + ([torch.zeros(2, x.shape[0])] if stats else []) + ([x] if hold_x else [])
        return y if len(out) == 1 else tuple(out)

    def hold(x, fmt="i8", stream=None):
        seen.append(("hold", fmt))
        return x

    monkeypatch.setattr(NR, "nr_linear", linear)
    monkeypatch.setattr(NR, "nr_layer_norm", norm)
    monkeypatch.setattr(NR, "nr_act_hold", hold)
    return seen


def inputs():
    g = torch.Generator().manual_seed(0)
    r = lambda *s: torch.randn(s, generator=g).requires_grad_(True)
    return r(5, 6), r(4, 6), r(4), r(5, 4), r(6), r(6)


@pytest.mark.parametrize("mode", [torch.no_grad, torch.inference_mode])
@pytest.mark.parametrize("hold", [None, "i8", "e4m3"])
def test_no_gradients_wanted(calls, mode, hold):
    x, w, b, r, g, gb = inputs()
    with mode():
        for act in ("none", "relu", "gelu", "silu"):
            y = LY.linear(x, w, b, act, r, hold=hold)
            assert not y.requires_grad
        LY.layer_norm(x, g, gb, hold=hold)
    assert calls == [("linear", False)] * 4 + [("norm", False, None)]


def test_gradients_wanted(calls):
    x, w, b, r, g, gb = inputs()
    LY.linear(x, w, b, "gelu", r)
    LY.linear(x, w, b, "gelu", r, hold="i8")
    LY.linear(x, w, b, "relu")
    LY.layer_norm(x, g, gb, hold="i8")
    assert calls == [("linear", True), ("linear", "i8"), ("hold", "i8"), ("linear", False),
                     ("norm", True, "i8")]
    # gradients turned on again inside
    del calls[:]
    with torch.no_grad(), torch.enable_grad():
        LY.linear(x, w, b, "gelu")
    assert calls == [("linear", True)]
    # and of inputs that want none
    del calls[:]
    LY.linear(*(v.detach() for v in (x, w, b)), act="gelu", hold="i8")
    LY.layer_norm(x.detach(), hold="i8")
    assert calls == [("linear", False), ("norm", False, None)]
