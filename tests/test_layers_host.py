"""Argument checks of the layers' C entry points that need no GPU: bad
descriptions are refused before any HIP call, and the structs are laid out as
the binding has them."""
import ctypes as C
import os
import subprocess

import pytest
import torch

from paper_2608_15438_amd import neuroute as NR
from tests import layers_ref as R

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
STRUCTS = (NR.nr_linear_desc, NR.nr_linear_grad_desc, NR.nr_layer_norm_desc,
           NR.nr_layer_norm_grad_desc)


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(NR.SO_PATH):
        from paper_2608_15438_amd import build_lib
        build_lib.build()
    return NR.lib()


def test_struct_layouts(tmp_path):
    body = "".join(f'  printf("%zu", sizeof({s.__name__}));\n' + "".join(
        f'  printf(" %zu", offsetof({s.__name__}, {f}));\n' for f, _ in s._fields_)
        + '  printf("\\n");\n' for s in STRUCTS)
    src = tmp_path / "layout.c"
    src.write_text("#include <stddef.h>\n#include <stdio.h>\n#include \"neuroute.h\"\n"
                   "int main(void) {\n" + body + "  return 0;\n}\n")
    exe = tmp_path / "layout"
    subprocess.run(["gcc", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"),
                    "-I", "/opt/rocm/include", str(src), "-o", str(exe)], check=True)
    out = subprocess.run([str(exe)], capture_output=True, text=True, check=True).stdout
    for s, line in zip(STRUCTS, out.splitlines()):
        want = [C.sizeof(s)] + [getattr(s, f).offset for f, _ in s._fields_]
        assert [int(v) for v in line.split()] == want, s.__name__


A = 0x10000      # a well-aligned address that no refused call touches


def linear(**kw):
    d = NR.nr_linear_desc()
    d.m, d.n, d.k, d.dtype, d.act = 4, 5, 6, NR.NR_F32, 0
    d.x, d.ldx, d.w, d.ldw, d.y, d.ldy = A, 6, A, 6, A, 5
    for k, v in kw.items():
        setattr(d, k, v)
    return d


@pytest.mark.parametrize("kw,status", [
    (dict(dtype=0), NR.NR_EINVAL), (dict(dtype=4), NR.NR_EINVAL), (dict(act=4), NR.NR_EINVAL),
    (dict(act=-1), NR.NR_EINVAL), (dict(m=-1), NR.NR_EINVAL), (dict(n=0), NR.NR_EINVAL),
    (dict(k=0), NR.NR_EINVAL), (dict(n=16385), NR.NR_EUNSUPPORTED),
    (dict(k=16385), NR.NR_EUNSUPPORTED), (dict(x=None), NR.NR_EINVAL), (dict(w=None), NR.NR_EINVAL),
    (dict(y=None), NR.NR_EINVAL), (dict(ldx=5), NR.NR_EINVAL), (dict(ldw=5), NR.NR_EINVAL),
    (dict(ldy=4), NR.NR_EINVAL), (dict(ldx=-6), NR.NR_EINVAL), (dict(x=A + 2), NR.NR_EINVAL),
    (dict(bias=A + 1), NR.NR_EINVAL), (dict(residual=A, ldr=4), NR.NR_EINVAL),
    (dict(pre=A, ldp=4), NR.NR_EINVAL), (dict(pre=A, ldp=32, pre_hold=3), NR.NR_EINVAL),
    (dict(pre=A, ldp=32, pre_hold=1), NR.NR_EINVAL),                      # no scales
    (dict(pre=A, ldp=5, pre_hold=1, pre_scale=A), NR.NR_EINVAL),          # not whole groups
    (dict(pre=A + 4, ldp=32, pre_hold=1, pre_scale=A), NR.NR_EINVAL),
    (dict(dtype=NR.NR_BF16, w=A + 1), NR.NR_EINVAL),
    (dict(m=(1 << 40) + 1), NR.NR_EUNSUPPORTED),
])
def test_linear_refusals(L, kw, status):
    assert L.nr_linear(C.byref(linear(**kw)), None, 0, None) == status
    assert L.nr_last_error()


def test_work_space_is_checked(L):
    d = linear(m=8, n=16, k=4096, ldx=4096, ldw=4096, ldy=16)
    g = NR.nr_linear_grad_desc()
    g.m, g.n, g.k, g.dtype, g.act = 4096, 64, 64, NR.NR_BF16, 2
    g.dy = g.x = g.w = g.pre = g.dx = g.dw = g.db = A
    g.lddy = g.ldx = g.ldw = g.ldp = g.lddx = g.lddw = 64
    n = NR.nr_layer_norm_grad_desc()
    n.m, n.d, n.dtype = 100, 64, NR.NR_F16
    n.dy = n.x = n.stats = n.dx = n.dweight = n.dbias = A
    n.lddy = n.ldx = n.lddx = 64
    for desc, ws, call in ((d, L.nr_linear_ws, L.nr_linear),
                           (g, L.nr_linear_grad_ws, L.nr_linear_grad),
                           (n, L.nr_layer_norm_grad_ws, L.nr_layer_norm_grad)):
        need = ws(C.byref(desc))
        if call is not L.nr_linear:
            assert need > 0
        if need:
            for p, have in ((None, need), (A, need - 1), (A + 8, need)):
                assert call(C.byref(desc), p, have, None) == NR.NR_EINVAL
        assert ws(None) == 0
        assert call(None, None, 0, None) == NR.NR_EINVAL


def test_linear_grad_refusals(L):
    def desc(**kw):
        g = NR.nr_linear_grad_desc()
        g.m, g.n, g.k, g.dtype, g.act = 4, 5, 6, NR.NR_F32, 1
        g.dy, g.lddy, g.x, g.ldx, g.w, g.ldw, g.pre, g.ldp = A, 5, A, 6, A, 6, A, 5
        g.dx, g.lddx, g.dw, g.lddw, g.db = A, 6, A, 6, A
        for k, v in kw.items():
            setattr(g, k, v)
        return g
    for kw in (dict(dy=None), dict(x=None), dict(w=None), dict(pre=None), dict(lddy=4), dict(ldx=5),
               dict(ldw=5), dict(ldp=4), dict(lddx=5), dict(lddw=5), dict(db=A + 2), dict(act=9),
               dict(dtype=0), dict(m=-1), dict(n=0), dict(k=0), dict(x_hold=7),
               dict(x_hold=1, ldx=32), dict(pre_hold=2, ldp=5, pre_scale=A)):
        assert L.nr_linear_grad(C.byref(desc(**kw)), A, 1 << 40, None) == NR.NR_EINVAL, kw
    # nothing asked for: nothing to do
    assert L.nr_linear_grad(C.byref(desc(dx=None, dw=None, db=None)), None, 0, None) == NR.NR_OK


def test_norm_and_hold_refusals(L):
    def desc(**kw):
        n = NR.nr_layer_norm_desc()
        n.m, n.d, n.dtype, n.eps, n.x, n.ldx, n.y, n.ldy = 4, 40, NR.NR_F32, 1e-5, A, 40, A, 40
        for k, v in kw.items():
            setattr(n, k, v)
        return n
    for kw, st in ((dict(d=0), 1), (dict(d=16385), 4), (dict(m=-1), 1), (dict(dtype=0), 1),
                   (dict(eps=-1e-5), 1), (dict(eps=float("nan")), 1), (dict(eps=float("inf")), 1),
                   (dict(x=None), 1), (dict(y=None), 1), (dict(ldx=39), 1), (dict(ldy=39), 1),
                   (dict(weight=A + 2), 1), (dict(stats=A + 2), 1), (dict(x_hold=1), 1),
                   (dict(y_hold=3, yq=A, y_scale=A), 1), (dict(y_hold=1, yq=A + 8, y_scale=A), 1)):
        assert L.nr_layer_norm(C.byref(desc(**kw)), None) == st, kw
    assert L.nr_layer_norm(None, None) == NR.NR_EINVAL
    ok = dict(x=A, ldx=40, m=4, d=40, dtype=NR.NR_F32, hold=1, q=A, scale=A)
    for kw, st in ((dict(dtype=0), 1), (dict(hold=0), 1), (dict(hold=3), 1), (dict(d=0), 1),
                   (dict(d=20000), 4), (dict(m=-2), 1), (dict(ldx=39), 1), (dict(x=None), 1),
                   (dict(q=None), 1), (dict(scale=None), 1), (dict(q=A + 1), 1), (dict(x=A + 2), 1)):
        a = dict(ok, **kw)
        assert L.nr_act_hold(a["x"], a["ldx"], a["m"], a["d"], a["dtype"], a["hold"], a["q"],
                             a["scale"], None) == st, kw
        assert L.nr_act_read(a["q"], a["scale"], a["m"], a["d"], a["hold"], a["dtype"], a["x"],
                             a["ldx"], None) == st, kw


def test_tensors_must_be_on_a_device():
    x, w = torch.rand(3, 4), torch.rand(5, 4)
    for call in (lambda: NR.nr_linear(x, w), lambda: NR.nr_linear_grad(x, x, w),
                 lambda: NR.nr_layer_norm(x), lambda: NR.nr_layer_norm_grad(x, x, x),
                 lambda: NR.nr_act_hold(x)):
        with pytest.raises(ValueError):
            call()


def test_the_plain_hold():
    # the 64-bit form that the GPU tests compare with, on worked values
    x = torch.zeros((1, 40))
    x[0, :4] = torch.tensor([127.0, -63.5, 0.5, 1.5])
    v, byte = R.hold(x, "i8", torch.float32)
    assert int(byte[0, 0]) == 127 and v[0, :4].tolist() == [127.0, -64.0, 0.0, 2.0]
    assert int(byte[0, 1]) == 1 and not v[0, 32:].any()
    x[0, 0] = 127.5                                      # would round to 128: one step up
    v, byte = R.hold(x, "i8", torch.float32)
    assert int(byte[0, 0]) == 128 and v[0, :4].tolist() == [128.0, -64.0, 0.0, 2.0]
    x[0, :4] = torch.tensor([448.0, 17.0, 2.0 ** -10, 3 * 2.0 ** -10])
    v, byte = R.hold(x, "e4m3", torch.float32)
    assert int(byte[0, 0]) == 127 and v[0, :4].tolist() == [448.0, 16.0, 0.0, 2.0 ** -8]


def test_training_layers_need_a_device():
    import numpy as np

    from paper_2608_15438_amd import train as TR
    from paper_2608_15438_amd.index_build import Encoder
    enc = Encoder(weights=[np.eye(4, dtype=np.float32)], biases=[np.zeros(4, np.float32)],
                  input_scale=1.0)
    for kw in (dict(layers="hip"), dict(layers="other"), dict(dtype=torch.bfloat16),
               dict(hold="i8")):
        with pytest.raises(ValueError):
            TR._Mlp(enc, "cpu", **kw)
