"""Work space of the layers' products: a 16-bit operand that starts off a 16-byte
boundary is given room for its copy as one whose rows lie off them is, and the
other operands are not."""
import ctypes as C
import os

import pytest

from paper_2608_15438_amd import neuroute as NR

A = 0x10000      # a well-aligned address; nothing is launched


@pytest.fixture(scope="module")
def L():
    if not os.path.exists(NR.SO_PATH):
        from paper_2608_15438_amd import build_lib
        build_lib.build()
    return NR.lib()


M, K, N = 16_384, 1024, 1024


def forward(L, dtype, **kw):
    d = NR.nr_linear_desc()
    d.m, d.n, d.k, d.dtype = M, N, K, dtype
    d.x, d.ldx, d.w, d.ldw, d.y, d.ldy = A, K, A, K, A, N
    for k, v in kw.items():
        setattr(d, k, v)
    return L.nr_linear_ws(C.byref(d))


def backward(L, dtype, **kw):
    d = NR.nr_linear_grad_desc()
    d.m, d.n, d.k, d.dtype = M, N, K, dtype
    d.dy, d.lddy, d.x, d.ldx, d.w, d.ldw = A, N, A, K, A, K
    d.dx, d.lddx, d.dw, d.lddw = A, K, A, K
    for k, v in kw.items():
        setattr(d, k, v)
    return L.nr_linear_grad_ws(C.byref(d))


@pytest.mark.parametrize("dtype", [NR.NR_BF16, NR.NR_F16])
def test_forward(L, dtype):
    plain = forward(L, dtype)
    for at in (A + 2, A + 8):
        assert forward(L, dtype, x=at) == plain + 2 * M * K
        assert forward(L, dtype, w=at) == plain + 2 * N * K
        assert forward(L, dtype, x=at, w=at) == plain + 2 * (M + N) * K
    assert forward(L, dtype, ldx=K + 1) == plain + 2 * M * K
    assert forward(L, dtype, ldx=K + 8, ldw=K + 16) == plain
    # what the product does not read into LDS may start anywhere
    assert forward(L, dtype, y=A + 2, bias=A + 2) == plain


@pytest.mark.parametrize("dtype", [NR.NR_BF16, NR.NR_F16])
def test_backward(L, dtype):
    plain = backward(L, dtype)
    for at in (A + 2, A + 8):
        assert backward(L, dtype, dy=at) == plain + 2 * M * N
        assert backward(L, dtype, x=at) == plain + 2 * M * K
        assert backward(L, dtype, w=at) == plain + 2 * N * K
        assert backward(L, dtype, dy=at, x=at, w=at) == plain + 2 * (M * N + M * K + N * K)
    assert backward(L, dtype, dx=A + 2, dw=A + 2) == plain
    # dz is written anyway: dy and pre may start anywhere
    act = dict(act=2, pre=A, ldp=N)
    assert backward(L, dtype, dy=A + 2, **dict(act, pre=A + 2)) == backward(L, dtype, **act)


def test_floats_need_no_copy(L):
    assert forward(L, NR.NR_F32, x=A + 4, w=A + 4) == forward(L, NR.NR_F32)
    assert backward(L, NR.NR_F32, dy=A + 4, x=A + 4, w=A + 4) == backward(L, NR.NR_F32)
