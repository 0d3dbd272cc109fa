"""Refusals of include/def_train.h, without a GPU: every bad argument becomes its error code before anything is
launched.  Addresses are made up and never dereferenced."""
import ctypes

import pytest
import torch

from paper_2004_05298_b200 import binding as B

HAS_GPU = torch.cuda.is_available()
L = B.lib
BASE = 0x7000_0000_0000


def at(i, off=0):
    """The i-th of a row of made-up buffers, 256 MB apart."""
    return BASE + i * (1 << 28) + off


@pytest.mark.parametrize("C", [1, 15, 16, 17, 32, 33, 128, 129, 4096, 50001])
def test_layout(C):
    ldq, lde = B.def_checkpoint_layout(C)
    assert ldq % 16 == 0 and C <= ldq < C + 16
    groups = (C + 31) // 32
    assert lde % 4 == 0 and groups <= lde < groups + 4


def test_layout_refuses():
    one = ctypes.c_int64(0)
    assert L.def_checkpoint_layout(0, ctypes.byref(one), ctypes.byref(one)) == B.DEF_ERR_ARG
    assert L.def_checkpoint_layout(5, None, ctypes.byref(one)) == B.DEF_ERR_NULL


def test_pack_and_unpack_refuse():
    f = L.def_checkpoint_pack
    ok = [1, 10, 64, at(0), 64, at(1), at(2), None]

    def rc(**changes):
        a = list(ok)
        for i, v in changes.items():
            a[int(i[1:])] = v
        return f(*a)

    assert rc(_0=3) == B.DEF_ERR_ARG and "dtype" in B.def_last_error()
    assert rc(_1=-1) == B.DEF_ERR_ARG
    assert rc(_2=0) == B.DEF_ERR_ARG
    assert rc(_3=None) == B.DEF_ERR_NULL and rc(_5=None) == B.DEF_ERR_NULL and rc(_6=None) == B.DEF_ERR_NULL
    assert rc(_4=63) == B.DEF_ERR_ARG and "stride" in B.def_last_error()
    assert rc(_3=at(0, 1)) == B.DEF_ERR_ALIGN and rc(_5=at(1, 8)) == B.DEF_ERR_ALIGN and rc(_6=at(2, 2)) == B.DEF_ERR_ALIGN
    assert rc(_4=1 << 59) == B.DEF_ERR_ARG and rc(_2=(1 << 30) + 1, _4=1 << 31) == B.DEF_ERR_ARG
    assert rc(_5=at(0, 128)) == B.DEF_ERR_ALIAS and "overlap" in B.def_last_error()
    assert rc(_1=0, _3=None, _5=None, _6=None) == B.DEF_OK            # no rows: a no-op
    if not HAS_GPU:
        assert rc() == B.DEF_ERR_DEVICE
    u = L.def_checkpoint_unpack
    assert u(1, 10, 64, at(1), at(2), None, 64, None) == B.DEF_ERR_NULL
    assert u(1, 10, 64, at(1), at(2), at(1), 64, None) == B.DEF_ERR_ALIAS
    assert u(1, 10, 64, at(1), at(2), at(3), 10, None) == B.DEF_ERR_ARG


def test_weight_grad_refuses():
    f = L.def_checkpoint_weight_grad
    need = ctypes.c_int64(-1)
    assert L.def_checkpoint_weight_grad_workspace(1, 100, 64, 32, at(0), 64, ctypes.byref(need)) == B.DEF_OK
    n = need.value
    assert 0 <= n <= (68 << 20) + 8 * 64 * 32 + 6 * 100 * 71
    assert f(1, 100, 64, 32, None, 64, at(1), at(2), at(3), 0, at(4), n, None) == B.DEF_ERR_NULL
    assert f(1, 100, 64, 32, at(0), 64, at(1), at(2), None, 0, at(4), n, None) == B.DEF_ERR_NULL
    assert f(1, 100, 64, 32, at(0), 60, at(1), at(2), at(3), 0, at(4), n, None) == B.DEF_ERR_ARG
    assert f(1, 100, 64, 0, at(0), 64, at(1), at(2), at(3), 0, at(4), n, None) == B.DEF_ERR_ARG
    assert f(1, 100, 64, 32, at(0), 64, at(1), at(2), at(3, 2), 0, at(4), n, None) == B.DEF_ERR_ALIGN
    assert f(1, 100, 64, 32, at(0), 64, at(1), at(2), at(0, 400), 0, at(4), n, None) == B.DEF_ERR_ALIAS
    # fp32 rows need an aligned copy: the workspace is required, and its size checked
    assert L.def_checkpoint_weight_grad_workspace(0, 100, 64, 32, at(0), 64, ctypes.byref(need)) == B.DEF_OK
    if need.value > 0:
        assert f(0, 100, 64, 32, at(0), 64, at(1), at(2), at(3), 0, None, 0, None) == B.DEF_ERR_NULL
        assert f(0, 100, 64, 32, at(0), 64, at(1), at(2), at(3), 0, at(4), need.value - 1, None) == B.DEF_ERR_ARG
        assert f(0, 100, 64, 32, at(0), 64, at(1), at(2), at(3), 0, at(4, 8), need.value, None) == B.DEF_ERR_ALIGN


def test_gated_refuses():
    f, g = L.def_gated_forward, L.def_gated_backward
    fw = [1, 10, 64, at(0), 128, at(0, 128), 128, at(1), 64, at(2), at(3), at(4), at(5), None]
    if not HAS_GPU:
        assert f(*fw) == B.DEF_ERR_DEVICE                              # halves of one buffer are apart
    assert f(*fw[:7], None, *fw[8:]) == B.DEF_ERR_NULL
    assert f(*fw[:10], None, *fw[11:]) == B.DEF_ERR_NULL and "gate" in B.def_last_error()
    assert f(*fw[:7], at(0, 64), 128, *fw[9:]) == B.DEF_ERR_ALIAS       # h over columns of gate
    assert f(*fw[:4], 32, *fw[5:]) == B.DEF_ERR_ARG
    bw = [1, 10, 64, at(0), 64, at(2), at(3), at(4), at(5), at(6), 128, at(6, 128), 128, None, 0, None, None, None]
    if not HAS_GPU:
        assert g(*bw) == B.DEF_ERR_DEVICE
    assert g(*bw[:11], at(6, 126), *bw[12:]) == B.DEF_ERR_ALIAS
    assert g(*bw[:5], None, *bw[6:]) == B.DEF_ERR_NULL
    assert g(*bw[:15], at(7), None, None) == B.DEF_ERR_NULL


def test_norm_refuses():
    f = L.def_norm_forward
    a = [1, 12, 64, at(0), 64, at(1), 64, at(2), at(3), 3, at(4), 1.0, 1e-6, at(5), 64, at(6), 64, at(7), at(8)] + [None] * 7

    def rc(**changes):
        b = list(a)
        for i, v in changes.items():
            b[int(i[1:])] = v
        return f(*b)

    if not HAS_GPU:
        assert rc() == B.DEF_ERR_DEVICE
        assert rc(_13=at(0)) == B.DEF_ERR_DEVICE                       # h_out may be h
    assert rc(_13=at(0), _14=72) == B.DEF_ERR_ALIAS                    # but not with another stride
    assert rc(_15=at(0)) == B.DEF_ERR_ALIAS
    assert rc(_2=16385, _4=20000, _6=20000, _14=20000, _16=20000) == B.DEF_ERR_ARG
    assert rc(_9=5) == B.DEF_ERR_ARG and "groups" in B.def_last_error()
    assert rc(_9=0) == B.DEF_ERR_ARG
    assert rc(_12=-1.0) == B.DEF_ERR_ARG and rc(_12=float("nan")) == B.DEF_ERR_ARG
    assert rc(_5=None) == B.DEF_ERR_ARG                                # no block, but its parameters
    assert rc(_7=None) == B.DEF_ERR_NULL and rc(_10=None) == B.DEF_ERR_NULL and rc(_18=None) == B.DEF_ERR_NULL
    assert rc(_19=at(9)) == B.DEF_ERR_NULL
    assert rc(_4=40) == B.DEF_ERR_ARG

    g = L.def_norm_backward
    need = ctypes.c_int64(0)
    assert L.def_norm_backward_workspace(12, 64, 3, ctypes.byref(need)) == B.DEF_OK and need.value > 0
    assert need.value <= 8 * 64 * (12 + 3 + 8) + 4096
    assert L.def_norm_backward_workspace(12, 64, 5, ctypes.byref(ctypes.c_int64(0))) == B.DEF_ERR_ARG
    n = need.value
    a = [1, 12, 64, at(0), 64, at(1), 64, at(2), 64, None, None, at(3), 64, None, None, at(4), at(5), 3, at(6), 1.0, at(7), at(8), at(9), 64, at(10), 64,
         at(11), at(12), at(13), 0, at(14), n, None]

    def rb(**changes):
        b = list(a)
        for i, v in changes.items():
            b[int(i[1:])] = v
        return g(*b)

    if not HAS_GPU:
        assert rb() == B.DEF_ERR_DEVICE
        assert rb(_22=at(1)) == B.DEF_ERR_DEVICE                       # dh over dh_in
    assert rb(_22=at(2)) == B.DEF_ERR_ALIAS
    assert rb(_31=n - 1) == B.DEF_ERR_ARG and "workspace" in B.def_last_error()
    assert rb(_30=None) == B.DEF_ERR_NULL and rb(_30=at(14, 4)) == B.DEF_ERR_ALIGN
    assert rb(_27=None) == B.DEF_ERR_NULL and rb(_16=None) == B.DEF_ERR_NULL
    assert rb(_9=at(15), _10=at(16)) == B.DEF_ERR_ARG                   # h twice
    assert rb(_7=None) == B.DEF_ERR_NULL
    assert rb(_11=None) == B.DEF_ERR_ARG                                # no block, but its parameters
    assert rb(_9=at(15)) == B.DEF_ERR_NULL


def test_logprob_refuses():
    f = L.def_logprob_forward
    a = [1, 10, 64, at(0), 64, at(1), at(2), at(3), at(4), 5, at(5), at(6), None]

    def rc(**changes):
        b = list(a)
        for i, v in changes.items():
            b[int(i[1:])] = v
        return f(*b)

    if not HAS_GPU:
        assert rc() == B.DEF_ERR_DEVICE
    assert rc(_9=33) == B.DEF_ERR_ARG and rc(_9=-1) == B.DEF_ERR_ARG
    assert rc(_2=4) == B.DEF_ERR_ARG                                    # more alternatives than logits
    assert rc(_9=0) == B.DEF_ERR_NULL and rc(_10=None) == B.DEF_ERR_NULL and rc(_11=None) == B.DEF_ERR_NULL
    assert rc(_5=at(1, 4)) == B.DEF_ERR_ALIGN
    assert rc(_6=at(0)) == B.DEF_ERR_ALIAS
    assert rc(_3=None) == B.DEF_ERR_NULL
    g = L.def_logprob_backward
    b = [1, 10, 64, at(0), 64, at(1), at(2), at(3), at(4), at(5), 5, at(6), at(7), at(8), 64, None]
    if not HAS_GPU:
        assert g(*b) == B.DEF_ERR_DEVICE
        assert g(*b[:13], at(0), 64, None) == B.DEF_ERR_DEVICE          # in place
    assert g(*b[:13], at(0), 65, None) == B.DEF_ERR_ALIAS
    assert g(*b[:13], at(2), 64, None) == B.DEF_ERR_ALIAS
    assert g(*b[:10], 0, *b[11:]) == B.DEF_ERR_NULL
    assert g(*b[:12], None, *b[13:]) == B.DEF_ERR_NULL


def test_binding_refuses():
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        B.def_checkpoint_pack(x, (x, x))                               # not on the GPU
    with pytest.raises(TypeError):
        B.def_checkpoint_pack(torch.zeros(4, 8, dtype=torch.float64), None)
    with pytest.raises(TypeError):
        B.def_logprob_forward(torch.zeros(8), None, None, None, None)
