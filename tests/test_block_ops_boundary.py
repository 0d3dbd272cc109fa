"""Refusals of the recurrence, the feed-forward block and the orthogonalised update, without a GPU, and their 64-bit
statements against differences."""
import ctypes

import pytest
import torch

import block_ref as R
from paper_2004_05298_b200 import binding as B

HAS_GPU = torch.cuda.is_available()
L = B.lib
BASE = 0x7000_0000_0000


def at(i, off=0):
    """The i-th of a row of made-up buffers, 256 MB apart."""
    return BASE + i * (1 << 28) + off


def caller(f, ok):
    def rc(**changes):
        a = list(ok)
        for i, v in changes.items():
            a[int(i[1:])] = v
        return f(*a)
    return rc


def test_recurrence_refuses():
    need = ctypes.c_int64(-1)
    assert L.def_recurrence_workspace(1, 100, 64, ctypes.byref(need)) == B.DEF_OK and need.value == 0     # one block of steps
    assert L.def_recurrence_workspace(1, 100, 64, None) == B.DEF_ERR_NULL
    assert L.def_recurrence_workspace(1, (1 << 30) + 1, 64, ctypes.byref(need)) == B.DEF_ERR_ARG
    for dt in (0, 1, 2):
        for T in (0, 1, 128, 129, 5000, 1 << 20, 1 << 30):
            for C in (1, 2, 64, 511, 4096, 100000):
                assert L.def_recurrence_workspace(dt, T, C, ctypes.byref(need)) == B.DEF_OK and 0 <= need.value <= 4096 * C
    f = caller(L.def_recurrence_forward, [1, 12, 64, 3, at(0), at(1), 64, at(2), 64, at(3), at(4), 64, at(5), None, 0, None])
    if not HAS_GPU:
        assert f() == B.DEF_ERR_DEVICE
        assert f(_10=at(1)) == B.DEF_ERR_DEVICE                            # y may be x
    assert f(_10=at(1), _11=66) == B.DEF_ERR_ALIAS                         # but not with another stride
    assert f(_10=at(2)) == B.DEF_ERR_ALIAS and f(_12=at(3)) == B.DEF_ERR_ALIAS and f(_12=at(0)) == B.DEF_ERR_ALIAS
    assert f(_0=3) == B.DEF_ERR_ARG and f(_1=-1) == B.DEF_ERR_ARG and f(_2=0) == B.DEF_ERR_ARG
    assert f(_3=0) == B.DEF_ERR_ARG and f(_3=5, _4=None) == B.DEF_ERR_ARG and "sequences" in B.def_last_error()
    assert f(_5=None) == B.DEF_ERR_NULL and f(_7=None) == B.DEF_ERR_NULL and f(_10=None) == B.DEF_ERR_NULL
    assert f(_6=63) == B.DEF_ERR_ARG and f(_8=1 << 59) == B.DEF_ERR_ARG
    assert f(_4=at(0, 4)) == B.DEF_ERR_ALIGN and f(_5=at(1, 1)) == B.DEF_ERR_ALIGN and f(_9=at(3, 2)) == B.DEF_ERR_ALIGN
    assert f(_1=0, _5=None, _7=None, _10=None, _12=None) == B.DEF_OK       # nothing to do
    assert L.def_recurrence_workspace(0, 100000, 8, ctypes.byref(need)) == B.DEF_OK and need.value > 0
    n = need.value
    f = caller(L.def_recurrence_forward, [0, 100000, 8, 1, None, at(1), 8, at(2), 8, None, at(4), 8, None, at(6), n, None])
    assert f(_13=None) == B.DEF_ERR_NULL and f(_14=n - 1) == B.DEF_ERR_ARG and f(_13=at(6, 8)) == B.DEF_ERR_ALIGN and f(_13=at(4)) == B.DEF_ERR_ALIAS
    g = caller(L.def_recurrence_backward, [1, 12, 64, 3, at(0), at(1), 64, at(2), at(3), 64, at(4), 64, at(5), 64, at(6), at(7), 64, at(8), 64, at(9), None, 0, None])
    if not HAS_GPU:
        assert g() == B.DEF_ERR_DEVICE
        assert g(_15=at(7), _16=128, _17=at(7, 128), _18=128) == B.DEF_ERR_DEVICE      # halves of one buffer
    for i in (5, 8, 10, 12, 15, 17):
        assert g(**{"_%d" % i: None}) == B.DEF_ERR_NULL
    for i in (1, 3, 4, 5):
        assert g(_15=at(i)) == B.DEF_ERR_ALIAS and g(_17=at(i)) == B.DEF_ERR_ALIAS
    assert g(_17=at(7)) == B.DEF_ERR_ALIAS and g(_19=at(2)) == B.DEF_ERR_ALIAS and g(_19=at(9, 1)) == B.DEF_ERR_ALIGN


def test_binding_refuses():
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        B.def_recurrence_forward(x, x, x)                                  # not on the GPU


def test_recurrence_gradient_against_differences():
    """The backward formulas against central differences of the forward one, both in 64 bits."""
    torch.manual_seed(0)
    T, C, S, offsets = 11, 3, 3, [0, 4, 4, 10]
    spans = R.spans(T, S, offsets)
    x, g, h0 = torch.randn(T, C, dtype=torch.float64), torch.randn(T, C, dtype=torch.float64), torch.randn(S, C, dtype=torch.float64)
    dy, dl = torch.randn(T, C, dtype=torch.float64), torch.randn(S, C, dtype=torch.float64)
    dy[10:] = 0

    def loss():
        y, _, last, _ = R.recurrence(x, g, spans, h0)
        return float((y * dy).sum() + (last * dl).sum())

    y = R.recurrence(x, g, spans, h0)[0]
    grads, _ = R.recurrence_backward(dy, x, g, y, spans, h0, dl)
    for v, grad in zip((x, g, h0), grads):
        for i in range(v.numel()):
            old, step = float(v.view(-1)[i]), 1e-5
            v.view(-1)[i] = old + step
            up = loss()
            v.view(-1)[i] = old - step
            down = loss()
            v.view(-1)[i] = old
            assert abs((up - down) / (2 * step) - float(grad.reshape(-1)[i])) < 1e-8
