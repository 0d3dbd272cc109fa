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


def feed_need(f, *args):
    need = ctypes.c_int64(-1)
    assert f(*args, ctypes.byref(need)) == B.DEF_OK
    return need.value


def test_feed_forward_refuses():
    T, C, F, O = 300, 64, 96, 40
    need = feed_need(L.def_feed_forward_workspace, 1, T, C, F, O, at(1), C, at(2), at(3), at(4), F)
    assert 0 <= need <= (20 << 20) + 2 * (T * (C + 7) + 2 * F * (C + 7) + T * (F + 7) + O * (F + 7))
    ok = [1, T, C, F, O, at(1), C, at(2), at(3), at(4), F, at(5), O, at(6), at(7), at(8), at(9), at(10), need, None]
    f = caller(L.def_feed_forward, ok)
    if not HAS_GPU:
        assert f() == B.DEF_ERR_DEVICE
        assert f(_8=None, _11=None) == B.DEF_ERR_DEVICE                    # h only
        assert f(_13=None, _14=None, _15=None, _16=None) == B.DEF_ERR_DEVICE
    for i in (5, 7, 9, 8, 11, 14, 15):
        assert f(**{"_%d" % i: None}) == B.DEF_ERR_NULL
    assert f(_13=None, _14=None) == B.DEF_ERR_NULL                         # one checkpoint without the other
    assert f(_0=5) == B.DEF_ERR_ARG and f(_1=-1) == B.DEF_ERR_ARG and f(_2=0) == B.DEF_ERR_ARG and f(_3=0) == B.DEF_ERR_ARG and f(_4=0) == B.DEF_ERR_ARG
    assert f(_1=(1 << 30) + 1) == B.DEF_ERR_ARG and f(_6=C - 1) == B.DEF_ERR_ARG and f(_10=F - 1) == B.DEF_ERR_ARG and f(_12=O - 1) == B.DEF_ERR_ARG
    assert f(_9=at(1)) == B.DEF_ERR_ALIAS and f(_11=at(4)) == B.DEF_ERR_ALIAS and f(_9=at(2)) == B.DEF_ERR_ALIAS and f(_11=at(3, 2)) == B.DEF_ERR_ALIAS
    assert f(_5=at(1, 1), _18=1 << 25) == B.DEF_ERR_ALIGN and f(_13=at(6, 8)) == B.DEF_ERR_ALIGN
    assert f(_1=0, _5=None) == B.DEF_OK
    # rows off 16-byte boundaries and fp32 need copies
    for dt, ld in ((1, C + 1), (0, C)):
        n = feed_need(L.def_feed_forward_workspace, dt, T, C, F, O, at(1), ld, at(2), at(3), at(4), F)
        p = 3 if dt == 0 else 1
        assert 0 < n <= (20 << 20) + 2 * p * (T * (C + 7) + 2 * F * (C + 7) + T * (F + 7) + O * (F + 7))
        g = caller(L.def_feed_forward, [dt, T, C, F, O, at(1), ld, *ok[7:18], n, None])
        assert g(_17=None) == B.DEF_ERR_NULL and g(_18=n - 1) == B.DEF_ERR_ARG and g(_17=at(10, 8)) == B.DEF_ERR_ALIGN and g(_17=at(4)) == B.DEF_ERR_ALIAS


def test_feed_forward_backward_refuses():
    T, C, F, O = 300, 64, 96, 40
    need = feed_need(L.def_feed_forward_backward_workspace, 1, T, C, F, O, at(1), O, at(2), at(3), at(8), 2 * F)
    ok = [1, T, C, F, O, at(1), O, at(2), at(3), at(4), at(5), at(6), at(7), at(8), 2 * F, at(9), C, at(10), F, at(11), at(12), at(13), need, None]
    f = caller(L.def_feed_forward_backward, ok)
    if not HAS_GPU:
        assert f() == B.DEF_ERR_DEVICE
        assert f(_7=None, _15=None) == B.DEF_ERR_DEVICE                    # without dx
        assert f(_17=None, _19=None, _20=None) == B.DEF_ERR_DEVICE
    for i in (5, 7, 8, 9, 10, 11, 12, 13, 15, 19):
        assert f(**{"_%d" % i: None}) == B.DEF_ERR_NULL
    assert f(_6=O - 1) == B.DEF_ERR_ARG and f(_14=2 * F - 1) == B.DEF_ERR_ARG and f(_16=C - 1) == B.DEF_ERR_ARG and f(_18=F - 1) == B.DEF_ERR_ARG
    for i in (1, 2, 3, 4, 6, 9, 10, 11):
        assert f(_13=at(i)) == B.DEF_ERR_ALIAS
    assert f(_15=at(1)) == B.DEF_ERR_ALIAS and f(_19=at(4)) == B.DEF_ERR_ALIAS


def test_orthogonalize_refuses():
    need = ctypes.c_int64(-1)
    for m, n in ((1, 1), (33, 70), (70, 33), (4096, 1000), (65536, 3)):
        for batch in (1, 3):
            assert L.def_orthogonalize_workspace(batch, m, n, ctypes.byref(need)) == B.DEF_OK
            a, b = min(m, n), max(m, n)
            assert 0 < need.value <= batch * (16 * (a + 8) * (b + a + 16) + 8192)
    assert L.def_orthogonalize_workspace(1, 65537, 3, ctypes.byref(need)) == B.DEF_ERR_ARG
    assert L.def_orthogonalize_workspace(1, 0, 3, ctypes.byref(need)) == B.DEF_ERR_ARG
    assert L.def_orthogonalize_workspace(1, 3, 3, None) == B.DEF_ERR_NULL
    assert L.def_orthogonalize_workspace(3, 48, 64, ctypes.byref(need)) == B.DEF_OK
    n = need.value
    co = (ctypes.c_float * 6)(3.4445, -4.775, 2.0315, 1.5, -0.5, 0.0)
    f = caller(L.def_orthogonalize, [0, 3, 48, 64, at(0), 64, 5000, at(1), 64, 5000, co, 2, 1e-7, 1.0, at(2), n, None])
    if not HAS_GPU:
        assert f() == B.DEF_ERR_DEVICE
        assert f(_7=at(0)) == B.DEF_ERR_DEVICE                             # in place
        assert f(_7=at(0, 4 * 3000), _2=20, _3=50) == B.DEF_ERR_DEVICE     # another weight of the same gradient rows
    assert f(_7=at(0), _9=5001) == B.DEF_ERR_ALIAS and f(_7=at(0, 4)) == B.DEF_ERR_ALIAS
    assert f(_0=3) == B.DEF_ERR_ARG and f(_1=-1) == B.DEF_ERR_ARG and f(_2=0) == B.DEF_ERR_ARG and f(_3=1 << 17) == B.DEF_ERR_ARG
    assert f(_5=63) == B.DEF_ERR_ARG and f(_6=48 * 64 - 1) == B.DEF_ERR_ARG and f(_9=100) == B.DEF_ERR_ARG
    assert f(_11=0) == B.DEF_ERR_ARG and f(_11=33) == B.DEF_ERR_ARG and f(_10=None) == B.DEF_ERR_NULL
    assert f(_10=(ctypes.c_float * 6)(1, 2, 3, 4, 5, 9)) == B.DEF_ERR_ARG and f(_10=(ctypes.c_float * 6)(1, float("nan"), 3, 4, 5, 6)) == B.DEF_ERR_ARG
    assert f(_12=-1.0) == B.DEF_ERR_ARG and f(_12=float("nan")) == B.DEF_ERR_ARG and f(_13=float("inf")) == B.DEF_ERR_ARG
    assert f(_4=None) == B.DEF_ERR_NULL and f(_7=None) == B.DEF_ERR_NULL and f(_14=None) == B.DEF_ERR_NULL
    assert f(_15=n - 1) == B.DEF_ERR_ARG and f(_14=at(2, 8)) == B.DEF_ERR_ALIGN and f(_4=at(0, 2)) == B.DEF_ERR_ALIGN and f(_14=at(1)) == B.DEF_ERR_ALIAS
    assert f(_1=0, _4=None, _7=None, _14=None) == B.DEF_OK


def test_a_bound_for_the_polynomial_steps():
    """What max |f'| says about a perturbed matrix holds for one."""
    torch.manual_seed(0)
    x = torch.randn(12, 20, dtype=torch.float64)
    e = 1e-6 * torch.randn(12, 20, dtype=torch.float64)
    a, b, c = R.MUON[0]
    f = lambda X: (a * torch.eye(12, dtype=torch.float64) + b * X @ X.t() + c * X @ X.t() @ X @ X.t()) @ X  # noqa: E731
    x = x / x.norm()
    s = torch.linspace(0, 1, 1001, dtype=torch.float64) * float(torch.linalg.matrix_norm(x, 2))
    slope = float((a + 3 * b * s ** 2 + 5 * c * s ** 4).abs().max())
    assert float((f(x + e) - f(x)).norm()) <= slope * float(e.norm()) * 1.001
