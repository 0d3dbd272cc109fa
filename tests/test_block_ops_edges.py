"""What the operators between a model's input and its gradient rows accept and refuse at the edges of their arguments, without a GPU."""
import ctypes

import torch

import block_ref as R
from paper_2004_05298_b200 import binding as B
from test_block_ops_boundary import at, caller

HAS_GPU = torch.cuda.is_available()
L = B.lib


def accepted(rc):
    """Without a GPU the last of the checks says so; made-up pointers go nowhere else."""
    return rc == B.DEF_ERR_DEVICE


def test_orthogonalize_takes_columns_beside_each_other():
    """x and out in the same rows: apart, as column halves of one buffer are everywhere, or overlapping by one column."""
    need = ctypes.c_int64(-1)
    assert L.def_orthogonalize_workspace(3, 48, 64, ctypes.byref(need)) == B.DEF_OK
    co = (ctypes.c_float * 3)(3.4445, -4.775, 2.0315)
    ok = [0, 3, 48, 64, at(0), 128, 48 * 128, at(0, 256), 128, 48 * 128, co, 1, 1e-7, 1.0, at(2), need.value, None]
    f = caller(L.def_orthogonalize, ok)
    if not HAS_GPU:
        assert accepted(f())                                               # right of x
        assert accepted(f(_4=at(0, 256), _7=at(0)))                        # left of it
        assert accepted(f(_1=1)) and accepted(f(_1=1, _6=0, _9=7))         # one matrix: any stride
        assert accepted(f(_6=50 * 128, _9=50 * 128))                       # rows between the matrices
        assert accepted(f(_9=49 * 128))                                    # matrices in other rows, columns apart all the same
        assert accepted(f(_5=130, _8=130, _6=48 * 130, _9=48 * 130))       # columns between them
        assert accepted(f(_6=48 * 128 + 64, _9=48 * 128 + 64, _7=at(0, 4 * 3 * (48 * 128 + 64))))    # behind the last matrix
    assert f(_7=at(0, 252)) == B.DEF_ERR_ALIAS                             # one column is x's
    assert f(_7=at(0, 260)) == B.DEF_ERR_ALIAS                             # the last one is x's first of the next row
    assert f(_8=129, _9=48 * 129) == B.DEF_ERR_ALIAS                       # other rows
    assert f(_6=48 * 128 + 64, _9=48 * 128 + 64) == B.DEF_ERR_ALIAS        # matrices that start in other columns


# A schedule of different steps whose first starts above 8: it takes singular values from 0.05 on to near 1.
STEEP = [(9.0, -26.0, 19.0), (2.0, -0.6, 0.06)] + [(1.875, -1.25, 0.375)] * 5


def test_orthogonalize_takes_any_polynomials_that_stay_small():
    need = ctypes.c_int64(-1)
    assert L.def_orthogonalize_workspace(1, 48, 64, ctypes.byref(need)) == B.DEF_OK

    def rc(steps):
        flat = [v for s in steps for v in s]
        return L.def_orthogonalize(0, 1, 48, 64, at(0), 64, 0, at(1), 64, 0, (ctypes.c_float * len(flat))(*flat), len(steps), 1e-7, 1.0, at(2), need.value, None)

    if not HAS_GPU:
        assert accepted(rc(STEEP))
        assert accepted(rc([(1.5, -0.5, 0.0)] * 20)) and accepted(rc([(3.0, -8.0, 8.0)]))
        assert accepted(rc([(1.0, 0.0, 0.0), (0.0, 9.0, -8.5)]))
        assert accepted(rc([(0.1, 0.0, 0.0), (9.0, 64.0, 64.0)]))          # from [0, 0.1] on these stay small
        assert accepted(rc([(8.0, 8.0, 8.0)] * 5))                         # within 8: taken, whatever comes of it
    for steps in ([(16.0, 0.0, 0.0)], [(1.0, 2.0, 3.0), (4.0, 5.0, 9.0)], [(9.0, 0.0, 0.0)], [(0.0, 0.0, 16.5)], [(-9.0, 4.0, 0.0)],
                  [(3.0, -12.0, 40.0)], [(0.0, 64.5, -64.5)], [(8.5, float("nan"), 0.0)], [(float("inf"), 0.0, 0.0)], [(1.0, 0.0, 0.0), (9.0, 64.0, 64.0)]):
        assert rc(steps) == B.DEF_ERR_ARG and "coefficients" in B.def_last_error()


def test_what_polynomials_do_to_singular_values():
    """The limits by which a schedule is taken, on a fine grid: STEEP's factors stay below 16, its singular values below 4."""
    s = torch.linspace(0, 1, 200001, dtype=torch.float64)
    for a, b, c in STEEP:
        f = a + b * s ** 2 + c * s ** 4
        s = s * f
        assert float(f.abs().max()) < 16 and float(s.abs().max()) < 4
    assert float((s[10000:] - 1).abs().max()) < 0.01


def test_the_precision_bound_tells_lost_pieces():
    """R.NEAR is passed by two pieces and missed, by far, where the lower piece of something is lost."""
    torch.manual_seed(0)
    for m, n in ((64, 64), (300, 200), (100, 2000), (600, 700)):
        for direction in (0, 3):
            x = torch.randn(m, n) + direction * torch.randn(m, 1) * torch.randn(1, n)
            want = R.newton_schulz(x, lost=None)
            off = lambda **kw: float((R.newton_schulz(x, **kw) - want).norm() / want.norm())      # noqa: E731
            assert off() < R.NEAR / 20
            assert all(off(lost=(k,)) > 20 * R.NEAR for k in "XAB")
            if m > 512:
                assert all(off(mirrored=(k,)) > 5 * R.NEAR for k in "AB")
