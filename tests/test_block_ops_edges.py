"""What the operators between a model's input and its gradient rows accept and refuse at the edges of their arguments, without a GPU."""
import ctypes

import torch

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
