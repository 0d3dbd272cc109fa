"""Orthogonalised updates on the GPU: places and polynomials at the edges of what is accepted, and the precision that 22 bits give."""
import pytest
import torch

import block_ref as R
from test_orthogonalize_gpu import _near, _normal, _work

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("this test needs a CUDA device")
    from paper_2004_05298_b200 import binding
    return binding


@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("rows,cols", [(40, 64), (300, 93), (70, 33)])
def test_columns_beside_each_other(B, rows, cols, dtype):
    """x and out in the same rows of one buffer, a matrix or a batch; the columns around out stay as they are."""
    for shape in ((rows, 2 * cols + 6), (3, rows, 2 * cols + 6)):
        big = _normal(shape, dtype, 1)
        old = big.clone()
        x, out = big[..., 1:cols + 1], big[..., cols + 3:2 * cols + 3]
        B.def_orthogonalize(x, out, workspace=_work(B, rows, cols, 3))
        for got, was in ((out[None], x[None]) if out.dim() == 2 else (out, x),):
            for i in range(got.shape[0]):
                _near(got[i], was[i])
        assert torch.equal(big[..., :cols + 3], old[..., :cols + 3]) and torch.equal(big[..., 2 * cols + 3:], old[..., 2 * cols + 3:])


def test_steps_that_start_steep(B):
    """A schedule whose first coefficients are beyond 8."""
    from test_block_ops_edges import STEEP
    for rows, cols in ((48, 80), (300, 200), (1300, 700)):
        x, out = _normal((rows, cols), F32, 1), torch.empty(rows, cols, device=DEV)
        B.def_orthogonalize(x, out, coeffs=STEEP, workspace=_work(B, rows, cols))
        _near(out, x, coeffs=STEEP)


def _precise(got, x):
    want = R.newton_schulz(x, lost=None)
    rel = float((got.double() - want).norm() / want.norm())
    assert rel < R.NEAR, rel


@pytest.mark.parametrize("rows,cols", [(64, 64), (300, 200), (257, 513), (640, 256), (777, 1000), (64, 5000), (5000, 33), (1300, 1300), (100, 8000), (1100, 600), (2500, 2900)])
def test_precision(B, rows, cols):
    """One tile and several, tall and wide, whole and cut along k, chains of 1, 2 and 4 stages."""
    for direction in (0, 3):
        x = _normal((rows, cols), F32, 1) + direction * _normal((rows, 1), F32, 2) * _normal((1, cols), F32, 3)
        out = torch.empty_like(x)
        B.def_orthogonalize(x, out, workspace=_work(B, rows, cols))
        _precise(out, x)


@pytest.mark.parametrize("rows,cols", [(256, 640), (700, 600), (600, 700), (33, 47)])
def test_precision_of_batches_in_place(B, rows, cols):
    W, d, at = 4, rows * cols + 5003, 1237
    grads = _normal((W, d), F32, 1, 1e-3)
    old = grads.clone()
    view = grads[:, at:at + rows * cols].view(W, rows, cols)
    B.def_orthogonalize(view, view, workspace=_work(B, rows, cols, W))
    for w in range(W):
        _precise(view[w], old[w, at:at + rows * cols].view(rows, cols))
