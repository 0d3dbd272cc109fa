"""Orthogonalised updates on the GPU: places and polynomials at the edges of what is accepted, and the precision that 22 bits give."""
import pytest
import torch

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
