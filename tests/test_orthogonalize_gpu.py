"""Orthogonalised updates on the GPU against their statement in 64 bits (tests/block_ref.py has the error bounds)."""
import math

import pytest
import torch

import block_ref as R
from train_ref import UNIT

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("this test needs a CUDA device")
    from paper_2004_05298_b200 import binding
    return binding


def _normal(shape, dtype, seed, std=1.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, device=DEV).normal_(0.0, std, generator=g).to(dtype)


def _work(B, rows, cols, batch=1):
    return torch.empty(B.def_orthogonalize_workspace(rows, cols, batch), dtype=torch.uint8, device=DEV)


def _near(got, x, **kw):
    want, err = R.orthogonalize(x, **kw)
    # stored values are rounded: at most half a step each (fp16 also has a smallest step)
    off = UNIT[x.dtype] * float(want.norm()) + (2.0 ** -25 * math.sqrt(want.numel()) if x.dtype == F16 else 0)
    diff = float((got.double() - want).norm())
    assert diff <= err + off, (diff, err, off)


SIZES = [(1, 1), (1, 7), (9, 1), (5, 3), (32, 32), (33, 70), (70, 33), (64, 64), (128, 256), (129, 257), (300, 200), (257, 513)]


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
def test_sizes(B, dtype):
    for i, (m, n) in enumerate(SIZES):
        x = _normal((m, n), dtype, i, 0.01)
        out = torch.full_like(x, 5.0)
        B.def_orthogonalize(x, out, scale=0.5, workspace=_work(B, m, n))
        _near(out, x, scale=0.5)


@pytest.mark.parametrize("shape", [(640, 256), (256, 640), (777, 1000), (64, 5000), (5000, 33), (1300, 1300)])
def test_larger(B, shape):
    for dtype in (F32, BF16):
        x = _normal(shape, dtype, 1) + _normal((shape[0], 1), dtype, 2, 3.0) * _normal((1, shape[1]), dtype, 3)     # one direction dominates
        out = torch.empty_like(x)
        B.def_orthogonalize(x, out, workspace=_work(B, *shape))
        _near(out, x)


@pytest.mark.parametrize("rows,cols", [(96, 160), (160, 96), (33, 47)])
def test_gradient_rows_in_place(B, rows, cols):
    """A weight's slice of each of W gradient rows, at an odd place in the row, in place; nothing beside it changes."""
    W, d, at = 5, 40001, 1237
    grads = _normal((W, d), F32, 1, 1e-3)
    old = grads.clone()
    view = grads[:, at:at + rows * cols].view(W, rows, cols)
    work = _work(B, rows, cols, W)
    B.def_orthogonalize(view, view, workspace=work)
    for w in range(W):
        _near(view[w], old[w, at:at + rows * cols].view(rows, cols))
    assert torch.equal(grads[:, :at], old[:, :at]) and torch.equal(grads[:, at + rows * cols:], old[:, at + rows * cols:])


def test_strided_rows_and_matrices(B):
    """Columns of a larger matrix to columns of another, batches at any stride, 16-bit types off alignment."""
    for dtype in (F32, BF16):
        big, out = _normal((4, 70, 141), dtype, 1), torch.full((4, 71, 150), 5.0, dtype=dtype, device=DEV)
        x, o = big[:, 3:60, 5:98], out[:, 7:64, 9:102]
        B.def_orthogonalize(x, o, workspace=_work(B, 57, 93, 4))
        for i in range(4):
            _near(o[i], x[i])
        mask = torch.ones_like(out, dtype=torch.bool)
        mask[:, 7:64, 9:102] = False
        assert bool((out[mask] == 5).all()), "written outside the result"


def test_other_polynomials(B):
    """The cubic that converges to the orthogonal factor; a schedule of different steps; signs and scales."""
    x = _normal((48, 80), F32, 1)
    out = torch.empty_like(x)
    work = _work(B, 48, 80)
    cubic = [(1.5, -0.5, 0.0)] * 20
    B.def_orthogonalize(x, out, coeffs=cubic, workspace=work)
    _near(out, x, coeffs=cubic)
    u, _, vt = torch.linalg.svd(x.double(), full_matrices=False)
    assert float((out.double() - u @ vt).abs().max()) < 1e-4               # 20 steps from 0.05 on are within 1e-6 of 1
    mixed = [(4.0, -7.0, 3.5), (3.4445, -4.775, 2.0315), (1.875, -1.25, 0.375), (-1.0, 0.0, 0.0)]
    B.def_orthogonalize(x, out, coeffs=mixed, scale=-2.5, workspace=work)
    _near(out, x, coeffs=mixed, scale=-2.5)


def test_values_of_every_size(B):
    """Norms near the ends of fp32's range, zeros, a matrix of one direction, and NaN or infinity in one matrix of a batch."""
    x = _normal((7, 40, 56), F32, 1)
    x[0] *= 1e30
    x[1] *= 1e-36
    x[2] = 0
    x[3] = torch.outer(x[3, :, 0], x[3, 0])
    x[4, 3, 5], x[5, 39, 55] = math.nan, -math.inf
    out = torch.empty_like(x)
    B.def_orthogonalize(x, out, eps=0.0, workspace=_work(B, 40, 56, 7))
    for i in (0, 1, 3, 6):
        _near(out[i], x[i], eps=0.0)
    assert bool((out[2] == 0).all()) and bool(torch.isnan(out[4]).all()) and bool(torch.isnan(out[5]).all())


def test_streams_graphs_and_bits(B):
    m, n = 200, 330
    x = _normal((3, m, n), F32, 1)
    out, work = torch.empty_like(x), _work(B, m, n, 3)
    B.def_orthogonalize(x, out, workspace=work)
    again = torch.empty_like(x)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    B.def_orthogonalize(x, again, workspace=_work(B, m, n, 3), stream=side)
    side.synchronize()
    torch.cuda.synchronize()
    assert torch.equal(out, again)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.def_orthogonalize(x, out, workspace=work, stream=torch.cuda.current_stream())
    x.copy_(_normal((3, m, n), F32, 2))
    graph.replay()
    torch.cuda.synchronize()
    for i in range(3):
        _near(out[i], x[i])


def test_a_large_matrix_with_uncut_and_cut_tiles(B):
    x = _normal((2500, 2900), F32, 1)
    out = torch.empty_like(x)
    B.def_orthogonalize(x, out, workspace=_work(B, 2500, 2900))
    _near(out, x)
