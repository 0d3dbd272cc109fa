"""Operators between a model's input and its gradient rows, where offsets pass 32 bits: the last rows of a large call against
a call of those rows alone."""
import pytest
import torch

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("this test needs a CUDA device")
    from paper_2004_05298_b200 import binding
    yield binding
    torch.cuda.empty_cache()


def _random(gen, *shape):
    return torch.empty(*shape, dtype=torch.bfloat16, device="cuda").normal_(generator=gen)


@pytest.mark.parametrize("C", [32768, 32767])                             # blocks by tensor copies; element by element
def test_recurrence(B, C):
    T, last = 65600, 1000                                                  # T * C > 2^31
    gen = torch.Generator(device="cuda").manual_seed(3)
    x, gate, dy = (_random(gen, T, C) for _ in range(3))
    y, dx, dg = (torch.empty_like(x) for _ in range(3))
    offsets = torch.tensor([0, 30000, T - last, T], device="cuda")
    work = torch.empty(max(1, B.def_recurrence_workspace(T, C, x.dtype)), dtype=torch.uint8, device="cuda")
    B.def_recurrence_forward(x, gate, y, offsets=offsets, workspace=work)
    B.def_recurrence_backward(dy, x, gate, y, dx, dg, offsets=offsets, workspace=work)
    end = [t[T - last:] for t in (x, gate, dy)]
    y1, dx1, dg1 = (torch.empty_like(end[0]) for _ in range(3))
    B.def_recurrence_forward(end[0], end[1], y1, workspace=work)
    B.def_recurrence_backward(end[2], end[0], end[1], y[T - last:], dx1, dg1, workspace=work)
    # Blocks are joined elsewhere, which moves fp32 states of size 10 at most by some 2^-24 of that each: one step of bf16, 2^-7 of the value.
    for whole, alone in ((y, y1), (dx, dx1), (dg, dg1)):
        torch.testing.assert_close(whole[T - last:].float(), alone.float(), rtol=2.0 ** -7, atol=2e-5)


def test_feed_forward(B):
    T, C, F, last = 105000, 64, 20480, 300                                 # T * F > 2^31
    gen = torch.Generator(device="cuda").manual_seed(4)
    x, dout = _random(gen, T, C), _random(gen, T, C)
    w_in, w_down = _random(gen, 2 * F, C) / 8, _random(gen, C, F) / 8
    results = []
    for rows in (slice(0, T), slice(T - last, T)):
        xs, ds = x[rows], dout[rows]
        n = xs.shape[0]
        h = torch.empty(n, F, dtype=x.dtype, device="cuda")
        dboth = torch.empty(n, 2 * F, dtype=x.dtype, device="cuda")
        cks = [B.def_checkpoint_alloc(n, F, "cuda") for _ in range(3)]
        size = max(B.def_feed_forward_workspace(xs, w_in, None, h), B.def_feed_forward_backward_workspace(ds, None, w_down, dboth))
        work = torch.empty(max(1, size), dtype=torch.uint8, device="cuda")
        B.def_feed_forward(xs, w_in, None, h, None, cks[0], cks[1], workspace=work)
        B.def_feed_forward_backward(ds, None, w_down, cks[0], cks[1], dboth, None, h_ck=cks[2], workspace=work)
        results.append([h, dboth] + [t for ck in cks for t in ck])
    for whole, alone in zip(*results):                                     # one stage of 64 terms: the same sums wherever the tile lies
        assert torch.equal(whole[T - last:], alone)


def test_orthogonalize(B):
    W, d, rows, cols = 3, (1 << 30) + 100 * 64, 100, 64                    # the last matrix starts behind 2^31
    gen = torch.Generator(device="cuda").manual_seed(5)
    grads = torch.empty(W, d, device="cuda")
    view = grads[:, d - rows * cols:].unflatten(1, (rows, cols))
    view.normal_(generator=gen)
    work = torch.empty(B.def_orthogonalize_workspace(rows, cols, W), dtype=torch.uint8, device="cuda")
    alone = [torch.empty(rows, cols, device="cuda") for _ in range(W)]
    for w in range(W):
        B.def_orthogonalize(view[w], alone[w], workspace=work)
    B.def_orthogonalize(view, view, workspace=work)
    assert all(torch.equal(view[w], alone[w]) for w in range(W))           # few stages, never cut: the same sums
