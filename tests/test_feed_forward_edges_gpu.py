"""The gated feed-forward block on the GPU where its variants meet: few tokens and one output, and sums of many terms of one sign."""
import pytest
import torch

from test_feed_forward_gpu import _check

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
DEV = "cuda"


@pytest.fixture(scope="module")
def B():
    if not torch.cuda.is_available():
        pytest.fail("this test needs a CUDA device")
    from paper_2004_05298_b200 import binding
    yield binding
    torch.cuda.empty_cache()


@pytest.mark.parametrize("dtype", [F32, BF16, F16])
@pytest.mark.parametrize("layout", ["rows", "padded", "off"])
def test_few_tokens_and_one_output(B, dtype, layout):
    """w_down has one row, whose length need not be a multiple of 16 bytes for it to be read in place."""
    for T in (1, 2, 32, 33):
        for C, F in ((64, 65), (64, 1), (72, 200), (65, 66), (8, 4097)):
            _check(B, T, C, F, 1, dtype, T, layout, train=False)
            _check(B, T, C, F, 1, dtype, T, layout)


# Sums of one sign in 16-bit types.  The matrix unit truncates: 2 u (u = 2^-24), a unit in the last place, for every 16 terms (measured:
# 1.7 u).  Its sums hold at most 4096 (fp16) or 32768 (bf16) terms, and are added in fp32: a rounding each.
CHAIN = {F16: 4096, BF16: 32768}
U32 = 2.0 ** -24


def _bound(dtype, n):
    return (2 * CHAIN[dtype] / 16 + -(-n // CHAIN[dtype])) * U32


def _uniform(shape, dtype, seed, lo, hi):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, dtype=dtype, device=DEV).uniform_(lo, hi, generator=g)


def _product(a, b, transposed):
    """a b (or a b^T) in 64 bits, a run of rows of b at a time."""
    out, step = 0, 1024
    for i in range(0, b.shape[0], step):
        part = b[i:i + step].double()
        if transposed:
            out = torch.cat([out, a.double() @ part.t()], 1) if i else a.double() @ part.t()
        else:
            out = out + a[:, i:i + step].double() @ part
    return out


def _rounded(got, want, rel, dtype):
    off = (got.double() - want).abs() - want.abs() * (rel + torch.finfo(dtype).eps / 2 * (1 + rel))
    assert float(off.max()) <= 0, "%d of %d are off" % (int((off > 0).sum()), off.numel())


# 128 tokens by 38 tiles of 256 columns: more than half of the 74 pairs of CTAs have a tile, so that none is cut along k
LONG = [(F16, 1 << 17, 2.0 ** -9), (BF16, 1 << 19, 1.0)]


@pytest.mark.parametrize("dtype,n,size", LONG)
def test_long_sums_forward(B, dtype, n, size):
    T, C, O = 128, 8, 38 * 256
    x, w_in, w_down = _uniform((T, C), dtype, 1, 0.5, 1), _uniform((2 * n, C), dtype, 2, 0.1, 0.3), _uniform((O, n), dtype, 3, 0.5 * size, size)
    h, out = torch.empty(T, n, dtype=dtype, device=DEV), torch.empty(T, O, dtype=dtype, device=DEV)
    work = torch.empty(B.def_feed_forward_workspace(x, w_in, w_down, h) + 16, dtype=torch.uint8, device=DEV)
    B.def_feed_forward(x, w_in, w_down, h, out, workspace=work)
    _rounded(out, _product(h, w_down, True), _bound(dtype, n), dtype)


@pytest.mark.parametrize("dtype,n,size", LONG)
def test_long_sums_backward(B, dtype, n, size):
    """dx from 2F = n columns of dboth as stored; dup = dh g s from O = n outputs, g^ = u^ = 1."""
    for T, C, F, O in ((128, 38 * 256, n // 2, 8), (128, 8, 38 * 256, n)):
        small = C > 8
        dout = _uniform((T, O), dtype, 1, 0.5, 1)
        w_down = _uniform((O, F), dtype, 2, 0.1, 0.3) if small else _uniform((O, F), dtype, 2, 0.5 * size, size)
        w_in = _uniform((2 * F, C), dtype, 3, 0.5 * size, size) if small else None
        cks = [B.def_checkpoint_alloc(T, F, DEV) for _ in range(2)]
        for q, e in cks:
            q.fill_(64)
            e.fill_(121)
        dboth, dx = torch.empty(T, 2 * F, dtype=dtype, device=DEV), torch.empty(T, C, dtype=dtype, device=DEV) if small else None
        work = torch.empty(B.def_feed_forward_backward_workspace(dout, w_in, w_down, dboth) + 16, dtype=torch.uint8, device=DEV)
        B.def_feed_forward_backward(dout, w_in, w_down, *cks, dboth, dx, workspace=work)
        if small:
            _rounded(dx, _product(dboth, w_in, False), _bound(dtype, n), dtype)
        else:
            s = torch.sigmoid(torch.tensor(1.0, dtype=torch.float64)).item()
            # beside the sum: g s and its product with dh; s by the hardware's exponential (2^-21 twice) and quotient (2^-21)
            _rounded(dboth[:, F:], _product(dout, w_down, False) * s, _bound(dtype, n) + 3 * 2.0 ** -21 + 4 * U32, dtype)


@pytest.mark.parametrize("dtype,n,size", [(F16, 1 << 16, 2.0 ** -9), (BF16, 1 << 18, 1.0)])
@pytest.mark.parametrize("T", [1, 20])
def test_long_sums_of_few_tokens(B, dtype, n, size, T):
    """Weights of 150 and more tiles of 128 rows, so that k is not cut over a cluster."""
    C, O = 8, 150 * 128
    x, w_in, w_down = _uniform((T, C), dtype, 1, 0.5, 1), _uniform((2 * n, C), dtype, 2, 0.1, 0.3), _uniform((O, n), dtype, 3, 0.5 * size, size)
    h, out = torch.empty(T, n, dtype=dtype, device=DEV), torch.empty(T, O, dtype=dtype, device=DEV)
    work = torch.empty(B.def_feed_forward_workspace(x, w_in, w_down, h) + 16, dtype=torch.uint8, device=DEV)
    B.def_feed_forward(x, w_in, w_down, h, out, workspace=work)
    _rounded(out, _product(h, w_down, True), _bound(dtype, n), dtype)


@pytest.mark.parametrize("T", [1, 20])
def test_few_tokens_empty_their_sums(B, T):
    """The gated product of few tokens over many terms of either sign, and one output: several emptyings a cluster's CTA."""
    C, F = 5000 * 8, 152
    x, w_in, w_down = _uniform((T, C), F16, 1, -1, 1), _uniform((2 * F, C), F16, 2, -2.0 ** -6, 2.0 ** -6), _uniform((8, F), F16, 3, -1, 1)
    h, out = torch.empty(T, F, dtype=F16, device=DEV), torch.empty(T, 8, dtype=F16, device=DEV)
    work = torch.empty(B.def_feed_forward_workspace(x, w_in, w_down, h) + 16, dtype=torch.uint8, device=DEV)
    B.def_feed_forward(x, w_in, w_down, h, out, workspace=work)
    both, mag = x.double() @ w_in.double().t(), x.double().abs() @ w_in.double().abs().t()
    g, u, err = both[:, :F], both[:, F:], _bound(F16, C) * mag
    want = g * torch.sigmoid(g) * u
    # silu's slope is at most 1.1; the logistic function is off by 2^-21 (2 + |g|), three roundings
    off = 1.1 * err[:, :F] * u.abs() + (g.abs() + err[:, :F]) * err[:, F:] + want.abs() * (2.0 ** -21 * (2 + g.abs()) + 4 * U32)
    over = (h.double() - want).abs() - off - 2.0 ** -11 * (want.abs() + off) - 2.0 ** -25
    assert float(over.max()) <= 0
