"""The gated feed-forward block on the GPU against its statement in 64 bits (tests/block_ref.py has the error bounds)."""
import math

import pytest
import torch

import block_ref as R
import train_ref

pytestmark = pytest.mark.gpu

F32, BF16, F16 = torch.float32, torch.bfloat16, torch.float16
TYPES = [F32, BF16, F16]
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


def _laid(x, layout):
    """x in contiguous rows, in rows padded to 16 bytes, or one element off any alignment with an odd stride."""
    T, C = x.shape
    if layout == "rows":
        return x.contiguous()
    pad = 16 - C % 8 if layout == "padded" else 3 - C % 2
    off = 0 if layout == "padded" else 1
    buf = torch.full((T * (C + pad) + 64,), 7.0, dtype=x.dtype, device=DEV)
    v = buf[off:off + T * (C + pad)].view(T, C + pad)[:, :C]
    v.copy_(x)
    return v


def _work(n):
    return torch.empty(max(n, 16), dtype=torch.uint8, device=DEV)


def _held(B, T, F):
    ck = B.def_checkpoint_alloc(T, F, DEV)
    ck[0].fill_(77)
    ck[1].fill_(77)
    return ck


def _values(ck, F):
    return train_ref.read(ck, F).to(DEV)


def _check_held(ck, x, err, F):
    """A checkpoint of x, known to within err: off by half a step and err, its step that of the group's largest magnitude (or,
    where err leaves that open, twice or half of it); the padding is left alone."""
    held = _values(ck, F)
    big = torch.nn.functional.pad((x.abs() + err), (0, -F % 32)).view(x.shape[0], -1, 32).amax(2).clamp(min=2.0 ** -120)
    step = torch.exp2(torch.floor(torch.log2(big)) - 6).repeat_interleave(32, 1)[:, :F]
    # 127.5 steps and more are held as 127
    assert bool(((held - x).abs() <= step * 0.5 + step * (x.abs() >= 127 * step) + err).all())
    groups = -(-F // 32)
    assert bool((ck[0][:, F:] == 77).all()) and bool((ck[1][:, groups:] == 77).all()), "padding was written"


def _check(B, T, C, F, O, dtype, seed=0, layout="rows", train=True):
    x = _laid(_normal((T, C), dtype, seed), layout)
    w_in, w_down = _normal((2 * F, C), dtype, seed + 1, 1 / math.sqrt(C)), _normal((O, F), dtype, seed + 2, 1 / math.sqrt(F))
    h, out = (_laid(torch.full((T, n), 5.0, dtype=dtype, device=DEV), layout) for n in (F, O))
    gate_ck, up_ck = (_held(B, T, F), _held(B, T, F)) if train else (None, None)
    work = _work(B.def_feed_forward_workspace(x, w_in, w_down, h))
    B.def_feed_forward(x, w_in, w_down, h, out, gate_ck, up_ck, workspace=work)
    (g, u, wh, wo), (eg, eu, eh, eo) = R.feed_forward(x, w_in, w_down)
    R.within(h, wh, eh.cpu(), dtype)
    R.within(out, wo, eo.cpu(), dtype)
    if not train:
        return
    _check_held(gate_ck, g, eg, F)
    _check_held(up_ck, u, eu, F)
    gv, uv = _values(gate_ck, F), _values(up_ck, F)
    dout = _laid(_normal((T, O), dtype, seed + 3, 0.1), layout)
    dboth, dx, back = (_laid(torch.full((T, n), 5.0, dtype=dtype, device=DEV), layout) for n in (2 * F, C, F))
    h_ck = _held(B, T, F)
    work = _work(B.def_feed_forward_backward_workspace(dout, w_in, w_down, dboth))
    B.def_feed_forward_backward(dout, w_in, w_down, gate_ck, up_ck, dboth, dx, h_out=back, h_ck=h_ck, workspace=work)
    (dg, du, wh, wx), (edg, edu, eh, ex) = R.feed_backward(dout, w_in, w_down, gv, uv)
    R.within(dboth[:, :F], dg, edg.cpu(), dtype)
    R.within(dboth[:, F:], du, edu.cpu(), dtype)
    R.within(back, wh, eh.cpu(), dtype)
    R.within(dx, wx, ex.cpu(), dtype)
    q, e = train_ref.pack(back)                                            # the checkpoint is that of the stored values
    assert torch.equal(h_ck[0][:, :F].long().cpu(), q) and torch.equal(h_ck[1][:, :e.shape[1]].long().cpu(), e)
    assert bool((h_ck[0][:, F:] == 77).all()) and bool((h_ck[1][:, e.shape[1]:] == 77).all()), "padding was written"


@pytest.mark.parametrize("layout", ["rows", "padded", "off"])
@pytest.mark.parametrize("dtype", TYPES)
def test_sizes(B, dtype, layout):
    for i, (T, C, F, O) in enumerate([(1, 1, 1, 1), (1, 64, 128, 64), (2, 7, 33, 5), (31, 100, 65, 129), (128, 64, 64, 256), (129, 65, 127, 40),
                                      (257, 72, 129, 257), (300, 200, 264, 96)]):
        _check(B, T, C, F, O, dtype, 10 * i, layout)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,C,F,O", [(5000, 64, 300, 64), (300, 1111, 2000, 777), (64, 2048, 1408, 2048), (700, 96, 9000, 32), (2500, 40, 1999, 33), (3000, 33, 5001, 70)])
def test_more_tiles_than_pairs_and_long_sums(B, dtype, T, C, F, O):
    _check(B, T, C, F, O, dtype, 5)


@pytest.mark.parametrize("dtype", TYPES)
def test_few_tokens(B, dtype):
    for T in (1, 2, 3, 5, 8, 9, 16, 17):
        for C, F, O in ((512, 704, 512), (2048, 300, 40), (33, 70, 1000)):
            _check(B, T, C, F, O, dtype, T, train=False)
        _check(B, T, 260, 140, 260, dtype, T)


def test_parts_alone(B):
    """h without the second product; the gradients of g and u without dx."""
    T, C, F = 200, 96, 160
    x, w_in, w_down = _normal((T, C), BF16, 1), _normal((2 * F, C), BF16, 2, 0.1), _normal((C, F), BF16, 3, 0.1)
    h, h2, out = torch.empty(T, F, dtype=BF16, device=DEV), torch.empty(T, F, dtype=BF16, device=DEV), torch.empty(T, C, dtype=BF16, device=DEV)
    cks = [_held(B, T, F) for _ in range(2)]
    B.def_feed_forward(x, w_in, w_down, h, out, *cks, workspace=_work(32 << 20))
    B.def_feed_forward(x, w_in, None, h2, None, workspace=_work(32 << 20))
    assert torch.equal(h, h2)
    dout, both, both2, dx = _normal((T, C), BF16, 4), *(torch.empty(T, 2 * F, dtype=BF16, device=DEV) for _ in range(2)), torch.empty(T, C, dtype=BF16, device=DEV)
    B.def_feed_forward_backward(dout, w_in, w_down, *cks, both, dx, workspace=_work(32 << 20))
    B.def_feed_forward_backward(dout, None, w_down, *cks, both2, None, workspace=_work(32 << 20))
    assert torch.equal(both, both2)
    empty = x[:0]
    B.def_feed_forward(empty, w_in, w_down, h[:0], out[:0])


def test_large_values_and_specials(B):
    """Gates far out saturate; a NaN or infinity in a token stays in its row; rows of zeros give zeros."""
    T, C, F = 130, 64, 96
    x, w_in, w_down = _normal((T, C), BF16, 1), _normal((2 * F, C), BF16, 2, 30.0), _normal((C, F), BF16, 3, 0.1)
    x[5], x[7, 3], x[9, 1] = 0, math.nan, math.inf
    h, out = torch.empty(T, F, dtype=BF16, device=DEV), torch.empty(T, C, dtype=BF16, device=DEV)
    cks = [_held(B, T, F) for _ in range(2)]
    B.def_feed_forward(x, w_in, w_down, h, out, *cks, workspace=_work(32 << 20))
    assert bool((h[5] == 0).all()) and bool((out[5] == 0).all())
    assert bool(torch.isnan(h[7]).all()) and bool(torch.isnan(out[7]).all()) and not bool(torch.isfinite(out[9]).any())
    rest = [i for i in range(T) if i not in (7, 9)]
    assert bool(torch.isfinite(h[rest]).all()) and bool(torch.isfinite(out[rest]).all())
    assert bool((cks[0][1][7, :3] == 255).all())
    (g, u, wh, _), (_, _, eh, _) = R.feed_forward(x[rest], w_in)
    R.within(h[rest], wh, eh.cpu(), BF16)


def test_streams_and_graphs(B):
    """On another stream, and captured and replayed on other values, the workspace included."""
    T, C, F = 333, 90, 130                                                 # rows that need aligned copies
    x, w_in, w_down = _normal((T, C), BF16, 1), _normal((2 * F, C), BF16, 2, 0.1), _normal((C, F), BF16, 3, 0.1)
    h, out = torch.empty(T, F, dtype=BF16, device=DEV), torch.empty(T, C, dtype=BF16, device=DEV)
    work = _work(B.def_feed_forward_workspace(x, w_in, w_down, h))
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        B.def_feed_forward(x, w_in, w_down, h, out, workspace=work, stream=side)
    side.synchronize()
    (_, _, wh, wo), (_, _, eh, eo) = R.feed_forward(x, w_in, w_down)
    R.within(out, wo, eo.cpu(), BF16)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.def_feed_forward(x, w_in, w_down, h, out, workspace=work, stream=torch.cuda.current_stream())
    x.copy_(_normal((T, C), BF16, 8))
    w_in.copy_(_normal((2 * F, C), BF16, 9, 0.1))
    graph.replay()
    torch.cuda.synchronize()
    (_, _, wh, wo), (_, _, eh, eo) = R.feed_forward(x, w_in, w_down)
    R.within(h, wh, eh.cpu(), BF16)
    R.within(out, wo, eo.cpu(), BF16)


def test_repeated_calls_give_the_same_bits(B):
    T, C, F = 700, 512, 640
    for dtype in (F32, BF16):
        x, w_in, w_down = _normal((T, C), dtype, 1), _normal((2 * F, C), dtype, 2, 0.1), _normal((C, F), dtype, 3, 0.1)
        hs, outs = [torch.empty(T, F, dtype=dtype, device=DEV) for _ in range(3)], [torch.empty(T, C, dtype=dtype, device=DEV) for _ in range(3)]
        work = _work(B.def_feed_forward_workspace(x, w_in, w_down, hs[0]))
        for h, out in zip(hs, outs):
            B.def_feed_forward(x, w_in, w_down, h, out, workspace=work)
        assert all(torch.equal(hs[0], v) for v in hs) and all(torch.equal(outs[0], v) for v in outs)


def test_a_whole_training_pass(B):
    """Forward, backward and the weights' gradients from the checkpoints, against the 64-bit gradient of the same loss: off by
    what 8 bits leave (half a step of 2^-6 of a group's largest magnitude) and 16-bit roundings."""
    T, C, F = 512, 256, 320
    x, w_in, w_down = _normal((T, C), BF16, 1), _normal((2 * F, C), BF16, 2, 1 / 16), _normal((C, F), BF16, 3, 1 / 18)
    dout = _normal((T, C), BF16, 4)
    h, out = torch.empty(T, F, dtype=BF16, device=DEV), torch.empty(T, C, dtype=BF16, device=DEV)
    gate_ck, up_ck, h_ck, x_ck = _held(B, T, F), _held(B, T, F), _held(B, T, F), _held(B, T, C)
    both, dx = torch.empty(T, 2 * F, dtype=BF16, device=DEV), torch.empty(T, C, dtype=BF16, device=DEV)
    dwi, dwd = torch.empty(2 * F, C, device=DEV), torch.empty(C, F, device=DEV)
    B.def_checkpoint_pack(x, x_ck)
    B.def_feed_forward(x, w_in, w_down, h, out, gate_ck, up_ck, workspace=_work(32 << 20))
    B.def_feed_forward_backward(dout, w_in, w_down, gate_ck, up_ck, both, dx, h_ck=h_ck, workspace=_work(32 << 20))
    for dy, ck, dw in ((both, x_ck, dwi), (dout, h_ck, dwd)):
        B.def_checkpoint_weight_grad(dy, ck, dw, _work(B.def_checkpoint_weight_grad_workspace(dy, dw.shape[1])))
    leaves = [v.double().requires_grad_() for v in (x, w_in, w_down)]
    gu = leaves[0] @ leaves[1].t()
    want = torch.nn.functional.silu(gu[:, :F]) * gu[:, F:] @ leaves[2].t()
    want.backward(dout.double())
    for got, leaf in zip((dx, dwi, dwd), leaves):
        rel = float((got.double() - leaf.grad).norm() / leaf.grad.norm())
        # g^, u^ and x^ or h^ are each within 2^-7 of a group's largest magnitude, uniformly (rms 2^-7 / sqrt(3) of up to 3.5 rms)
        assert rel < 3 * 3.5 * 2.0 ** -7 / math.sqrt(3), rel
