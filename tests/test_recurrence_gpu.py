"""The gated linear recurrence on the GPU against its statement in 64 bits (tests/block_ref.py has the error bounds)."""
import math

import pytest
import torch

import block_ref as R

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


def _normal(shape, dtype, seed, std=1.0, mean=0.0):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return torch.empty(shape, device=DEV).normal_(mean, std, generator=g).to(dtype)


def _laid(x, layout):
    """x in contiguous rows, in padded rows, or one element off any alignment with an odd stride."""
    T, C = x.shape
    if layout == "rows":
        return x.contiguous()
    pad = 16 - C % 8 if layout == "padded" else 3 - C % 2
    off = 0 if layout == "padded" else 1
    buf = torch.full((T * (C + pad) + 64,), 7.0, dtype=x.dtype, device=DEV)
    v = buf[off:off + T * (C + pad)].view(T, C + pad)[:, :C]
    v.copy_(x)
    return v


def _work(B, T, C, dtype):
    return torch.empty(max(16, B.def_recurrence_workspace(T, C, dtype)), dtype=torch.uint8, device=DEV)


def _cuts(T, S, seed, used):
    g = torch.Generator()
    g.manual_seed(seed)
    return [0] + sorted(torch.randint(0, used + 1, (S - 1,), generator=g).tolist()) + [used]


def _check(B, T, C, dtype, seed=0, layout="rows", S=1, offsets=None, state=True, mean=2.0):
    spans = R.spans(T, S, offsets)
    x, gate = _laid(_normal((T, C), dtype, seed), layout), _laid(_normal((T, C), dtype, seed + 1, 2.0, mean), layout)
    h0 = _normal((S, C), F32, seed + 2) if state else None
    y, last = _laid(torch.full((T, C), 5.0, dtype=dtype, device=DEV), layout), torch.full((S, C), 5.0, device=DEV)
    off = None if offsets is None else torch.tensor(offsets, dtype=torch.int64, device=DEV)
    work = _work(B, T, C, dtype)
    B.def_recurrence_forward(x, gate, y, h0=h0, h_last=last, sequences=S, offsets=off, workspace=work)
    want, err, want_last, last_err = R.recurrence(x, gate, spans, h0)
    held = torch.zeros(T, dtype=torch.bool)
    for lo, hi in spans:
        held[lo:hi] = True
    R.within(y[held.to(DEV)], want[held], err[held], dtype)
    R.within(last, want_last, last_err, F32)
    assert bool((y[~held.to(DEV)] == 5).all()), "a row of no sequence was written"

    dy = _laid(_normal((T, C), dtype, seed + 3, 0.1), layout)
    dlast = _normal((S, C), F32, seed + 4, 0.1) if state else None
    dx, dg = (_laid(torch.full((T, C), 5.0, dtype=dtype, device=DEV), layout) for _ in range(2))
    dh0 = torch.full((S, C), 5.0, device=DEV)
    B.def_recurrence_backward(dy, x, gate, y, dx, dg, h0=h0, dh_last=dlast, dh0=dh0, sequences=S, offsets=off, workspace=work)
    (wx, wg, w0), (ex, eg, e0) = R.recurrence_backward(dy, x, gate, y, spans, h0, dlast)
    R.within(dx[held.to(DEV)], wx[held], ex[held], dtype)
    R.within(dg[held.to(DEV)], wg[held], eg[held], dtype)
    R.within(dh0, w0, e0, F32)
    assert bool((dx[~held.to(DEV)] == 5).all()) and bool((dg[~held.to(DEV)] == 5).all()), "a row of no sequence was written"


@pytest.mark.parametrize("layout", ["rows", "padded", "off"])
@pytest.mark.parametrize("dtype", TYPES)
def test_sizes(B, dtype, layout):
    for i, (T, C) in enumerate([(1, 1), (1, 64), (2, 65), (15, 2), (16, 33), (17, 31), (127, 64), (128, 66), (129, 128), (300, 130), (777, 5)]):
        _check(B, T, C, dtype, 10 * i, layout, state=i % 2 == 0)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,C", [(2501, 700), (1100, 2050), (300, 9000), (5000, 8), (4097, 1)])
def test_clusters_and_parts(B, T, C, dtype):
    """Sizes at which CTAs of a cluster, one CTA alone, and parts of time share a sequence."""
    _check(B, T, C, dtype, 3, mean=4.0)


@pytest.mark.parametrize("dtype", TYPES)
def test_packed_sequences(B, dtype):
    for i, (T, C, S, used) in enumerate([(40, 66, 13, 33), (1533, 111, 7, 1533), (700, 640, 300, 650), (2000, 3, 1500, 1999), (130, 64, 5, 0), (3000, 700, 9, 2900)]):
        _check(B, T, C, dtype, 20 * i, S=S, offsets=_cuts(T, S, i, used), layout="off" if i % 2 else "rows", state=i != 2)


def test_packed_sequences_that_start_late(B):
    _check(B, 100, 64, BF16, 1, S=3, offsets=[20, 50, 50, 90])


@pytest.mark.parametrize("dtype", TYPES)
def test_equally_long_sequences(B, dtype):
    for T, S in ((64, 64), (96, 32), (640, 2), (1500, 3), (300, 300)):
        _check(B, T, 130, dtype, T, S=S)


def test_no_tokens(B):
    e = torch.empty(0, 6, dtype=BF16, device=DEV)
    h0, last = _normal((4, 6), F32, 1), torch.empty(4, 6, device=DEV)
    B.def_recurrence_forward(e, e, e, h0=h0, h_last=last, sequences=4)
    assert torch.equal(last, h0)
    B.def_recurrence_forward(e, e, e, h_last=last, sequences=4, offsets=torch.zeros(5, dtype=torch.int64, device=DEV))
    assert bool((last == 0).all())
    B.def_recurrence_backward(e, e, e, e, e, e, dh_last=h0, dh0=last, sequences=4)
    assert torch.equal(last, h0)


def test_token_by_token_is_the_whole(B):
    """A state handed on from call to call is the state of one call: the same steps, each bounded by the same error."""
    T, S, C = 24, 5, 70
    x, gate = _normal((S * T, C), BF16, 1), _normal((S * T, C), BF16, 2, 2.0, 1.0)
    y, last = torch.empty_like(x), torch.empty(S, C, device=DEV)
    B.def_recurrence_forward(x, gate, y, h_last=last, sequences=S)
    state, step = torch.zeros(S, C, device=DEV), torch.empty(S, C, dtype=BF16, device=DEV)
    for t in range(T):
        new = torch.empty_like(state)
        B.def_recurrence_forward(x[t::T], gate[t::T], step, h0=state, h_last=new, sequences=S)
        state = new
    want, err, want_last, last_err = R.recurrence(x, gate, R.spans(S * T, S, None))
    R.within(state, want_last, last_err, F32)
    R.within(step, want[T - 1::T], err[T - 1::T], BF16)


@pytest.mark.parametrize("C", [64, 700])
def test_infinities_and_nan_stay_in_their_sequence(B, C):
    T = 600
    offsets = [0, 100, 250, 250, 500]
    x, gate = _normal((T, C), F32, 1), _normal((T, C), F32, 2)
    x[120, 3], gate[130, 5], x[130, 7], gate[110, 9], gate[111, 10] = math.inf, math.nan, math.nan, math.inf, -math.inf
    x[500:] = math.nan                                                       # rows of no sequence
    y, last = torch.zeros_like(x), torch.empty(4, C, device=DEV)
    off, work = torch.tensor(offsets, device=DEV), _work(B, T, C, F32)
    B.def_recurrence_forward(x, gate, y, h_last=last, sequences=4, offsets=off, workspace=work)
    want, _, _, _ = R.recurrence(x, gate, R.spans(T, 4, offsets))
    assert bool(torch.isfinite(y[:100]).all()) and bool(torch.isfinite(y[250:]).all())
    ok = torch.ones(C, dtype=torch.bool)
    ok[[3, 5, 7]] = False
    assert bool(torch.isfinite(y[100:250].cpu()[:, ok]).all()) and not bool(torch.isfinite(last[1].cpu()[~ok]).any())
    assert bool((y[110, 9] == y[109, 9]).all()), "a gate of infinity keeps the state"
    assert bool((y[111, 10] == x[111, 10]).all()), "a gate of -infinity lets the token through"
    dx, dg, dh0 = torch.zeros_like(x), torch.zeros_like(x), torch.empty(4, C, device=DEV)
    dy = _normal((T, C), F32, 3)
    dy[200, 11], dy[510:] = math.nan, math.nan
    B.def_recurrence_backward(dy, x, gate, y, dx, dg, dh0=dh0, sequences=4, offsets=off, workspace=work)
    assert bool(torch.isfinite(dx[:100]).all()) and bool(torch.isfinite(dx[250:]).all()) and bool(torch.isnan(dx[100:201, 11]).all())
    assert bool(torch.isfinite(dx[201:250, 11]).all())


def test_in_place_strides_streams_and_graphs(B):
    """y over x; columns of one projection's output; another stream; a captured call replayed on other values and offsets."""
    T, C, S = 900, 96, 6
    both = _normal((T, 2 * C), BF16, 5)
    x, gate = both[:, :C], both[:, C:]
    y = torch.empty(T, C, dtype=BF16, device=DEV)
    work = _work(B, T, C, BF16)
    B.def_recurrence_forward(x, gate, y, sequences=S, workspace=work)
    again = x.clone()
    B.def_recurrence_forward(again, gate, again, sequences=S, workspace=work)
    assert torch.equal(again, y)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    z, off = torch.zeros_like(y), torch.tensor(_cuts(T, S, 1, T), device=DEV)
    with torch.cuda.stream(side):
        B.def_recurrence_forward(x, gate, z, sequences=S, offsets=off, workspace=work, stream=side)
    side.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        B.def_recurrence_forward(x, gate, z, sequences=S, offsets=off, workspace=work, stream=torch.cuda.current_stream())
    new = _cuts(T, S, 2, T - 30)
    both.copy_(_normal((T, 2 * C), BF16, 6))
    off.copy_(torch.tensor(new))
    z.fill_(5)
    graph.replay()
    torch.cuda.synchronize()
    want, err, _, _ = R.recurrence(x, gate, R.spans(T, S, new))
    R.within(z[:T - 30], want[:T - 30], err[:T - 30], BF16)
    assert bool((z[T - 30:] == 5).all())


def test_repeated_calls_give_the_same_bits(B):
    for T, C in ((3000, 700), (5000, 16)):
        x, gate = _normal((T, C), F32, 1), _normal((T, C), F32, 2, 1.0, 3.0)
        work, outs = _work(B, T, C, F32), [torch.empty(T, C, device=DEV) for _ in range(4)]
        for y in outs:
            B.def_recurrence_forward(x, gate, y, workspace=work)
        assert all(torch.equal(outs[0], y) for y in outs[1:])


def test_offsets_that_make_no_sense_stay_inside(B):
    """Decreasing offsets and offsets outside [0, T]: what is computed is not specified, but nothing else is written."""
    T, C = 400, 66
    buf = torch.full((T + 20, C), 5.0, dtype=BF16, device=DEV)
    y = buf[10:T + 10]
    x, gate, work = _normal((T, C), BF16, 1), _normal((T, C), BF16, 2), _work(B, T, C, BF16)
    for off in ([0, 300, 100, 400], [-50, 10, 20, 100000], [400, 300, 200, 0], [0, 1 << 40, -(1 << 50), 7]):
        last = torch.full((5, C), 5.0, device=DEV)
        B.def_recurrence_forward(x, gate, y, h_last=last[1:4], sequences=3, offsets=torch.tensor(off, device=DEV), workspace=work)
        assert bool((buf[:10] == 5).all()) and bool((buf[T + 10:] == 5).all()) and bool((last[0] == 5).all()) and bool((last[4] == 5).all())
