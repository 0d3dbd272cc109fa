"""The gated linear recurrence on the GPU in every form it takes (blocks by tensor copies or element by element; in clusters, alone, and in
parts of time): sequences kept apart whatever they hold, packed sequences in parts, memories of very many tokens."""
import math

import pytest
import torch

from test_recurrence_gpu import _check, _cuts, _laid, _normal, _work

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


# few steps; clusters; elements off alignment; odd widths; parts of time, by copies and by elements
FORMS = [(60, 64, "rows"), (600, 64, "rows"), (600, 700, "padded"), (600, 65, "rows"), (600, 66, "off"), (3000, 700, "off"), (16384, 8, "rows"), (16384, 66, "padded"),
         (6000, 7, "rows"), (6000, 200, "off")]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,C,layout", FORMS)
def test_what_a_sequence_holds_stays_there(B, T, C, layout, dtype):
    """NaN and infinities in tokens, gates, states and gradients of some sequences and channels, and in rows of no sequence: all else has
    the bits it has without them."""
    cuts = [i * T // 60 for i in (0, 10, 25, 25, 40, 47, 50)]
    S, pad = len(cuts) - 1, cuts[-1]
    one, two = (3 % C, C // 2)
    x, gate, dy = (_normal((T, C), dtype, i, 1.0, m) for i, m in ((1, 0.0), (2, 2.0), (3, 0.0)))
    h0, dlast = _normal((S, C), F32, 4), _normal((S, C), F32, 5)
    off, work = torch.tensor(cuts, device=DEV), _work(B, T, C, dtype)

    def run(x, gate, dy, h0, dlast):
        x, gate, dy = (_laid(v, layout) for v in (x, gate, dy))
        y, dx, dg = (_laid(torch.full((T, C), 5.0, dtype=dtype, device=DEV), layout) for _ in range(3))
        last, dh0 = (torch.full((S, C), 5.0, device=DEV) for _ in range(2))
        B.def_recurrence_forward(x, gate, y, h0=h0, h_last=last, sequences=S, offsets=off, workspace=work)
        B.def_recurrence_backward(dy, x, gate, y, dx, dg, h0=h0, dh_last=dlast, dh0=dh0, sequences=S, offsets=off, workspace=work)
        return y, last, dx, dg, dh0

    clean = run(x, gate, dy, h0, dlast)
    assert all(bool(torch.isfinite(v).all()) for v in clean)
    bad = [v.clone() for v in (x, gate, dy, h0, dlast)]
    x_, gate_, dy_, h0_, dlast_ = bad
    early, late = cuts[1] + (cuts[2] - cuts[1]) // 3, cuts[4] + 2          # in sequences 1 and 4
    x_[early, one], gate_[early + 1, two], dy_[early + 2, one] = math.inf, math.nan, math.nan
    x_[late, two], dy_[late, two] = math.nan, -math.inf
    h0_[2, one], dlast_[2, two] = math.nan, math.inf                       # of the empty sequence: it hands them on
    h0_[4, one], dlast_[4, one] = -math.inf, math.nan
    x_[pad:], gate_[pad:], dy_[pad:] = math.nan, math.inf, math.nan
    y, last, dx, dg, dh0 = run(*bad)

    touched = torch.zeros(T, C, dtype=torch.bool, device=DEV)              # rows by channels that may differ
    states = torch.zeros(S, C, dtype=torch.bool, device=DEV)
    touched[cuts[1]:cuts[2], [one, two]] = True
    touched[cuts[4]:cuts[5], [one, two]] = True
    for s in (1, 2, 4):
        states[s, [one, two]] = True
    for got, want, mask in zip((y, last, dx, dg, dh0), clean, (touched, states, touched, touched, states)):
        assert torch.equal(got[~mask], want[~mask])
    assert torch.equal(y[cuts[1]:early, [one, two]], clean[0][cuts[1]:early, [one, two]])          # before them, in their own sequence
    assert torch.equal(dx[early + 3:cuts[2], one], clean[2][early + 3:cuts[2], one])               # behind them
    assert not bool(torch.isfinite(y[early, one])) and bool(torch.isnan(last[1, two])) and bool(torch.isnan(dx[early + 2, one]))
    assert bool(torch.isnan(last[2, one])) and bool(torch.isinf(dh0[2, two])) and bool(torch.isnan(dg[cuts[4]:cuts[5], one]).any())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,C,layout", [(16384, 8, "rows"), (9000, 66, "padded"), (6000, 7, "rows"), (4500, 200, "off")])
def test_packed_sequences_in_parts(B, T, C, layout, dtype):
    """Sequences that start, end and are empty anywhere in the parts, states in and out, rows of none behind."""
    assert B.def_recurrence_workspace(T, C, dtype) > 0
    _check(B, T, C, dtype, 3, layout, S=9, offsets=_cuts(T, 9, 1, T - 77), mean=4.0)
    _check(B, T, C, dtype, 4, layout, S=200, offsets=_cuts(T, 200, 2, T), mean=4.0, state=False)
    _check(B, T, C, dtype, 5, layout, S=5, offsets=[100, 100, T // 2, T // 2, T - 1, T], mean=6.0)


def _scan(a, b):
    """s_t = a_t s_{t-1} + b_t along the rows, 64 bits: each round joins runs of k rows to runs of 2 k."""
    k = 1
    while k < a.shape[0]:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


@pytest.mark.parametrize("T,C,layout", [(1 << 18, 64, "rows"), (1 << 18, 33, "off"), (1 << 16, 1024, "rows"), (1 << 15, 4800, "rows")])
def test_memories_of_many_tokens(B, T, C, layout):
    """c = (k + 1/2) 2^-24, which 1 - c in fp32 is off by half a unit from: a state that is folded with it at every step drifts by 2^-25
    a step, a fraction 1 / (2 k + 1) of what it should lose.  Runs of 8 steps are folded at once here: a rounding of what they keep
    (2^-25), one where runs are joined, one of the state (2^-24), all at most 2^-26 a step; 2^-20 for what happens within a block."""
    k = 60 + torch.arange(C, device=DEV, dtype=torch.float64) % 40
    c = (k + 0.5) * 2.0 ** -24
    g = torch.log((1 - c) / c).float()
    exact = torch.sigmoid(-g.double())
    assert float(((exact * 2 ** 24 - k - 0.5).abs()).max()) < 0.02
    gate = _laid(g.expand(T, C), layout)
    x, dy = (_laid(1 + _normal((T, C), F32, i, 0.3), layout) for i in (1, 2))
    y, dx, dg = (_laid(torch.zeros(T, C, device=DEV), layout) for _ in range(3))
    last, dh0, work = torch.empty(1, C, device=DEV), torch.empty(1, C, device=DEV), _work(B, T, C, F32)
    B.def_recurrence_forward(x, gate, y, h_last=last, workspace=work)
    B.def_recurrence_backward(dy, x, gate, y, dx, dg, dh0=dh0, workspace=work)
    step = max(1, (1 << 23) // T)
    for i in range(0, C, step):                                            # some channels at a time
        part = slice(i, min(C, i + step))
        e = exact[part].expand(T, -1)
        for gots, b in (((last[0, part], y[-1, part]), e * x[:, part].double()), ((dh0[0, part],), (1 - e) * dy[:, part].double().flip(0))):
            want, most = _scan(1 - e, b), _scan(1 - e, b.abs())
            off = _scan(1 - e, 2.0 ** -26 * most)[-1] + 2.0 ** -20 * most[-1]
            for got in gots:
                worst = float(((got.double() - want[-1]).abs() / off).max())
                assert worst <= 1, worst


@pytest.mark.parametrize("S,C,layout", [(40, 64, "rows"), (200, 64, "rows"), (40, 33, "off")])
def test_states_handed_on_from_call_to_call(B, S, C, layout):
    """One token of each sequence a call, c = (k + 1/2) 2^-24: what a step with a rounded 1 - c drifts, 2^-25, adds up to 6 10^-4 in all channels
    alike.  The other roundings, of the state by up to half a unit in the last place, 2^-24 / sqrt(12) of it in the mean square, are as
    random as the tokens.  But 50 tokens recur, and the state moves by a thousandth only, so that what they leave may recur, too: N / 50 times
    the sum of 50 such errors, N / sqrt(50) 2^-24 / sqrt(12) = 4.9 10^-5 (8 standard deviations allowed), independent from one channel and
    sequence to another, so that their mean over all S C of them is less by sqrt(S C)."""
    N = 20000
    k = 60 + torch.arange(C, device=DEV, dtype=torch.float64) % 40
    g = torch.log((1 - (k + 0.5) * 2.0 ** -24) / ((k + 0.5) * 2.0 ** -24)).float()
    c = torch.sigmoid(-g.double())
    gate = _laid(g.expand(S, C), layout)
    tokens = [_laid(1 + _normal((S, C), F32, i, 0.3), layout) for i in range(50)]
    dys = [_laid(1e-5 * t, layout) for t in tokens]
    y, dx, dg = (_laid(torch.zeros(S, C, device=DEV), layout) for _ in range(3))
    state, grad, spare, spare_grad = (torch.ones(S, C, device=DEV) for _ in range(4))
    want, want_grad = (torch.ones(S, C, device=DEV, dtype=torch.float64) for _ in range(2))
    x64, dy64 = [t.double() for t in tokens], [t.double() for t in dys]
    for i in range(N):
        B.def_recurrence_forward(tokens[i % 50], gate, y, h0=state, h_last=spare, sequences=S)
        B.def_recurrence_backward(dys[i % 50], tokens[0], gate, y, dx, dg, dh_last=grad, dh0=spare_grad, sequences=S)
        state, spare, grad, spare_grad = spare, state, spare_grad, grad
        want = (1 - c) * want + c * x64[i % 50]
        want_grad = (1 - c) * (want_grad + dy64[i % 50])
    # (backward dy + mu is rounded, too)
    for got, exact, roundings in ((state, want, 1), (grad, want_grad, 2)):
        off = (got.double() - exact) / exact
        most = 8 * 2.0 ** -24 * N / math.sqrt(50) * math.sqrt(roundings / 12)
        assert float(off.abs().max()) < most and abs(float(off.mean())) < most / math.sqrt(S * C)
