"""The recurrence, the feed-forward block and the orthogonalised update stated plainly in 64 bits, with bounds for what fp32
arithmetic may be off."""
import torch

from train_ref import U32, UNIT


def spans(T, S, offsets):
    o = [i * (T // S) for i in range(S + 1)] if offsets is None else [int(v) for v in offsets]
    return list(zip(o[:-1], o[1:]))


def gate_error(gate, dtype):
    """Relative error of 1 / (1 + exp(g)): the exponential (2 units in the last place in fp32, 2^-21 (1 + |g|) by the hardware's
    instruction for 16-bit types), a sum and an approximate quotient (2 units)."""
    g = gate.double().abs()
    return (2.0 ** -22 if dtype == torch.float32 else 2.0 ** -21 * (1 + g)) + 2.0 ** -21 + 0 * g


def recurrence(x, gate, spans_, h0=None):
    """h of every row (0 where there is no sequence), the states behind the sequences, and for both a bound of the error that
    fp32 states carry.  A step adds to the error (c e + 6 u)(m + |x|), m the magnitudes the state is made of: e the gate's
    error, u for each of the difference, the product, the sum, 1 - c, and what joining runs adds for a step."""
    dtype, x, g = x.dtype, x.double().cpu(), gate.double().cpu()
    c, a, e = torch.sigmoid(-g), torch.sigmoid(g), gate_error(gate.cpu(), dtype)
    C = x.shape[1]
    y, err = torch.zeros_like(x), torch.zeros_like(x)
    last, last_err = torch.zeros(len(spans_), C, dtype=torch.float64), torch.zeros(len(spans_), C, dtype=torch.float64)
    for s, (lo, hi) in enumerate(spans_):
        h = torch.zeros(C, dtype=torch.float64) if h0 is None else h0[s].double().cpu()
        m, E = h.abs(), torch.zeros_like(h)
        for t in range(lo, hi):
            E = a[t] * E + (c[t] * e[t] + 6 * U32) * (m + x[t].abs())
            h = a[t] * h + c[t] * x[t]
            m = a[t] * m + c[t] * x[t].abs()
            y[t], err[t] = h, E
        last[s], last_err[s] = h, E
    return y, err, last, last_err


def recurrence_backward(dy, x, gate, y, spans_, h0=None, dh_last=None):
    """(dx, dgate, dh0) and a bound of what fp32 leaves them off (before a 16-bit output is rounded)."""
    dtype = x.dtype
    dy, x, g, y = (v.double().cpu() for v in (dy, x, gate, y))
    c, a, e = torch.sigmoid(-g), torch.sigmoid(g), gate_error(gate.cpu(), dtype)
    out = [torch.zeros_like(x) for _ in range(4)]
    dx, dg, dx_err, dg_err = out
    dh0, dh0_err = (torch.zeros(len(spans_), x.shape[1], dtype=torch.float64) for _ in range(2))
    for s, (lo, hi) in enumerate(spans_):
        mu = torch.zeros(x.shape[1], dtype=torch.float64) if dh_last is None else dh_last[s].double().cpu()
        m, E = mu.abs(), torch.zeros_like(mu)
        for t in range(hi - 1, lo - 1, -1):
            lam, m = dy[t] + mu, dy[t].abs() + m
            E = E + U32 * m
            before = y[t - 1] if t > lo else torch.zeros_like(mu) if h0 is None else h0[s].double().cpu()
            diff, size = before - x[t], before.abs() + x[t].abs()
            dx[t], dg[t] = c[t] * lam, lam * diff * a[t] * c[t]
            dx_err[t] = c[t] * (E + (e[t] + 2 * U32) * m)
            # 1 - c is off by c e + u, absolutely
            dg_err[t] = c[t] * (a[t] * diff.abs() * E + m * size * (a[t] * (e[t] + 6 * U32) + c[t] * e[t] + 2 * U32))
            E = a[t] * E + (c[t] * e[t] + 6 * U32) * m
            mu, m = a[t] * lam, a[t] * m
        dh0[s], dh0_err[s] = mu, E
    return (dx, dg, dh0), (dx_err, dg_err, dh0_err)


def within(got, want, err, dtype):
    """Asserts that got is want with one rounding to dtype and an error of at most err before it."""
    got, want = got.double().cpu(), want.double().cpu()
    tiny = {torch.float32: 2.0 ** -126, torch.bfloat16: 2.0 ** -126, torch.float16: 2.0 ** -25}[dtype]
    tol = UNIT[dtype] * want.abs() + err * (1 + UNIT[dtype]) + tiny
    assert torch.equal(torch.isnan(got), torch.isnan(want))
    over = torch.nan_to_num((got - want).abs() - tol, nan=0.0)
    assert over.numel() == 0 or float(over.max()) <= 0, "off by %g beyond the bound" % float(over.max())
