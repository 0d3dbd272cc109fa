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


def chain(n, pieces):
    """What fp32 sums of n exact products on tensor cores may be off, relative to the magnitudes summed: 1024 terms in a chain that
    truncates, 16 at a time, to a unit in the last place (64 u of 2 each), chains added in fp32, and, in pieces, the products that are
    left out (mid lo, lo mid, lo lo: 3 times 2^-24)."""
    return (2 * min(64, -(-n // 16)) + -(-n // 1024) + (3 + 6 if pieces else 0)) * U32


def feed_forward(x, w_in, w_down=None, h_dtype=None):
    """(g, u, h, out) in 64 bits and bounds for (g, u, h, out) before their rounding; out from h rounded to its type."""
    dtype, x, w_in = x.dtype, x.double(), w_in.double()
    F, pieces = w_in.shape[0] // 2, dtype == torch.float32
    both, mag = x @ w_in.t(), x.abs() @ w_in.abs().t()
    err = chain(x.shape[1], pieces) * mag
    g, u, eg, eu = both[:, :F], both[:, F:], err[:, :F], err[:, F:]
    h = g * torch.sigmoid(g) * u
    # silu's slope is at most 1.1; the gate's own error is that of the logistic function, and three roundings
    eh = 1.1 * eg * u.abs() + (g.abs() * eu + eg * eu) * torch.sigmoid(g).clamp(min=0) * 1.1 + h.abs() * (gate_error(g, dtype) + 4 * U32)
    if w_down is None:
        return (g, u, h, None), (eg, eu, eh, None)
    w = w_down.double()
    out = h @ w.t()
    eo = (eh + h.abs() * (0 if pieces else UNIT[dtype])) @ w.abs().t() * 1.01 + chain(F, pieces) * (h.abs() @ w.abs().t())
    return (g, u, h, out), (eg, eu, eh, eo)


def feed_backward(dout, w_in, w_down, g, u):
    """(dgate, dup, h^, dx) in 64 bits from the values g^, u^ that the checkpoints hold, and bounds before their rounding."""
    dtype = dout.dtype
    dout, w_in, w, g, u = (v.double() for v in (dout, w_in, w_down, g, u))
    F, pieces = g.shape[1], dtype == torch.float32
    dh, mag = dout @ w, dout.abs() @ w.abs()
    edh = chain(dout.shape[1], pieces) * mag
    s, e = torch.sigmoid(g), gate_error(g, dtype)
    slope = s * (1 + g * (1 - s))
    dg, du, h = dh * u * slope, dh * g * s, g * s * u
    # s (1 + g (1 - s)): s is off by s e; 1 - s by s e + U32 absolutely; a few roundings of terms of at most s (1 + |g|)
    e_slope = s * (1 + g.abs()) * (2 * e + 6 * U32)
    edg = u.abs() * (edh * slope.abs() + (dh.abs() + edh) * e_slope) + 3 * U32 * dg.abs()
    edu = (g * s).abs() * edh + du.abs() * (e + 4 * U32)
    eh = h.abs() * (e + 4 * U32)
    both, eboth = torch.cat([dg, du], 1), torch.cat([edg, edu], 1)
    dx = both @ w_in
    edx = (eboth + both.abs() * (0 if pieces else UNIT[dtype])) @ w_in.abs() * 1.01 + chain(2 * F, pieces) * (both.abs() @ w_in.abs())
    return (dg, du, h, dx), (edg, edu, eh, edx)


MUON = ((3.4445, -4.7750, 2.0315),) * 5


def orthogonalize(x, coeffs=MUON, eps=1e-7, scale=1.0):
    """(out, bound of the error's Frobenius norm) of one matrix in 64 bits.  f(s) = s (a + b s^2 + c s^4) takes an error of X to at
    most max |f'| times its Frobenius norm (divided differences of an odd function); a step adds what its three products and
    the 22 bits of A, B and X leave: 2^-22 of a value, 3 2^-22 for the product of the lower pieces, and the chains' truncation
    (512 terms, 16 at a time, two units each)."""
    x = x.double()
    tall = x.shape[0] > x.shape[1]
    X = x.t() if tall else x
    X = X / (X.norm() + eps)
    bits = 2.0 ** -22

    def chain(k, mags):
        return (2 * min(32, -(-k // 16)) * U32 + 3 * bits + -(-3 * k // 512) * U32) * float(mags.norm())

    err = bits * float(X.norm())
    for a, b, c in coeffs:
        m, n = X.shape
        A = X @ X.t()
        B = a * torch.eye(m, dtype=X.dtype, device=X.device) + b * A + c * A @ A
        sx, sa = float(torch.linalg.matrix_norm(X, 2)), float(torch.linalg.matrix_norm(A, 2))
        s = torch.linspace(0, sx, 1001, dtype=torch.float64)
        slope = float((a + 3 * b * s ** 2 + 5 * c * s ** 4).abs().max())
        eA = chain(n, X.abs() @ X.abs().t()) + bits * float(A.norm())
        eB = (abs(b) + 2 * abs(c) * sa) * eA + abs(c) * chain(m, A.abs() @ A.abs()) + bits * float(B.norm())
        Y = B @ X
        err = slope * err + sx * eB + chain(m, B.abs() @ X.abs()) + bits * float(Y.norm())
        X = Y
    return scale * (X.t() if tall else X), abs(scale) * err


def newton_schulz(x, coeffs=MUON, eps=1e-7, lost=(), mirrored=()):
    """The steps of one matrix in 64 bits (tall or wide); with X, A and B held in two fp16 pieces where `lost` is given: those it
    names without their lower piece, A or B of `mirrored` without it in tiles of 256 above the diagonal."""
    X = x.double().t() if x.shape[0] > x.shape[1] else x.double()
    pieces = lost is not None

    def hold(v, name):
        if not pieces:
            return v
        hi = (v * 4096).half().double()
        lo = (v * 4096 - hi).half().double() * (name not in lost)
        if name in mirrored:
            tile = torch.arange(v.shape[0]) // 256
            lo = torch.where(tile[:, None] < tile[None, :], 0.0, lo)
        return (hi + lo) / 4096

    X = hold(X / (X.norm() + eps), "X")
    for i, (a, b, c) in enumerate(coeffs):
        A = hold(X @ X.t(), "A")
        X = hold(a * torch.eye(len(A), dtype=X.dtype, device=X.device) + b * A + c * A @ A, "B") @ X
        if i + 1 < len(coeffs):
            X = hold(X, "X")
    return X.t() if x.shape[0] > x.shape[1] else X


# What fp32 results of five steps may be off, relative in Frobenius norm: plain fp32 sums leave 1 to 2 10^-6 at these sizes, two pieces
# 2 to 3 10^-7 more, the matrix unit's truncation (1.7 2^-24 for each of the 4 to 16 additions of a chain) somewhat more than the sums.
# Without the lower piece of X, A or B anywhere 3 10^-4 and more are missing, in mirrored tiles alone 9 10^-5 (600 x 700).
NEAR = 1e-5
