"""Cases and plain forms of the operators between a language model's input and the gradient rows def_step reads: a gated
linear recurrence over tokens, the gated feed-forward block, and the orthogonalised update of a weight matrix.

`run` computes a case in elementary torch operations (fp32 inside, one rounding at the end), or through the library's
entry points when `own` is set.  `exact` states each operator again in fp64."""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
SIZE = {"float32": 4, "bfloat16": 2, "float16": 2}
GROUP = 32                                  # columns of a row that share one exponent of a checkpoint
COEFFS = (3.4445, -4.7750, 2.0315)          # of the odd polynomial that drives singular values towards 1
EPS = 1e-7


def listed():
    return [
        # Recurrence over tokens.  One token of each of 64 sequences, states kept between calls: sampling while training.
        {"name": "recurrence 64 single tokens", "op": "rec_fwd", "dtype": "bfloat16", "T": 64, "C": 2048, "sequences": 64, "ragged": False, "state": True},
        # A training forward pass over a packed batch: eight documents of different lengths, padding at the end.
        {"name": "recurrence packed batch", "op": "rec_fwd", "dtype": "bfloat16", "T": 16384, "C": 4096, "sequences": 8, "ragged": True, "state": False},
        # One long document through a narrow fp32 model: few channels, so time itself has to be cut.
        {"name": "recurrence narrow and long", "op": "rec_fwd", "dtype": "float32", "T": 16384, "C": 512, "sequences": 1, "ragged": False, "state": True},
        # Backward of a short ragged batch of odd width (rows are not aligned), with states carried in and out.
        {"name": "recurrence back odd", "op": "rec_bwd", "dtype": "float16", "T": 1533, "C": 1111, "sequences": 13, "ragged": True, "state": True},
        # Backward of the packed training batch.
        {"name": "recurrence back packed batch", "op": "rec_bwd", "dtype": "bfloat16", "T": 16384, "C": 4096, "sequences": 8, "ragged": True, "state": False},
        # Feed-forward block.  One token: the weights are what has to be read.
        {"name": "feed-forward 1 token", "op": "ffn_fwd", "dtype": "bfloat16", "T": 1, "C": 2048, "F": 5632},
        # Evaluation of a small fp32 model.
        {"name": "feed-forward fp32", "op": "ffn_fwd", "dtype": "float32", "T": 1024, "C": 1024, "F": 2816},
        # A training step's forward and backward pass through a small layer, ragged on all sides.
        {"name": "feed-forward train ragged", "op": "ffn_train", "dtype": "float16", "T": 1501, "C": 777, "F": 1000},
        # The same for a large block and a whole batch: where the matrix products count.
        {"name": "feed-forward train large", "op": "ffn_train", "dtype": "bfloat16", "T": 8192, "C": 4096, "F": 10240},
        # Orthogonalised updates.  One small weight of a language model in the gradient rows of four workers.
        {"name": "orthogonalize 4 small", "op": "ortho", "dtype": "float32", "batch": 4, "rows": 256, "cols": 640, "steps": 5},
        # A tall 16-bit momentum of odd sizes.
        {"name": "orthogonalize odd bf16", "op": "ortho", "dtype": "bfloat16", "batch": 1, "rows": 1000, "cols": 777, "steps": 5},
        # The large projection of a block.
        {"name": "orthogonalize large", "op": "ortho", "dtype": "float32", "batch": 1, "rows": 4096, "cols": 10240, "steps": 5},
    ]


def _size(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5 and n >= 128:
        n = n // 64 * 64
    return min(hi, max(lo, n))


def draw(rng):
    op = rng.choice(["rec_fwd", "rec_bwd", "ffn_fwd", "ffn_train", "ffn_bwd", "ortho"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    wide = 2 if dtype == "float32" else 1
    if op == "ortho":
        m, n, steps = _size(rng, 16, 4096), _size(rng, 16, 10240), rng.choice([3, 5])
        m, n = min(m, n), max(m, n)
        batch = min(rng.choice([1, 1, 2, 4, 7]), max(1, 4096 * 4096 * 10240 // (m * m * n)))
        rows, cols = (n, m) if rng.random() < 0.4 else (m, n)
        return {"op": op, "dtype": dtype, "batch": batch, "rows": rows, "cols": cols, "steps": steps}
    if op in ("rec_fwd", "rec_bwd"):
        C = _size(rng, 16, 8192)
        T = min(_size(rng, 1, 16384), max(1, 16384 * 4096 // (C * wide)))
        ragged = rng.random() < 0.6
        sequences = _size(rng, 1, max(1, min(T, 300))) if ragged else rng.choice([s for s in (1, 2, 3, 5, 8, 16, T) if T % s == 0])
        return {"op": op, "dtype": dtype, "T": T, "C": C, "sequences": sequences, "ragged": ragged, "state": rng.random() < 0.5}
    if op == "ffn_train" and dtype == "float32":
        op = "ffn_bwd"
    C, F = _size(rng, 32, 4096), _size(rng, 32, 10240)
    most = 8192 * 4096 * 10240 // (8 if dtype == "float32" else 1)
    return {"op": op, "dtype": dtype, "T": min(_size(rng, 1, 8192), max(1, most // (C * F))), "C": C, "F": F}


def work(case):
    op, s = case["op"], SIZE[case["dtype"]]
    if op == "ortho":
        m, n = sorted((case["rows"], case["cols"]))
        return {"bytes": 2 * s * case["batch"] * m * n, "flops": case["steps"] * case["batch"] * (3 * m * m * n + m ** 3)}
    T, C = case["T"], case["C"]
    if op in ("rec_fwd", "rec_bwd"):
        states = case["sequences"] * C * 4 * (2 if op == "rec_fwd" else 3) if case["state"] else 0
        return {"bytes": s * T * C * (3 if op == "rec_fwd" else 6) + states, "flops": (10 if op == "rec_fwd" else 16) * T * C}
    F = case["F"]
    ck = T * (F + -(-F // GROUP))                        # bytes of a checkpoint of [T, F]
    weights, fwd, bwd = 3 * s * C * F, s * T * (2 * C + F), s * T * (2 * C + 2 * F)
    if op == "ffn_fwd":                                  # x in; h, out out
        return {"bytes": weights + fwd, "flops": 6 * T * C * F}
    if op == "ffn_bwd":                                  # dout and two checkpoints in; [dg | du], dx, h^ out
        return {"bytes": weights + bwd + 3 * ck, "flops": 6 * T * C * F}
    return {"bytes": 2 * weights + fwd + bwd + 5 * ck, "flops": 12 * T * C * F}


def _padded(C):
    """Bytes per row of a checkpoint: of the 8-bit integers, and of the exponents."""
    return -(-C // 16) * 16, -(-(-(-C // GROUP)) // 4) * 4


def _quantise(x):
    """The checkpoint (q, e) of x [T, C]: k = max(floor(log2 amax) - 6, -126) for each group of 32 columns,
    q = rne(x 2^-k) within +-127, e = k + 127."""
    T, C = x.shape
    g = torch.nn.functional.pad(x.float(), (0, -C % GROUP)).view(T, -1, GROUP)
    amax = g.abs().amax(2, keepdim=True)
    k = torch.where(amax > 0, (torch.frexp(amax)[1] - 7).clamp(min=-126), -126).int()
    q = (g * ((127 - k) << 23).view(torch.float32)).round().clamp(-127, 127).to(torch.int8).view(T, -1)[:, :C]
    ldq, lde = _padded(C)
    e = (k + 127).to(torch.uint8).view(T, -1)
    return (torch.nn.functional.pad(q, (0, ldq - C)).contiguous(),
            torch.nn.functional.pad(e, (0, lde - e.shape[1])).contiguous())


def _values(ck, C):
    """The fp32 values a checkpoint stands for: q 2^(e - 127)."""
    q, e = ck
    T = q.shape[0]
    scale = (e[:, :-(-C // GROUP)].int() << 23).view(torch.float32)
    q = torch.nn.functional.pad(q[:, :C].float(), (0, -C % GROUP)).view(T, -1, GROUP)
    return (q * scale[:, :, None]).view(T, -1)[:, :C]


def prepare(case, seed):
    dev = torch.device("cuda")
    gen = torch.Generator(device=dev)
    gen.manual_seed(seed)
    op, dt, f32 = case["op"], DTYPES[case["dtype"]], torch.float32

    def normal(*shape, std=1.0, mean=0.0, dtype=dt):
        return torch.empty(shape, dtype=f32, device=dev).normal_(mean, std, generator=gen).to(dtype)

    def empty(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=dev)

    def channels(*shape):                               # a few channels of an activation are far larger than the others
        x = normal(*shape, dtype=f32)
        loud = torch.rand(shape[-1], device=dev, generator=gen) < 0.01
        return torch.where(loud, x * 12, x).to(dt)

    s = {"case": case}
    if op == "ortho":
        b, m, n = case["batch"], case["rows"], case["cols"]
        # a momentum: a few directions carry most of it
        x, k = normal(b, m, n, std=1e-3, dtype=f32), min(m, n, 8)
        x += normal(b, m, k, std=2e-3, dtype=f32) @ normal(b, k, n, dtype=f32)
        s.update(x=x.to(dt), out=empty(b, m, n), scale=math.sqrt(max(1.0, m / n)))
        m, n = min(m, n), max(m, n)
        s["workspace"] = empty(b * (16 * (m + 8) * (n + m + 16) + 8192) + 4096, dtype=torch.uint8)
        return s
    T, C = case["T"], case["C"]
    if op in ("rec_fwd", "rec_bwd"):
        S = case["sequences"]
        s.update(x=normal(T, C), offsets=None, h0=normal(S, C, dtype=f32) if case["state"] else None)
        bias = torch.rand(C, device=dev, generator=gen) * 6 - 1     # channels remember from one token to some hundred
        s["gate"] = (normal(T, C, dtype=f32) + bias).to(dt)
        if case["ragged"]:                              # sorted cuts (some sequences are empty), padding at the end
            used = T - int(torch.randint(0, T // 16 + 1, (), device=dev, generator=gen))
            cuts = torch.randint(0, used + 1, (S - 1,), device=dev, generator=gen).sort().values
            s["offsets"] = torch.cat([cuts.new_zeros(1), cuts, cuts.new_full((1,), used)])
        s["workspace"] = empty(4096 * C + 4096, dtype=torch.uint8)
        if op == "rec_fwd":
            s.update(y=torch.zeros(T, C, dtype=dt, device=dev), h_last=empty(S, C, dtype=f32) if case["state"] else None)
        else:
            y = _plain_rec_fwd(dict(s, y=torch.zeros(T, C, dtype=dt, device=dev), h_last=None))["y"]
            s.update(y=y, dy=normal(T, C, std=0.02), dx=torch.zeros(T, C, dtype=dt, device=dev), dgate=torch.zeros(T, C, dtype=dt, device=dev),
                     dh_last=normal(S, C, std=0.02, dtype=f32) if case["state"] else None, dh0=empty(S, C, dtype=f32) if case["state"] else None)
        return s
    F = case["F"]

    def checkpoint(cols):
        ldq, lde = _padded(cols)
        return empty(T, ldq, dtype=torch.int8), empty(T, lde, dtype=torch.uint8)

    s.update(w_in=normal(2 * F, C, std=1 / math.sqrt(C)), w_down=normal(C, F, std=1 / math.sqrt(F)), x=channels(T, C), h=empty(T, F), out=empty(T, C))
    if op != "ffn_fwd":
        s.update(dout=normal(T, C, std=0.02), dboth=empty(T, 2 * F), dx=empty(T, C), gate_ck=checkpoint(F), up_ck=checkpoint(F), h_ck=checkpoint(F),
                 held=[empty(T, F, dtype=torch.bfloat16) for _ in range(3)])
    if op == "ffn_bwd":
        both = s["x"] @ s["w_in"].t()
        s.update(gate_ck=_quantise(both[:, :F]), up_ck=_quantise(both[:, F:]))
    planes, r = 3 if dt is f32 else 1, lambda n: n + 8
    s["workspace"] = empty(2 * planes * (T * (r(C) + r(2 * F)) + 2 * F * r(C) + C * r(F)) + (72 << 20), dtype=torch.uint8)
    return s


def run(s):
    op = s["case"]["op"]
    return (OWN if own else PLAIN)[op](s)


# --- plain forms ------------------------------------------------------------------------------------------------


def _scan(a, b):
    """h_t = a_t h_{t-1} + b_t along the rows: each round joins runs of k rows to runs of 2 k."""
    k = 1
    while k < a.shape[0]:
        b = torch.cat([b[:k], b[k:] + a[k:] * b[:-k]])
        a = torch.cat([a[:k], a[k:] * a[:-k]])
        k *= 2
    return b


def _sequences(s):
    """(first rows, rows behind the last ones) of the sequences, and for each row: its sequence, whether there is one, whether
    it is the first, whether it is the last of it."""
    T, S = s["x"].shape[0], s["case"]["sequences"]
    o = s["offsets"]
    if o is None:
        o = torch.arange(S + 1, device=s["x"].device) * (T // S)
    t = torch.arange(T, device=o.device)
    seq = torch.searchsorted(o[1:].contiguous(), t, right=True).clamp(max=S - 1)
    there = t < o[S]
    return o[:-1], o[1:], seq, there, there & (t == o[:-1][seq]), there & (t == o[1:][seq] - 1)


def _plain_rec_fwd(s):
    x, c = s["x"].float(), 1 / (1 + torch.exp(s["gate"].float()))
    first, behind, seq, there, starts, _ = _sequences(s)
    a, b = 1 - c, c * x
    if s["h0"] is not None:
        b = torch.where(starts[:, None], a * s["h0"][seq] + b, b)
    h = _scan(torch.where(starts[:, None], 0.0, a), b)
    out = {"y": torch.where(there[:, None], h.to(s["x"].dtype), s["y"])}
    if s["h_last"] is not None:
        out["h_last"] = torch.where((behind > first)[:, None], h[(behind - 1).clamp(min=0)], s["h0"])
    return out


def _plain_rec_bwd(s):
    x, dy, dt = s["x"].float(), s["dy"].float(), s["x"].dtype
    c = 1 / (1 + torch.exp(s["gate"].float()))
    first, behind, seq, there, starts, ends = _sequences(s)
    a = 1 - c
    if s["dh_last"] is not None:
        dy = torch.where(ends[:, None], dy + s["dh_last"][seq], dy)
    later = torch.cat([a[1:], a[:1]])                   # of the token behind
    lam = _scan(torch.where(ends[:, None], 0.0, later).flip(0), torch.where(there[:, None], dy, 0.0).flip(0)).flip(0)
    before = torch.cat([s["y"][:1], s["y"][:-1]]).float()
    before = torch.where(starts[:, None], 0.0 if s["h0"] is None else s["h0"][seq], before)
    dx, dgate = c * lam, lam * (before - x) * (a * c)
    out = {"dx": torch.where(there[:, None], dx.to(dt), s["dx"]), "dgate": torch.where(there[:, None], dgate.to(dt), s["dgate"])}
    if s["dh0"] is not None:
        at = first.clamp(max=x.shape[0] - 1)
        out["dh0"] = torch.where((behind > first)[:, None], a[at] * lam[at], s["dh_last"])
    return out


def _plain_ffn_fwd(s):
    F, dt = s["case"]["F"], s["x"].dtype
    both = s["x"].float() @ s["w_in"].float().t()
    g, u = both[:, :F], both[:, F:]
    h = g / (1 + torch.exp(-g)) * u
    return {"h": h.to(dt), "out": (h @ s["w_down"].float().t()).to(dt)}, g, u


def _plain_ffn_back(s, gate_ck, up_ck):
    F, dt = s["case"]["F"], s["x"].dtype
    g, u = _values(gate_ck, F), _values(up_ck, F)
    dh = s["dout"].float() @ s["w_down"].float()
    sg = 1 / (1 + torch.exp(-g))
    dboth = torch.cat([dh * u * (sg * (1 + g * (1 - sg))), dh * (g * sg)], 1)
    h = _values(_quantise((g * sg * u).to(dt)), F)
    return {"dboth": dboth.to(dt), "dx": (dboth @ s["w_in"].float()).to(dt), "h_held": h.to(torch.bfloat16)}


def _plain_ffn_bwd(s):
    return _plain_ffn_back(s, s["gate_ck"], s["up_ck"])


def _plain_ffn_train(s):
    out, g, u = _plain_ffn_fwd(s)
    gate_ck, up_ck, F = _quantise(g), _quantise(u), s["case"]["F"]
    out.update(_plain_ffn_back(s, gate_ck, up_ck))
    return dict(out, gate_held=_values(gate_ck, F).to(torch.bfloat16), up_held=_values(up_ck, F).to(torch.bfloat16))


def _plain_ortho(s):
    x, (a, b, c) = s["x"].float(), COEFFS
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    x = x / (torch.sqrt(x.double().square().sum((1, 2), keepdim=True)) + EPS).float()
    for _ in range(s["case"]["steps"]):                 # each step reads what the one before gives
        gram = x @ x.transpose(1, 2)
        x = a * x + (b * gram + c * (gram @ gram)) @ x
    x = x.transpose(1, 2) if tall else x
    return {"out": (s["scale"] * x).to(s["x"].dtype).contiguous()}


PLAIN = {"rec_fwd": _plain_rec_fwd, "rec_bwd": _plain_rec_bwd, "ffn_fwd": lambda s: _plain_ffn_fwd(s)[0], "ffn_bwd": _plain_ffn_bwd,
         "ffn_train": _plain_ffn_train, "ortho": _plain_ortho}


# --- the library's entry points ---------------------------------------------------------------------------------


def _lib():
    from paper_2004_05298_b200 import binding
    return binding


def _own_rec_fwd(s):
    _lib().def_recurrence_forward(s["x"], s["gate"], s["y"], h0=s["h0"], h_last=s["h_last"], sequences=s["case"]["sequences"],
                                  offsets=s["offsets"], workspace=s["workspace"])
    return {"y": s["y"]} if s["h_last"] is None else {"y": s["y"], "h_last": s["h_last"]}


def _own_rec_bwd(s):
    _lib().def_recurrence_backward(s["dy"], s["x"], s["gate"], s["y"], s["dx"], s["dgate"], h0=s["h0"], dh_last=s["dh_last"], dh0=s["dh0"],
                                   sequences=s["case"]["sequences"], offsets=s["offsets"], workspace=s["workspace"])
    out = {"dx": s["dx"], "dgate": s["dgate"]}
    return out if s["dh0"] is None else dict(out, dh0=s["dh0"])


def _own_ffn_fwd(s):
    _lib().def_feed_forward(s["x"], s["w_in"], s["w_down"], s["h"], s["out"], workspace=s["workspace"])
    return {"h": s["h"], "out": s["out"]}


def _own_ffn_bwd(s):
    B = _lib()
    B.def_feed_forward_backward(s["dout"], s["w_in"], s["w_down"], s["gate_ck"], s["up_ck"], s["dboth"], s["dx"], h_ck=s["h_ck"], workspace=s["workspace"])
    B.def_checkpoint_unpack(s["h_ck"], s["held"][0])
    return {"dboth": s["dboth"], "dx": s["dx"], "h_held": s["held"][0]}


def _own_ffn_train(s):
    B = _lib()
    B.def_feed_forward(s["x"], s["w_in"], s["w_down"], s["h"], s["out"], gate_ck=s["gate_ck"], up_ck=s["up_ck"], workspace=s["workspace"])
    out = _own_ffn_bwd(s)
    B.def_checkpoint_unpack(s["gate_ck"], s["held"][1])
    B.def_checkpoint_unpack(s["up_ck"], s["held"][2])
    return dict(out, h=s["h"], out=s["out"], gate_held=s["held"][1], up_held=s["held"][2])


def _own_ortho(s):
    _lib().def_orthogonalize(s["x"], s["out"], coeffs=[COEFFS] * s["case"]["steps"], eps=EPS, scale=s["scale"], workspace=s["workspace"])
    return {"out": s["out"]}


OWN = {"rec_fwd": _own_rec_fwd, "rec_bwd": _own_rec_bwd, "ffn_fwd": _own_ffn_fwd, "ffn_bwd": _own_ffn_bwd, "ffn_train": _own_ffn_train,
       "ortho": _own_ortho}


# --- the definitions in 64 bits -----------------------------------------------------------------------------------


def _spans(s):
    """(first row, row behind the last) of each sequence, as numbers."""
    T, S = s["case"]["T"], s["case"]["sequences"]
    o = [i * (T // S) for i in range(S + 1)] if s["offsets"] is None else s["offsets"].tolist()
    return list(zip(o[:-1], o[1:]))


def _rec_forward64(s):
    x, g = s["x"].double(), s["gate"].double()
    y = torch.zeros_like(x)
    last = torch.zeros(s["case"]["sequences"], x.shape[1], dtype=torch.float64, device=x.device)
    keep = torch.sigmoid(g)
    for i, (lo, hi) in enumerate(_spans(s)):
        h = last[i] if s["h0"] is None else s["h0"][i].double()
        for t in range(lo, hi):                          # token after token
            h = torch.lerp(x[t], h, keep[t])
            y[t] = h
        last[i] = h
    return {"y": y, "h_last": last} if s["h0"] is not None else {"y": y}


def _rec_backward64(s):
    x, g, dy, y = (s[k].double() for k in ("x", "gate", "dy", "y"))
    keep, let = torch.sigmoid(g), torch.sigmoid(-g)
    dx, dgate = torch.zeros_like(x), torch.zeros_like(x)
    dh0 = torch.zeros(s["case"]["sequences"], x.shape[1], dtype=torch.float64, device=x.device)
    for i, (lo, hi) in enumerate(_spans(s)):
        into = dh0[i] if s["dh_last"] is None else s["dh_last"][i].double()   # what reaches h_t from behind
        for t in range(hi - 1, lo - 1, -1):
            into = into + dy[t]
            dx[t] = into                                 # of h_t; its parts are taken below for all tokens at once
            into = into * keep[t]
        dh0[i] = into
        before = torch.cat([torch.zeros_like(dh0[i:i + 1]) if s["h0"] is None else s["h0"][i:i + 1].double(), y[lo:max(lo, hi - 1)]])[:hi - lo]
        dgate[lo:hi] = dx[lo:hi] * keep[lo:hi] * let[lo:hi] * (before - x[lo:hi])
        dx[lo:hi] *= let[lo:hi]
    return {"dx": dx, "dgate": dgate, "dh0": dh0} if s["dh0"] is not None else {"dx": dx, "dgate": dgate}


def _held(x):
    """What an 8-bit checkpoint of x holds, in 64 bits: a group's step is the power of two that puts its largest
    magnitude in [64, 128)."""
    x = x.double()
    T, C = x.shape
    out = torch.empty_like(x)
    whole = C // GROUP * GROUP
    for part, width in ((slice(0, whole), GROUP), (slice(whole, C), C - whole)):
        if width and x[:, part].numel():
            v = x[:, part].reshape(T, -1, width)
            top = v.abs().max(2, keepdim=True).values
            step = torch.exp2(torch.round(torch.log2(top.clamp(min=2.0 ** -140))) - 6)
            step = torch.where(top < 64 * step, step / 2, step).clamp(min=2.0 ** -126)
            out[:, part] = (torch.round(v / step).clamp(-127, 127) * step).reshape(T, -1)
    return out


def _ffn64(s):
    op, F = s["case"]["op"], s["case"]["F"]
    w_in, w_down, o = s["w_in"].double(), s["w_down"].double(), {}
    if op == "ffn_bwd":
        g, u = (q[:, :F].double() * torch.exp2(e.double() - 127).repeat_interleave(GROUP, 1)[:, :F] for q, e in (s["gate_ck"], s["up_ck"]))
    else:
        x = s["x"].double()
        g, u = torch.matmul(x, w_in[:F].t()), torch.matmul(x, w_in[F:].t())
        h = g * torch.sigmoid(g) * u
        o.update(h=h, out=torch.matmul(h, w_down.t()))
        if op == "ffn_fwd":
            return o
        g, u = _held(g), _held(u)
        o.update(gate_held=g, up_held=u)
    sig = torch.sigmoid(g)
    dh = torch.matmul(s["dout"].double(), w_down)
    dg, du = dh * u * (sig + g * sig * (1 - sig)), dh * g * sig
    o.update(dboth=torch.cat([dg, du], 1), dx=torch.matmul(dg, w_in[:F]) + torch.matmul(du, w_in[F:]),
             h_held=_held((g * sig * u).to(s["x"].dtype)))
    return o


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "rec_fwd":
        return _rec_forward64(s)
    if op == "rec_bwd":
        return _rec_backward64(s)
    if op != "ortho":
        return _ffn64(s)
    # X <- p(X X^T) X moves each singular value by itself: x <- x (a + b x^2 + c x^4).  With the eigenvalues t = x^2 of the
    # scaled X X^T the whole is X times a polynomial in t, in the basis of the eigenvectors.
    x = s["x"].double()
    tall = x.shape[1] > x.shape[2]
    x = x.transpose(1, 2) if tall else x
    x = x / (torch.linalg.matrix_norm(x, keepdim=True) + EPS)
    t, v = torch.linalg.eigh(torch.matmul(x, x.transpose(1, 2)))
    factor = torch.ones_like(t)
    for _ in range(case["steps"]):
        now = t * factor ** 2
        factor = factor * (COEFFS[0] + now * (COEFFS[1] + now * COEFFS[2]))
    x = torch.matmul(v * factor[:, None, :], torch.matmul(v.transpose(1, 2), x))
    return {"out": s["scale"] * (x.transpose(1, 2) if tall else x).contiguous()}
