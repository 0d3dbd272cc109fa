"""Cases and plain forms of the operators around the optimizer step: norms before and after a block, 8-bit activation
checkpoints with the backward passes that read them, and token log probabilities with their gradient.

`run` computes a case in elementary torch operations (fp32 inside, one rounding at the end), or through the library's
entry points when `own` is set.  `exact` states each operator again in fp64."""
import math

import torch

own = False

DTYPES = {"float32": torch.float32, "bfloat16": torch.bfloat16, "float16": torch.float16}
SIZE = {"float32": 4, "bfloat16": 2, "float16": 2}
GROUP = 32                     # columns of a row that share one exponent of a checkpoint
EPS = 1e-6


def listed():
    return [
        # Norms around a block.  One token: a model evaluated token by token while samples are drawn from it, where
        # the launch counts.
        {"name": "norm forward, 1 token", "op": "norm_fwd", "dtype": "bfloat16", "T": 1, "C": 2048, "groups": 1},
        # A training forward pass: eight sequences of 2048 tokens, each with its own gate row.
        {"name": "norm forward, 16k tokens", "op": "norm_fwd", "dtype": "bfloat16", "T": 16384, "C": 4096, "groups": 8},
        # Backward on a short ragged batch with an odd width (rows are not aligned), activations kept as they are.
        {"name": "norm backward, odd", "op": "norm_bwd", "dtype": "float16", "T": 1533, "C": 1111, "groups": 1, "saved8": False},
        # Backward of a training step that kept its activations in 8 bits.
        {"name": "norm backward, 8-bit saves", "op": "norm_bwd", "dtype": "bfloat16", "T": 16384, "C": 4096, "groups": 8, "saved8": True},
        # Checkpoint written and read back: an fp32 model of odd width, a short batch.
        {"name": "checkpoint, fp32 odd", "op": "pack", "dtype": "float32", "T": 515, "C": 2501},
        # The same for a wide bf16 activation over a whole batch.
        {"name": "checkpoint, wide", "op": "pack", "dtype": "bfloat16", "T": 16384, "C": 8192},
        # Gated activation with its checkpoint, forward and backward: a small fp16 model, a handful of tokens.
        {"name": "gated, 48 tokens", "op": "gated", "dtype": "float16", "T": 48, "C": 1408},
        # The same in a large block.
        {"name": "gated, 8k tokens", "op": "gated", "dtype": "bfloat16", "T": 8192, "C": 10240},
        # Weight gradient from a checkpoint: a small layer, ragged on all sides.
        {"name": "weight gradient, ragged", "op": "wgrad", "dtype": "float16", "T": 1501, "C": 777, "O": 1000},
        # The large projection of a block over a whole batch: where the matrix product counts.
        {"name": "weight gradient, large", "op": "wgrad", "dtype": "bfloat16", "T": 8192, "C": 4096, "O": 8192},
        # One sampled token scored with its alternatives.
        {"name": "log probability, 1 token", "op": "logprob", "dtype": "float32", "T": 1, "C": 50001, "top": 20, "grad": False, "masked": False},
        # Loss and its gradient for a batch of tokens over a large vocabulary, part of it masked off.
        {"name": "log probability, 4k tokens", "op": "logprob", "dtype": "bfloat16", "T": 4096, "C": 128000, "top": 8, "grad": True, "masked": True},
    ]


def _size(rng, lo, hi):
    n = int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))
    if rng.random() < 0.5:
        n = max(lo, n // 64 * 64) if n >= 128 else n
    n = min(hi, max(lo, n))
    return n + 1 if n == 3 * 1024 else n


def draw(rng):
    op = rng.choice(["norm_fwd", "norm_bwd", "pack", "gated", "wgrad", "logprob"])
    dtype = rng.choice(["bfloat16", "bfloat16", "float16", "float32"])
    case = {"op": op, "dtype": dtype, "T": _size(rng, 1, 16384)}
    wide = 2 if dtype == "float32" else 1
    if op in ("norm_fwd", "norm_bwd"):
        case["C"] = _size(rng, 64, 8192)
        case["T"] = min(case["T"], max(1, (16384 * 4096) // (case["C"] * wide)))
        case["groups"] = rng.choice([g for g in (1, 2, 3, 5, 8) if case["T"] % g == 0])
        if op == "norm_bwd":
            case["saved8"] = rng.random() < 0.5
    elif op == "pack":
        case["C"] = _size(rng, 16, 16384)
        case["T"] = min(case["T"], max(1, (16384 * 8192) // (case["C"] * wide)))
    elif op == "gated":
        case["C"] = _size(rng, 64, 16384)
        case["T"] = min(case["T"], max(1, (8192 * 10240) // (case["C"] * wide)))
    elif op == "wgrad":
        case["C"], case["O"] = _size(rng, 32, 8192), _size(rng, 32, 8192)
        most = (8192 * 4096 * 8192) // (4 if dtype == "float32" else 1)
        case["T"] = min(case["T"], max(1, most // (case["C"] * case["O"])))
    else:
        case["C"] = _size(rng, 100, 200000)
        case["T"] = min(case["T"], max(1, (4096 * 128000) // (case["C"] * wide)))
        case["top"] = rng.choice([0, 1, 5, 8, 20, 32])
        case["grad"] = rng.random() < 0.6
        case["masked"] = rng.random() < 0.4
    return case


def work(case):
    T, C, s, op = case["T"], case["C"], SIZE[case["dtype"]], case["op"]
    ck = T * (C + -(-C // GROUP))                       # bytes of a checkpoint of [T, C]
    if op == "norm_fwd":
        return {"bytes": 4 * s * T * C + 8 * T + 4 * C * (2 + case["groups"]), "flops": 9 * T * C}
    if op == "norm_bwd":
        saves = 2 * ck if case["saved8"] else 2 * s * T * C
        return {"bytes": saves + 4 * s * T * C + 8 * T + 8 * C * (2 + case["groups"]), "flops": 20 * T * C}
    if op == "pack":                                    # written once, read back once
        return {"bytes": 2 * s * T * C + 2 * ck, "flops": 4 * T * C}
    if op == "gated":                                   # g, u, dh in; h, h^, dg, du out; two checkpoints written and read
        return {"bytes": 7 * s * T * C + 4 * ck, "flops": 30 * T * C}
    if op == "wgrad":
        return {"bytes": s * T * case["O"] + ck + 4 * case["O"] * C, "flops": 2 * T * C * case["O"]}
    grad = case["grad"]
    return {"bytes": s * T * C * (3 if grad else 1) + T * (24 + 12 * case["top"]), "flops": (11 if grad else 6) * T * C}


def _padded(C):
    """Bytes per row of a checkpoint: of the 8-bit integers, and of the exponents."""
    return -(-C // 16) * 16, -(-(-(-C // GROUP)) // 4) * 4


def _quantise(x):
    """The checkpoint (q, e) of x [T, C]: k = max(floor(log2 amax) - 6, -126) for each group of 32 columns,
    q = rne(x 2^-k) within +-127, e = k + 127; 255 marks a group that holds an infinity or a NaN."""
    T, C = x.shape
    g = torch.nn.functional.pad(x.float(), (0, -C % GROUP)).view(T, -1, GROUP)
    amax = g.abs().amax(2, keepdim=True)
    k = torch.where(amax > 0, (torch.frexp(amax)[1] - 7).clamp(min=-126), -126)
    bad = ~torch.isfinite(amax)
    k = torch.where(bad, 128, k).int()
    q = (g * ((127 - torch.where(bad, 0, k)) << 23).int().view(torch.float32)).round().clamp(-127, 127)
    q = torch.where(bad, 0.0, q).to(torch.int8).view(T, -1)[:, :C]
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
    T, C, op, dt = case["T"], case["C"], case["op"], DTYPES[case["dtype"]]

    def normal(*shape, std=1.0, mean=0.0, dtype=dt):
        return torch.empty(shape, dtype=torch.float32, device=dev).normal_(mean, std, generator=gen).to(dtype)

    def channels(*shape):                               # a few channels of an activation are far larger than the others
        x = normal(*shape, dtype=torch.float32)
        loud = torch.rand(shape[-1], device=dev, generator=gen) < 0.01
        return torch.where(loud, x * 12, x).to(dt)

    def empty(*shape, dtype=dt):
        return torch.empty(shape, dtype=dtype, device=dev)

    def checkpoint(cols):
        ldq, lde = _padded(cols)
        return empty(T, ldq, dtype=torch.int8), empty(T, lde, dtype=torch.uint8)

    s = {"case": case}
    if op in ("norm_fwd", "norm_bwd"):
        G = case["groups"]
        s.update(w_post=normal(C, std=0.2, mean=1.0, dtype=torch.float32), w_pre=normal(C, std=0.2, mean=1.0, dtype=torch.float32),
                 gate=normal(G, C, std=0.3, mean=0.5, dtype=torch.float32), scale=0.9375)
        h, b = channels(T, C), channels(T, C)
        if op == "norm_fwd":
            s.update(h=h, b=b, h_out=empty(T, C), n_out=empty(T, C), rstd_post=empty(T, dtype=torch.float32), rstd_pre=empty(T, dtype=torch.float32))
        else:
            f32 = torch.float32
            s.update(dn=normal(T, C, std=0.02), dh_in=normal(T, C, std=0.02),
                     rstd_post=torch.rsqrt(b.float().square().mean(1) + EPS), rstd_pre=torch.rsqrt(h.float().square().mean(1) + EPS),
                     h=_quantise(h) if case["saved8"] else h, b=_quantise(b) if case["saved8"] else b,
                     dh=empty(T, C), db=empty(T, C), dw_post=empty(C, dtype=f32), dgate=empty(G, C, dtype=f32), dw_pre=empty(C, dtype=f32))
            s["workspace"] = empty(_norm_workspace(T, C, G), dtype=torch.uint8)
    elif op == "pack":
        s.update(x=channels(T, C), ck=checkpoint(C), back=empty(T, C))
    elif op == "gated":
        both = normal(T, 2 * C, std=1.5)                # one projection's output: gate columns, then up columns
        s.update(gate=both[:, :C], up=both[:, C:], dh=normal(T, C, std=0.02), gate_ck=checkpoint(C), up_ck=checkpoint(C),
                 h=empty(T, C), h_back=empty(T, C), dboth=empty(T, 2 * C))
    elif op == "wgrad":
        s.update(dy=normal(T, case["O"], std=0.02), ck=_quantise(channels(T, C)), dw=empty(case["O"], C, dtype=torch.float32))
        s["workspace"] = empty(_wgrad_workspace(T, C, case["O"]), dtype=torch.uint8)
    else:
        x = normal(T, C, std=2.0)
        y = torch.randint(0, C, (T,), device=dev, generator=gen)
        rows = torch.arange(T, device=dev)
        x[rows, y] += 6.0                               # a model that has learnt something
        if case["masked"]:                              # tokens that may not come next, and prompt positions
            off = torch.rand(C, device=dev, generator=gen) < 0.2
            x = x.masked_fill_(off, -math.inf)
            x[rows, y] = 4.0
            y = torch.where(torch.rand(T, device=dev, generator=gen) < 0.1, -100, y)
        f32, k = torch.float32, case["top"]
        s.update(x=x, y=y, logp=empty(T, dtype=f32), entropy=empty(T, dtype=f32), lse=empty(T, 2, dtype=f32),
                 top_ids=empty(T, k, dtype=torch.int64) if k else None, top_logp=empty(T, k, dtype=f32) if k else None)
        if case["grad"]:                                # minus an advantage for each token, and an entropy bonus
            s.update(dlogp=normal(T, std=1.0 / T, dtype=f32), dentropy=torch.full((T,), -0.01 / T, device=dev),
                     dtop=normal(T, k, std=0.1 / T, dtype=f32) if k else None, dx=empty(T, C))
    return s


def _norm_workspace(T, C, G):
    """Bytes a user of the backward pass sets aside: at most 2048 partial rows of two sums, and a row per group."""
    return 8 * C * (min(T, 2048) + G + 8) + 4096


def _wgrad_workspace(T, C, O):
    """Bytes a user of the weight gradient sets aside: partial products, and an aligned copy of dY."""
    pad = -(-O // 8) * 8
    return 64 * 1024 * 1024 + 4 * 1024 * 1024 + 6 * T * pad + 4 * O * C * 2


def run(s):
    op = s["case"]["op"]
    return (OWN if own else PLAIN)[op](s)


# --- plain forms ------------------------------------------------------------------------------------------------


def _plain_norm_fwd(s):
    h, b = s["h"].float(), s["b"].float()
    T, C = h.shape
    G = s["gate"].shape[0]
    r2 = torch.rsqrt(b.square().mean(1) + EPS)
    gate = s["gate"].repeat_interleave(T // G, 0)
    h1 = s["scale"] * h + gate * (b * r2[:, None] * s["w_post"])
    r1 = torch.rsqrt(h1.square().mean(1) + EPS)
    n = h1 * r1[:, None] * s["w_pre"]
    return {"h": h1.to(s["h"].dtype), "n": n.to(s["h"].dtype), "rstd_post": r2, "rstd_pre": r1}


def _plain_norm_bwd(s):
    C, dt = s["dn"].shape[1], s["dn"].dtype
    h, b = (_values(s[k], C) if s["case"]["saved8"] else s[k].float() for k in ("h", "b"))
    T, G = h.shape[0], s["gate"].shape[0]
    dn, r1, r2 = s["dn"].float(), s["rstd_pre"][:, None], s["rstd_post"][:, None]
    x, y = h * r1, b * r2
    a = dn * s["w_pre"]
    D = s["dh_in"].float() + r1 * (a - x * (a * x).mean(1, keepdim=True))
    S = (D * y).view(G, T // G, C).sum(1)
    c = D * (s["gate"] * s["w_post"]).repeat_interleave(T // G, 0)
    db = r2 * (c - y * (c * y).mean(1, keepdim=True))
    return {"dh": (s["scale"] * D).to(dt), "db": db.to(dt), "dw_pre": (dn * x).sum(0), "dgate": s["w_post"] * S, "dw_post": (s["gate"] * S).sum(0)}


def _plain_pack(s):
    return {"x": _values(_quantise(s["x"]), s["x"].shape[1]).to(s["x"].dtype)}


def _plain_gated(s):
    g, u, dh, dt = s["gate"].float(), s["up"].float(), s["dh"].float(), s["dh"].dtype
    F = g.shape[1]
    h = g / (1 + torch.exp(-g)) * u
    g, u = _values(_quantise(g), F), _values(_quantise(u), F)
    sg = 1 / (1 + torch.exp(-g))
    dg = dh * u * (sg * (1 + g * (1 - sg)))
    return {"h": h.to(dt), "h_back": (g * sg * u).to(dt), "dboth": torch.cat([dg, dh * (g * sg)], 1).to(dt)}


def _plain_wgrad(s):
    return {"dw": s["dy"].float().t() @ _values(s["ck"], s["dw"].shape[1])}


def _plain_logprob(s):
    x, y = s["x"].float(), s["y"]
    T, V = x.shape
    m = x.amax(1, keepdim=True)
    ex = torch.exp(x - m)
    z = ex.sum(1, keepdim=True)
    lse = m + torch.log(z)
    p = ex / z
    at = torch.where(y < 0, 0, y)[:, None]
    logp = torch.where(y < 0, 0.0, (x.gather(1, at) - lse)[:, 0])
    lp = torch.where(p > 0, x - lse, 0.0)
    H = -(p * lp).sum(1)
    out = {"logp": logp, "entropy": H, "lse": torch.cat([m, torch.log(z)], 1)}
    k = s["case"]["top"]
    if k:                                               # by value, ties to the lowest index: unique 64-bit keys
        bits = torch.where(x == 0, 0.0, x).view(torch.int32).long()
        key = (torch.where(bits < 0, -2 ** 31 - 1 - bits, bits) << 32) + (2 ** 31 - 1 - torch.arange(V, device=x.device))
        ids = torch.topk(key, k, 1).indices
        out.update(top_ids=ids, top_logp=x.gather(1, ids) - lse)
    if s["case"]["grad"]:
        dlogp = torch.where(y < 0, 0.0, s["dlogp"])[:, None]
        dH = s["dentropy"][:, None]
        total = dlogp + s["dtop"].sum(1, keepdim=True) if k else dlogp
        dx = -p * (total + dH * (lp + H[:, None]))
        dx = dx.scatter_add(1, at, dlogp)
        dx = dx.scatter_add(1, ids, s["dtop"]) if k else dx
        out["dx"] = dx.to(s["x"].dtype)
    return out


PLAIN = {"norm_fwd": _plain_norm_fwd, "norm_bwd": _plain_norm_bwd, "pack": _plain_pack, "gated": _plain_gated,
         "wgrad": _plain_wgrad, "logprob": _plain_logprob}


# --- the library's entry points ---------------------------------------------------------------------------------


def _lib():
    from paper_2004_05298_b200 import binding
    return binding


def _own_norm_fwd(s):
    _lib().def_norm_forward(s["h"], s["b"], s["w_post"], s["gate"], s["w_pre"], s["h_out"], s["n_out"], s["rstd_post"], s["rstd_pre"],
                            res_scale=s["scale"], eps=EPS)
    return {"h": s["h_out"], "n": s["n_out"], "rstd_post": s["rstd_post"], "rstd_pre": s["rstd_pre"]}


def _own_norm_bwd(s):
    _lib().def_norm_backward(s["dn"], s["dh_in"], s["h"], s["b"], s["w_post"], s["gate"], s["w_pre"], s["rstd_post"], s["rstd_pre"],
                             s["dh"], s["db"], s["dw_post"], s["dgate"], s["dw_pre"], s["workspace"], res_scale=s["scale"])
    return {k: s[k] for k in ("dh", "db", "dw_pre", "dgate", "dw_post")}


def _own_pack(s):
    B = _lib()
    B.def_checkpoint_pack(s["x"], s["ck"])
    B.def_checkpoint_unpack(s["ck"], s["back"])
    return {"x": s["back"]}


def _own_gated(s):
    B, F = _lib(), s["h"].shape[1]
    B.def_gated_forward(s["gate"], s["up"], s["h"], s["gate_ck"], s["up_ck"])
    B.def_gated_backward(s["dh"], s["gate_ck"], s["up_ck"], s["dboth"][:, :F], s["dboth"][:, F:], h_out=s["h_back"])
    return {"h": s["h"], "h_back": s["h_back"], "dboth": s["dboth"]}


def _own_wgrad(s):
    _lib().def_checkpoint_weight_grad(s["dy"], s["ck"], s["dw"], s["workspace"])
    return {"dw": s["dw"]}


def _own_logprob(s):
    B = _lib()
    B.def_logprob_forward(s["x"], s["y"], s["logp"], s["entropy"], s["lse"], s["top_ids"], s["top_logp"])
    out = {"logp": s["logp"], "entropy": s["entropy"], "lse": s["lse"]}
    if s["top_ids"] is not None:
        out.update(top_ids=s["top_ids"], top_logp=s["top_logp"])
    if s["case"]["grad"]:
        B.def_logprob_backward(s["x"], s["y"], s["lse"], s["entropy"], s["dx"], dlogp=s["dlogp"], dentropy=s["dentropy"],
                               top_ids=s["top_ids"], dtop_logp=s["dtop"])
        out["dx"] = s["dx"]
    return out


OWN = {"norm_fwd": _own_norm_fwd, "norm_bwd": _own_norm_bwd, "pack": _own_pack, "gated": _own_gated, "wgrad": _own_wgrad,
       "logprob": _own_logprob}


# --- the definitions in 64 bits -----------------------------------------------------------------------------------


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


def _read(ck, C):
    q, e = ck
    step = torch.exp2(e.double() - 127).repeat_interleave(GROUP, 1)[:, :C]
    return q[:, :C].double() * step


def exact(case, seed):
    s, op = prepare(case, seed), case["op"]
    if op == "norm_fwd":
        h, b = s["h"].double(), s["b"].double()
        rp = 1 / torch.sqrt((b * b).mean(1) + EPS)
        per = h.shape[0] // case["groups"]
        h1 = torch.empty_like(h)
        for g in range(case["groups"]):
            at = slice(g * per, (g + 1) * per)
            h1[at] = s["scale"] * h[at] + s["gate"][g].double() * s["w_post"].double() * b[at] * rp[at, None]
        r = 1 / torch.sqrt((h1 * h1).mean(1) + EPS)
        return {"h": h1, "n": h1 * s["w_pre"].double() * r[:, None], "rstd_post": rp, "rstd_pre": r}
    if op == "norm_bwd":
        # The Jacobian of v -> v r(v) applied to a vector is r (a - v r^2 <a, v> / C); rows of a group at a time.
        C, T, G = case["C"], case["T"], case["groups"]
        per = T // G
        wp, w = s["w_post"].double(), s["w_pre"].double()
        dw, dwp = torch.zeros_like(w), torch.zeros_like(wp)
        dh, db, dgate = [], [], []
        for g in range(G):
            at = slice(g * per, (g + 1) * per)
            h, b = ((_read((s[k][0][at], s[k][1][at]), C)) if case["saved8"] else s[k][at].double() for k in ("h", "b"))
            r, rp, dn = s["rstd_pre"][at, None].double(), s["rstd_post"][at, None].double(), s["dn"][at].double()
            v = w * dn
            tot = s["dh_in"][at].double() + r * v - h * (r ** 3 * (v * h).sum(1, keepdim=True) / C)
            v = s["gate"][g].double() * wp * tot
            dh.append(s["scale"] * tot)
            db.append(rp * v - b * (rp ** 3 * (v * b).sum(1, keepdim=True) / C))
            dw += (dn * h * r).sum(0)
            through = (tot * b * rp).sum(0)
            dgate.append(wp * through)
            dwp += s["gate"][g].double() * through
        return {"dh": torch.cat(dh), "db": torch.cat(db), "dw_pre": dw, "dgate": torch.stack(dgate), "dw_post": dwp}
    if op == "pack":
        return {"x": _held(s["x"])}
    if op == "gated":
        g, u, dh = s["gate"].double(), s["up"].double(), s["dh"].double()
        h = g * torch.sigmoid(g) * u
        g, u = _held(g), _held(u)
        sig = torch.sigmoid(g)
        return {"h": h, "h_back": g * sig * u, "dboth": torch.cat([dh * u * (sig + g * sig * (1 - sig)), dh * g * sig], 1)}
    if op == "wgrad":
        return {"dw": torch.matmul(s["dy"].double().t(), _read(s["ck"], case["C"]))}
    outs = []
    for at in range(0, case["T"], 512):                 # some rows at a time: 64 bits of a large vocabulary are many bytes
        at = slice(at, at + 512)
        x, y = s["x"][at].double(), s["y"][at]
        lp = torch.log_softmax(x, 1)
        p = lp.exp()
        plp = torch.where(p > 0, p * lp, 0.0)
        H = -plp.sum(1)
        given = y >= 0
        rows = torch.arange(x.shape[0], device=x.device)
        o = {"logp": torch.where(given, lp[rows, y.clamp(min=0)], 0.0), "entropy": H, "lse": torch.stack([x.amax(1), torch.logsumexp(x, 1) - x.amax(1)], 1)}
        if case["top"]:
            ids = torch.sort(x, dim=1, descending=True, stable=True).indices[:, :case["top"]]
            o.update(top_ids=ids, top_logp=lp.gather(1, ids))
        if case["grad"]:
            w, d = torch.where(given, s["dlogp"][at].double(), 0.0), torch.zeros_like(x)
            d[rows, y.clamp(min=0)] += w
            mass = w.clone()
            if case["top"]:
                d.scatter_add_(1, ids, s["dtop"][at].double())
                mass += s["dtop"][at].double().sum(1)
            gH = s["dentropy"][at].double()
            o["dx"] = d - p * mass[:, None] - gH[:, None] * (plp + p * H[:, None])
        outs.append(o)
    out = {k: torch.cat([o[k] for o in outs]) for k in outs[0]}
    if "top_ids" in out:
        out["top_ids"] = None
    return out
