"""The operators of include/def_train.h stated plainly in 64 bits (numpy / torch float64), for the tests."""
import math

import torch

UNIT = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}   # half a unit in the last place, relative
U32 = 2.0 ** -24


def group_pad(x):
    T, C = x.shape
    return torch.nn.functional.pad(x, (0, -C % 32)).view(T, -1, 32)


def pack(x):
    """(q [T, C], e [T, ceil(C / 32)]) as int64, by search over the exponents rather than from the bits."""
    g = group_pad(x.double().cpu())
    amax = g.abs().amax(2)
    bad = ~torch.isfinite(amax)
    k = torch.full(amax.shape, -126.0, dtype=torch.float64)
    for c in range(-125, 123):
        k = torch.where(amax >= 2.0 ** (c + 6), float(c), k)
    q = torch.round(g / torch.exp2(k)[..., None]).clamp(-127, 127)
    q = torch.where(bad[..., None], 0.0, q)
    e = torch.where(bad, 255, (k + 127).long())
    return q.long().view(x.shape[0], -1)[:, :x.shape[1]], e


def held(q, e):
    """float64 values of (q [T, C], e [T, groups])."""
    step = torch.exp2(e.double() - 127)
    step = torch.where(e == 255, math.nan, step)
    return q.double() * step.repeat_interleave(32, 1)[:, :q.shape[1]]


def read(ck, C):
    q, e = ck
    return held(q[:, :C].long().cpu(), e[:, :-(-C // 32)].long().cpu())


def norm_forward(h, b, w_post, gate, w_pre, scale, eps):
    h, w_pre = h.double(), w_pre.double()
    out = {}
    if b is not None:
        b = b.double()
        r2 = 1 / torch.sqrt((b * b).mean(1) + eps)
        branch = b * r2[:, None] * w_post.double()
        if gate is not None:
            branch = branch * gate.double().repeat_interleave(h.shape[0] // gate.shape[0], 0)
        out["scale_h"] = (scale * h).abs() + branch.abs()
        h = scale * h + branch
        out.update(h=h, rstd_post=r2)
    r1 = 1 / torch.sqrt((h * h).mean(1) + eps)
    out.update(n=h * r1[:, None] * w_pre, rstd_pre=r1)
    return out


def norm_backward(dn, dh_in, h, b, w_post, gate, w_pre, scale, r2, r1):
    """Values, and for each the sum of the magnitudes it is made of (for error bounds)."""
    dn, h, r1 = dn.double(), h.double(), r1.double()[:, None]
    x, a = h * r1, dn * w_pre.double()
    m = (a * x).mean(1, keepdim=True)
    ma = (a * x).abs().mean(1, keepdim=True)
    D = r1 * (a - x * m)
    Da = r1 * (a.abs() + x.abs() * ma)
    if dh_in is not None:
        D, Da = D + dh_in.double(), Da + dh_in.double().abs()
    out = {"dh": scale * D, "dw_pre": (dn * x).sum(0)}
    mag = {"dh": abs(scale) * Da, "dw_pre": (dn * x).abs().sum(0)}
    if b is not None:
        r2, wp = r2.double()[:, None], w_post.double()
        y = b.double() * r2
        G = 1 if gate is None else gate.shape[0]
        gr = torch.ones(1, h.shape[1], dtype=torch.float64, device=h.device) if gate is None else gate.double()
        rows = gr.repeat_interleave(h.shape[0] // G, 0)
        S, Sa = (D * y).view(G, -1, h.shape[1]).sum(1), (Da * y.abs()).view(G, -1, h.shape[1]).sum(1)
        c, ca = D * rows * wp, Da * (rows * wp).abs()
        out["db"] = r2 * (c - y * (c * y).mean(1, keepdim=True))
        mag["db"] = r2 * (ca + y.abs() * (ca * y.abs()).mean(1, keepdim=True))
        out["dw_post"], mag["dw_post"] = (gr * S).sum(0), (gr.abs() * Sa).sum(0)
        if gate is not None:
            out["dgate"], mag["dgate"] = wp * S, wp.abs() * Sa
    return out, mag


def gated_forward(g, u):
    g, u = g.double(), u.double()
    return g * torch.sigmoid(g) * u


def gated_backward(dh, g, u):
    dh, g, u = dh.double(), g.double(), u.double()
    s = torch.sigmoid(g)
    return dh * u * s * (1 + g * (1 - s)), dh * g * s, g * s * u


def order(x, top):
    """Indices of the `top` largest of each row: value descending, ties by lowest index, NaN as -infinity."""
    x = x.double().cpu()
    x = torch.where(torch.isnan(x), -math.inf, x)
    return torch.sort(x, dim=1, descending=True, stable=True).indices[:, :top]


def logprob(x, y, top):
    x = x.double()
    T, V = x.shape
    m = x.amax(1, keepdim=True)
    z = torch.exp(x - m)
    lp = (x - m) - torch.log(z.sum(1, keepdim=True))
    p = torch.exp(lp)
    H = -torch.where(p == 0, 0.0, p * lp).sum(1)
    masked = (m <= -1e30)[:, 0]                        # false for NaN
    lp = torch.where(masked[:, None], -math.inf, lp)
    at = y.clamp(0, V - 1)[:, None]
    logp = lp.gather(1, at)[:, 0]
    logp = torch.where(y < 0, 0.0, torch.where(y >= V, math.nan, logp))
    ids = order(x, top).to(x.device)
    return {"logp": logp, "entropy": torch.where(masked, 0.0, H), "lse": torch.where(masked[:, None], torch.tensor([-math.inf, 0.0], dtype=torch.float64, device=x.device),
                               torch.cat([m, torch.log(z.sum(1, keepdim=True))], 1)), "top_ids": ids,
            "top_logp": lp.gather(1, ids), "p": torch.where(masked[:, None], 0.0, p), "lp": lp, "masked": masked}


def logprob_backward(f, y, dlogp, dH, ids, dtop):
    """From logprob()'s answer: the gradient, and the magnitudes the common term is made of."""
    p, lp, H = f["p"], f["lp"], f["entropy"][:, None]
    T, V = p.shape
    zero = torch.zeros(T, dtype=torch.float64, device=p.device)
    dl = zero if dlogp is None else torch.where(y < 0, 0.0, torch.where(y >= V, math.nan, dlogp.double()))
    dH = zero if dH is None else dH.double()
    G = dl.clone()
    own = torch.zeros_like(p)
    rows = torch.arange(T, device=p.device)
    inside = (y >= 0) & (y < V)
    own[rows[inside], y[inside]] += dl[inside]
    if dtop is not None:
        G = G + dtop.double().sum(1)
        own.scatter_add_(1, ids, dtop.double())
    inner = G[:, None] + dH[:, None] * (torch.where(p > 0, lp, 0.0) + H)
    dx = torch.where(p == 0, 0.0, -p * inner) + own
    mag = p * (G[:, None].abs() + dH[:, None].abs() * (torch.where(p > 0, lp.abs(), 0.0) + H)) + own.abs()
    return torch.where(f["masked"][:, None], 0.0, dx), mag
