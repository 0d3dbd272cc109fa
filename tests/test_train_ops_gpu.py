"""The operators of include/def_train.h on the GPU against plain 64-bit statements of them (tests/train_ref.py).

Error bounds: a stored value carries half a unit in the last place of its type; fp32 arithmetic adds, per term,
N 2^-24 of the sum of the magnitudes the value is made of, N the longest chain of roundings (a thread's elements of a
row plus the steps of a tree: at most 64; over tokens: the tokens of the sum).  The hardware exponential of the 16-bit
paths is good to 2^-21 (1 + |argument|)."""
import math

import pytest
import torch

import train_ref as R

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


def _gen(seed):
    g = torch.Generator(device=DEV)
    g.manual_seed(seed)
    return g


def _normal(shape, dtype, seed, std=1.0, mean=0.0):
    return torch.empty(shape, device=DEV).normal_(mean, std, generator=_gen(seed)).to(dtype)


def _laid(x, layout):
    """x with the rows of a layout: contiguous, in padded rows, or one element off any alignment."""
    T, C = x.shape
    if layout == "rows":
        return x.contiguous()
    pad = 16 - C % 8 if layout == "padded" else 3
    off = 0 if layout == "padded" else 1
    buf = torch.full((T * (C + pad) + 64,), float("nan"), dtype=x.dtype, device=DEV)
    v = buf[off:off + T * (C + pad)].view(T, C + pad)[:, :C]
    v.copy_(x)
    return v


def _out(T, C, dtype, layout="rows"):
    return _laid(torch.full((T, C), float("nan"), dtype=dtype, device=DEV), layout)


def _close(got, want, mag, dtype, n=64, extra=0.0):
    got, want, mag = got.double().cpu(), want.double().cpu(), mag.double().cpu()
    fine = torch.isfinite(want)
    assert torch.equal(fine, torch.isfinite(got)), "finite where it should not be, or the other way round"
    assert torch.equal(torch.isnan(want), torch.isnan(got))
    smallest = {F32: 0.0, BF16: 0.0, F16: 2.0 ** -25}[dtype]            # half of fp16's smallest step
    tol = R.UNIT[dtype] * want.abs() + (n * R.U32 + extra) * mag * (1 + R.UNIT[dtype]) + smallest + 1e-37
    over = ((got - want).abs() - tol)[fine]
    assert over.numel() == 0 or float(over.max()) <= 0, "off by %g beyond the bound" % float(over.max())


def _checkpoint(B, x):
    ck = B.def_checkpoint_alloc(x.shape[0], x.shape[1], DEV)
    B.def_checkpoint_pack(x, ck)
    return ck


# --- checkpoints -----------------------------------------------------------------------------------------------------

SHAPES = [(1, 1), (1, 31), (2, 32), (3, 33), (5, 64), (7, 97), (1, 2048), (129, 264), (64, 1000), (33, 1111), (2, 9000)]


@pytest.mark.parametrize("layout", ["rows", "padded", "off"])
@pytest.mark.parametrize("dtype", TYPES)
def test_pack_and_unpack_every_element(B, dtype, layout):
    for i, (T, C) in enumerate(SHAPES):
        x = _normal((T, C), F32, 100 + i)
        x = x * torch.exp2(torch.randint(-12, 5, (T, 1), device=DEV, generator=_gen(i)))      # groups of very different size
        x[0, 0] = 0.0
        x = _laid(x.to(dtype), layout)
        q, e = B.def_checkpoint_alloc(T, C, DEV)
        q.fill_(77)
        e.fill_(77)
        B.def_checkpoint_pack(x, (q, e))
        wq, we = R.pack(x)
        groups = -(-C // 32)
        assert torch.equal(q[:, :C].long().cpu(), wq) and torch.equal(e[:, :groups].long().cpu(), we)
        assert bool((q[:, C:] == 77).all()) and bool((e[:, groups:] == 77).all()), "padding was written"
        for to in TYPES:
            out = _out(T, C, to, layout)
            B.def_checkpoint_unpack((q, e), out)
            assert torch.equal(out.cpu(), R.held(wq, we).to(to)), (to, T, C)


def test_pack_of_specials(B):
    big, tiny = torch.finfo(F32).max, 2.0 ** -149
    rows = [[0.0, -0.0, 0.0], [math.nan, 1.0, 2.0], [math.inf, 1.0, 2.0], [-math.inf, 1.0, 0.0], [big, -big, 1.0], [tiny, -tiny, 0.0],
            [2.0 ** -120, 2.0 ** -121, 0.0], [127.4, 127.5, 127.6], [2.0, 127.0 / 64, 1.0], [0.5, 1.5 / 64, 2.5 / 64]]
    x = torch.tensor(rows, device=DEV)
    x = torch.nn.functional.pad(x, (0, 37))                                # a second, all-zero group
    ck = _checkpoint(B, x)
    wq, we = R.pack(x)
    assert torch.equal(ck[0][:, :40].long().cpu(), wq) and torch.equal(ck[1][:, :2].long().cpu(), we)
    out = torch.empty_like(x)
    B.def_checkpoint_unpack(ck, out)
    want = R.held(wq, we).float()
    assert torch.equal(torch.isnan(out.cpu()), torch.isnan(want)) and torch.equal(torch.nan_to_num(out.cpu()), torch.nan_to_num(want))
    assert bool(torch.isnan(out[1, :32]).all()) and bool((out[1, 32:] == 0).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,O,I", [(1, 1, 1), (1, 129, 70), (3, 8, 16), (64, 64, 64), (65, 128, 256), (100, 200, 300), (257, 136, 520),
                                   (1000, 72, 40), (2049, 264, 136), (777, 333, 555)])
def test_weight_grad(B, dtype, T, O, I):
    for layout in ("rows", "off", "padded"):
        dy = _laid(_normal((T, O), dtype, 1, std=0.1), layout)
        ck = _checkpoint(B, _normal((T, I), BF16, 2))
        work = torch.empty(max(1, B.def_checkpoint_weight_grad_workspace(dy, I)), dtype=torch.uint8, device=DEV)
        buf = torch.full((O * I + 3,), 7.0, device=DEV)
        dw = buf[1:1 + O * I].view(O, I)                                  # 4-byte aligned, as a slice of a gradient row is
        B.def_checkpoint_weight_grad(dy, ck, dw, work)
        x = R.read(ck, I)
        x = x.to(F16).double() if dtype == F16 else x
        want, mag = dy.double().cpu().t() @ x, dy.double().cpu().abs().t() @ x.abs()
        _close(dw, want, mag, F32, n=2 * (T + 16))
        first = dw.clone()
        B.def_checkpoint_weight_grad(dy, ck, dw, work)
        assert torch.equal(first, dw)
        B.def_checkpoint_weight_grad(dy, ck, dw, work, accumulate=True)
        _close(dw, 2 * want, 2 * mag, F32, n=2 * (T + 16))
        assert float(buf[0]) == 7.0 and bool((buf[1 + O * I:] == 7.0).all())


@pytest.mark.parametrize("dtype,T,O,I", [
    (BF16, 130, 4100, 1300),        # rounds of whole tiles and tiles that are cut; x^ widened once
    (F16, 130, 4100, 1300),
    (BF16, 1100, 2560, 2048),       # widened in shared memory, exponents by wide copies; more than one accumulator hand-over
    (F16, 200, 2500, 2100),         # the same with small copies of exponents
    (F32, 200, 1100, 2500),         # three pieces of dy
    (BF16, 40, 4608, 4224),         # one block of tokens: nothing to cut
    (F32, 70, 300, 2500),
    (BF16, 5000, 40, 8),
])
def test_weight_grad_many_tiles(B, dtype, T, O, I):
    dy = _normal((T, O), dtype, 1, std=0.1)
    ck = _checkpoint(B, _normal((T, I), BF16, 2))
    work = torch.empty(max(1, B.def_checkpoint_weight_grad_workspace(dy, I)), dtype=torch.uint8, device=DEV)
    assert work.numel() <= (68 << 20) + 8 * O * I + 6 * T * (O + 7)
    dw = torch.full((O, I), float("nan"), device=DEV)
    B.def_checkpoint_weight_grad(dy, ck, dw, work)
    x = R.read(ck, I).to(DEV)
    x = x.to(F16).double() if dtype == F16 else x
    want, mag = dy.double().t() @ x, dy.double().abs().t() @ x.abs()
    _close(dw, want, mag, F32, n=2 * (T + 16))
    first = dw.clone()
    B.def_checkpoint_weight_grad(dy, ck, dw, work, accumulate=True)
    _close(dw, 2 * want, 2 * mag, F32, n=2 * (T + 16))
    B.def_checkpoint_weight_grad(dy, ck, dw, work)
    assert torch.equal(first, dw)


def test_weight_grad_overlapping_calls(B):
    """Calls back to back on one stream and one workspace, without waiting, of shapes that use it differently."""
    shapes = [(300, 520, 264, BF16), (64, 136, 1000, F16), (700, 3400, 72, BF16), (129, 257, 333, F32)]
    runs = []
    for i, (T, O, I, dt) in enumerate(shapes):
        dy, ck = _normal((T, O), dt, 3 * i, std=0.1), _checkpoint(B, _normal((T, I), BF16, 3 * i + 1))
        runs.append((dy, ck, torch.empty(O, I, device=DEV)))
    work = torch.empty(max(B.def_checkpoint_weight_grad_workspace(dy, dw.shape[1]) for dy, _, dw in runs), dtype=torch.uint8, device=DEV)
    alone = []
    for dy, ck, dw in runs:
        B.def_checkpoint_weight_grad(dy, ck, dw, work)
        torch.cuda.synchronize()
        alone.append(dw.clone())
        dw.fill_(float("nan"))
    for _ in range(5):
        for dy, ck, dw in runs:
            B.def_checkpoint_weight_grad(dy, ck, dw, work)
    for (_, _, dw), want in zip(runs, alone):
        assert torch.equal(dw, want)


def test_weight_grad_no_tokens_and_nan(B):
    dw = torch.full((24, 40), 3.0, device=DEV)
    none = (torch.empty((0, 48), dtype=torch.int8, device=DEV), torch.empty((0, 4), dtype=torch.uint8, device=DEV))
    dy = torch.empty((0, 24), dtype=BF16, device=DEV)
    B.def_checkpoint_weight_grad(dy, none, dw, None, accumulate=True)
    assert bool((dw == 3).all())
    B.def_checkpoint_weight_grad(dy, none, dw, None)
    assert bool((dw == 0).all())
    x = _normal((70, 96), BF16, 5)
    x[3, 40] = math.nan                                                   # one group of one token
    dy = _normal((70, 24), BF16, 6)
    dw = torch.empty((24, 96), device=DEV)
    ck = _checkpoint(B, x)
    work = torch.empty(max(1, B.def_checkpoint_weight_grad_workspace(dy, 96)), dtype=torch.uint8, device=DEV)
    B.def_checkpoint_weight_grad(dy, ck, dw, work)
    assert bool(torch.isnan(dw[:, 32:64]).all()) and bool(torch.isfinite(dw[:, :32]).all()) and bool(torch.isfinite(dw[:, 64:]).all())


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["rows", "padded", "off", "halves"])
def test_gated(B, dtype, layout):
    fast = 2.0 ** -20 if dtype != F32 else 8 * R.U32                      # the exponential, twice
    for i, (T, F) in enumerate(SHAPES):
        if layout == "halves":
            both, dboth = _normal((T, 2 * F), dtype, 30 + i, std=2.0), _out(T, 2 * F, dtype)
            g, u, dg, du = both[:, :F], both[:, F:], dboth[:, :F], dboth[:, F:]
        else:
            g, u = (_laid(_normal((T, F), dtype, 30 + i + k, std=2.0), layout) for k in (0, 50))
            dg, du = _out(T, F, dtype, layout), _out(T, F, dtype, layout)
        g[0, 0] = -60000.0
        h = _out(T, F, dtype, layout if layout != "halves" else "rows")
        gck, uck, hck = (B.def_checkpoint_alloc(T, F, DEV) for _ in range(3))
        B.def_gated_forward(g, u, h, gck, uck)
        want = R.gated_forward(g, u)
        _close(h, want, want.abs() * (1 + g.double().abs().clamp(max=100)), dtype, n=8, extra=fast)
        for x, ck in ((g, gck), (u, uck)):
            wq, we = R.pack(x)
            assert torch.equal(ck[0][:, :F].long().cpu(), wq) and torch.equal(ck[1][:, :-(-F // 32)].long().cpu(), we)
        dh = _normal((T, F), dtype, 90 + i, std=0.1)
        back = _out(T, F, dtype)
        B.def_gated_backward(dh, gck, uck, dg, du, h_out=back, h_ck=hck)
        gh, uh, d = R.read(gck, F), R.read(uck, F), dh.double().cpu()
        wg, wu, wh = R.gated_backward(d, gh, uh)
        far = 1 + gh.abs().clamp(max=100)
        _close(dg, wg, (d * uh).abs() * far * far * torch.sigmoid(gh), dtype, n=16, extra=2 * fast)
        _close(du, wu, wu.abs() * far, dtype, n=8, extra=fast)
        _close(back, wh, wh.abs() * far, dtype, n=8, extra=fast)
        wq, we = R.pack(back)
        assert torch.equal(hck[0][:, :F].long().cpu(), wq) and torch.equal(hck[1][:, :-(-F // 32)].long().cpu(), we)
        only = (torch.empty_like(dg), torch.empty_like(du))
        B.def_gated_backward(dh, gck, uck, *only)                          # without the recomputed product
        assert torch.equal(only[0], dg) and torch.equal(only[1], du)
        bare = torch.empty_like(h)
        B.def_gated_forward(g, u, bare)
        assert torch.equal(bare, h)


# --- norms -----------------------------------------------------------------------------------------------------------

NORM_SHAPES = [(1, 1), (1, 8), (3, 33), (4, 64), (6, 256), (5, 257), (2, 1024), (30, 1000), (12, 1111), (3, 2048), (2, 4096), (4, 4100),
               (2, 8192), (2, 8200), (1, 16384), (1, 16383), (700, 40), (1203, 96)]


def _norm_inputs(T, C, dtype, layout, groups, seed):
    h, b = (_laid(_normal((T, C), dtype, seed + k, std=s), layout) for k, s in ((0, 1.0), (1, 3.0)))
    w_post, w_pre = (_normal((C,), F32, seed + k, 0.3, 1.0) for k in (2, 3))
    gate = None if groups == 0 else _normal((groups, C), F32, seed + 4, 0.5, 0.3)
    return h, b, w_post, gate, w_pre


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["rows", "padded", "off"])
def test_norm_forward(B, dtype, layout):
    for i, (T, C) in enumerate(NORM_SHAPES):
        for groups in {0, 1, T if T < 8 else 3 if T % 3 == 0 else 2}:
            h, b, w_post, gate, w_pre = _norm_inputs(T, C, dtype, layout, groups, 10 * i)
            h_out, n_out = _out(T, C, dtype, layout), _out(T, C, dtype, layout)
            r2, r1 = torch.empty(T, device=DEV), torch.empty(T, device=DEV)
            cks = [B.def_checkpoint_alloc(T, C, DEV) for _ in range(3)]
            B.def_norm_forward(h, b, w_post, gate, w_pre, h_out, n_out, r2, r1, res_scale=0.75, eps=1e-5, b_ck=cks[0], h_ck=cks[1], n_ck=cks[2])
            f = R.norm_forward(h, b, w_post, gate, w_pre, 0.75, 1e-5)
            _close(r2, f["rstd_post"], f["rstd_post"], F32)
            _close(h_out, f["h"], f["scale_h"], dtype)
            # n: the error of h' and that of the row's norm, relative to the row
            row = (f["scale_h"] ** 2).mean(1).sqrt() * f["rstd_pre"]
            _close(r1, f["rstd_pre"], f["rstd_pre"] * row, F32, n=128)
            _close(n_out, f["n"], (f["scale_h"] * f["rstd_pre"][:, None] + f["n"].abs() / w_pre.double().abs() * row[:, None]) * w_pre.double().abs(), dtype, n=128)
            for x, ck in ((b, cks[0]), (h_out, cks[1]), (n_out, cks[2])):
                wq, we = R.pack(x)
                assert torch.equal(ck[0][:, :C].long().cpu(), wq) and torch.equal(ck[1][:, :-(-C // 32)].long().cpu(), we)
            # in place, without checkpoints: the same bits
            n2, s2, s1 = torch.empty_like(n_out), torch.empty_like(r2), torch.empty_like(r1)
            B.def_norm_forward(h, b, w_post, gate, w_pre, h, n2, s2, s1, res_scale=0.75, eps=1e-5)
            assert torch.equal(h, h_out) and torch.equal(n2, n_out) and torch.equal(s2, r2) and torch.equal(s1, r1)
        # no block yet
        h = _laid(_normal((T, C), dtype, 5 + i), layout)
        n_out, r1, ck = _out(T, C, dtype, layout), torch.empty(T, device=DEV), B.def_checkpoint_alloc(T, C, DEV)
        B.def_norm_forward(h, None, None, None, w_pre, None, n_out, None, r1, n_ck=ck)
        f = R.norm_forward(h, None, None, None, w_pre, 1.0, 1e-6)
        _close(n_out, f["n"], f["n"].abs(), dtype)
        _close(r1, f["rstd_pre"], f["rstd_pre"], F32)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("saves", ["values", "checkpoints", "mixed"])
def test_norm_backward(B, dtype, saves):
    for i, (T, C) in enumerate(NORM_SHAPES):
        layout = ("rows", "padded", "off")[i % 3]
        groups = (0, 1, T if T < 8 else 3 if T % 3 == 0 else 2)[(i + TYPES.index(dtype)) % 3]
        h, b, w_post, gate, w_pre = _norm_inputs(T, C, dtype, layout, groups, 400 + 10 * i)
        dn, dh_in = (_laid(_normal((T, C), dtype, 500 + 10 * i + k, std=0.1), layout) for k in (0, 1))
        r2, r1 = (torch.rsqrt(v.float().square().mean(1) + 1e-5) for v in (b, h))
        hs, bs, hv, bv = h, b, h, b
        if saves != "values":
            hs = _checkpoint(B, h)
            hv = R.read(hs, C).to(DEV)
        if saves == "checkpoints":
            bs = _checkpoint(B, b)
            bv = R.read(bs, C).to(DEV)
        dh, db = _out(T, C, dtype, layout), _out(T, C, dtype, layout)
        dwp, dw = torch.full((C,), 9.0, device=DEV), torch.full((C,), 9.0, device=DEV)
        dg = None if gate is None else torch.full((groups, C), 9.0, device=DEV)
        work = torch.empty(B.def_norm_backward_workspace(T, C, max(1, groups)), dtype=torch.uint8, device=DEV)
        args = (dn, dh_in, hs, bs, w_post, gate, w_pre, r2, r1, dh, db, dwp, dg, dw, work)
        B.def_norm_backward(*args, res_scale=0.75)
        want, mag = R.norm_backward(dn, dh_in, hv, bv, w_post, gate, w_pre, 0.75, r2, r1)
        _close(dh, want["dh"], mag["dh"], dtype, n=128)
        _close(db, want["db"], mag["db"], dtype, n=256)
        names = (("dw_pre", dw), ("dw_post", dwp)) + ((("dgate", dg),) if dg is not None else ())
        for name, got in names:
            _close(got, want[name], mag[name], F32, n=T + 128)
        once = [g.clone() for _, g in names] + [dh.clone(), db.clone()]
        B.def_norm_backward(*args, res_scale=0.75)
        assert all(torch.equal(x, y) for x, y in zip(once, [g for _, g in names] + [dh, db])), "two calls differ"
        B.def_norm_backward(*args, res_scale=0.75, accumulate=True)
        for name, got in names:
            _close(got, 2 * want[name], 2 * mag[name], F32, n=T + 128)
        # dh written over dh_in
        B.def_norm_backward(dn, dh_in, hs, bs, w_post, gate, w_pre, r2, r1, dh_in, db, dwp, dg, dw, work, res_scale=0.75)
        assert torch.equal(dh_in, dh)
        # no block, no incoming gradient
        work = torch.empty(B.def_norm_backward_workspace(T, C), dtype=torch.uint8, device=DEV)
        B.def_norm_backward(dn, None, hs, None, None, None, w_pre, None, r1, dh, None, None, None, dw, work)
        want, mag = R.norm_backward(dn, None, hv, None, None, None, w_pre, 1.0, None, r1)
        _close(dh, want["dh"], mag["dh"], dtype, n=128)
        _close(dw, want["dw_pre"], mag["dw_pre"], F32, n=T + 128)


MANY_ROWS = [(2700, 64, 1), (2701, 200, 0), (2672, 1024, 8), (1800, 1032, 3), (1776, 2048, 1), (900, 2056, 4), (889, 4096, 0), (450, 4104, 5),
             (444, 8192, 2), (450, 8200, 1), (446, 12288, 2)]
MANY_ODD = [(3000, 1, 2, "rows"), (2701, 3, 1, "off"), (2672, 33, 8, "rows"), (2700, 257, 0, "off"), (1800, 1111, 3, "rows"), (1777, 2047, 1, "rows"),
            (1790, 1284, 2, "off"), (900, 2052, 4, "rows"), (889, 4095, 1, "off"), (450, 4097, 5, "rows"), (448, 8191, 2, "rows"), (450, 8201, 0, "rows")]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("T,C,groups,layout", [m + ("rows",) for m in MANY_ROWS] + MANY_ODD)
def test_norm_many_rows(B, dtype, T, C, groups, layout):
    """Enough rows that each CTA walks several of them; rows that are not a whole number of accesses per thread."""
    h, b, w_post, gate, w_pre = _norm_inputs(T, C, dtype, layout, groups, T)
    n_out, h_out, r2, r1 = _out(T, C, dtype, layout), _out(T, C, dtype, layout), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
    cks = [B.def_checkpoint_alloc(T, C, DEV) for _ in range(3)]
    B.def_norm_forward(h, b, w_post, gate, w_pre, h_out, n_out, r2, r1, res_scale=0.75, eps=1e-5, b_ck=cks[0], h_ck=cks[1], n_ck=cks[2])
    f = R.norm_forward(h, b, w_post, gate, w_pre, 0.75, 1e-5)
    row = (f["scale_h"] ** 2).mean(1).sqrt() * f["rstd_pre"]
    _close(r2, f["rstd_post"], f["rstd_post"], F32)
    _close(r1, f["rstd_pre"], f["rstd_pre"] * row, F32, n=128)
    _close(h_out, f["h"], f["scale_h"], dtype)
    _close(n_out, f["n"], (f["scale_h"] * f["rstd_pre"][:, None] + f["n"].abs() / w_pre.double().abs() * row[:, None]) * w_pre.double().abs(), dtype, n=128)
    for x, ck in ((b, cks[0]), (h_out, cks[1]), (n_out, cks[2])):
        mine = _checkpoint(B, x)
        assert torch.equal(mine[0][:, :C], ck[0][:, :C]) and torch.equal(mine[1][:, :-(-C // 32)], ck[1][:, :-(-C // 32)])
    alone, s1 = _out(T, C, dtype, layout), torch.empty(T, device=DEV)
    B.def_norm_forward(b, None, None, None, w_pre, None, alone, None, s1)
    g = R.norm_forward(b, None, None, None, w_pre, 1.0, 1e-6)
    _close(alone, g["n"], g["n"].abs(), dtype)
    dn, dh_in = (_laid(_normal((T, C), dtype, T + k, std=0.1), layout) for k in (7, 8))
    hs, bs = _checkpoint(B, h), _checkpoint(B, b)
    hv, bv = R.read(hs, C).to(DEV), R.read(bs, C).to(DEV)
    r2, r1 = (torch.rsqrt(v.float().square().mean(1) + 1e-5) for v in (b, h))
    dh, db, dwp, dw = _out(T, C, dtype, layout), _out(T, C, dtype, layout), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
    dg = None if gate is None else torch.empty(groups, C, device=DEV)
    work = torch.empty(B.def_norm_backward_workspace(T, C, max(1, groups)), dtype=torch.uint8, device=DEV)
    for hx, bx, hy, by, into in ((h, b, h, b, dh_in), (hs, bs, hv, bv, None), (h, bs, h, bv, dh_in), (hs, b, hv, b, dh_in)):
        B.def_norm_backward(dn, into, hx, bx, w_post, gate, w_pre, r2, r1, dh, db, dwp, dg, dw, work, res_scale=0.75)
        want, mag = R.norm_backward(dn, into, hy, by, w_post, gate, w_pre, 0.75, r2, r1)
        _close(dh, want["dh"], mag["dh"], dtype, n=128)
        _close(db, want["db"], mag["db"], dtype, n=256)
        for name, got in (("dw_pre", dw), ("dw_post", dwp)) + ((("dgate", dg),) if dg is not None else ()):
            _close(got, want[name], mag[name], F32, n=T + 128)
    B.def_norm_backward(dn, None, hs, None, None, None, w_pre, None, r1, dh, None, None, None, dw, work)
    want, mag = R.norm_backward(dn, None, hv, None, None, None, w_pre, 1.0, None, r1)
    _close(dh, want["dh"], mag["dh"], dtype, n=128)
    _close(dw, want["dw_pre"], mag["dw_pre"], F32, n=T + 128)
    if layout == "off":                                                       # nothing beside the rows is written
        for out in (h_out, n_out, dh, db):
            whole = torch.as_strided(out, (T * out.stride(0) + 1,), (1,), out.storage_offset() - 1)
            gap = torch.cat([whole[:1], whole[1:1 + (T - 1) * out.stride(0)].view(T - 1, -1)[:, C:].reshape(-1), whole[1 + (T - 1) * out.stride(0) + C:]])
            assert bool(torch.isnan(gap).all())
    inplace_h, inplace_n = _laid(h, layout), _out(T, C, dtype, layout)
    B.def_norm_forward(inplace_h, b, w_post, gate, w_pre, inplace_h, inplace_n, r2.clone(), s1, res_scale=0.75, eps=1e-5)
    assert torch.equal(inplace_h, h_out) and torch.equal(inplace_n, n_out)
    first = (dh.clone(), dw.clone())
    B.def_norm_backward(dn, None, hs, None, None, None, w_pre, None, r1, dh, None, None, None, dw, work)
    assert torch.equal(first[0], dh) and torch.equal(first[1], dw)


def test_norm_many_groups_and_no_rows(B):
    T, C = 600, 72
    for groups in (600, 200, 40):
        h, b, w_post, gate, w_pre = _norm_inputs(T, C, BF16, "rows", groups, 3)
        dn = _normal((T, C), BF16, 8, std=0.1)
        r2, r1 = (torch.rsqrt(v.float().square().mean(1) + 1e-5) for v in (b, h))
        dh, db, dw, dwp, dg = _out(T, C, BF16), _out(T, C, BF16), _out(1, C, F32)[0], _out(1, C, F32)[0], _out(groups, C, F32)
        work = torch.empty(B.def_norm_backward_workspace(T, C, groups), dtype=torch.uint8, device=DEV)
        B.def_norm_backward(dn, None, h, b, w_post, gate, w_pre, r2, r1, dh, db, dwp, dg, dw, work)
        want, mag = R.norm_backward(dn, None, h, b, w_post, gate, w_pre, 1.0, r2, r1)
        for name, got in (("dw_pre", dw), ("dw_post", dwp), ("dgate", dg)):
            _close(got, want[name], mag[name], F32, n=T + 128)
    e = torch.empty((0, C), dtype=BF16, device=DEV)
    s = torch.empty(0, device=DEV)
    B.def_norm_forward(e, e, w_post, None, w_pre, e, e, s, s)
    B.def_norm_backward(e, None, e, e, w_post, None, w_pre, s, s, e, e, dwp, None, dw, None)
    assert bool((dw == 0).all()) and bool((dwp == 0).all())


# --- log probabilities -------------------------------------------------------------------------------------------------

LOGIT_SHAPES = [(1, 1, 1), (2, 2, 2), (3, 7, 5), (5, 32, 32), (4, 100, 8), (7, 1000, 20), (3, 4096, 32), (2, 4097, 1), (9, 5003, 0), (1, 50001, 20),
                (2, 65536, 32), (1, 200000, 32), (300, 264, 4)]


def _logit_inputs(T, V, dtype, seed, layout="rows"):
    x = _normal((T, V), F32, seed, std=3.0)
    y = torch.randint(0, V, (T,), device=DEV, generator=_gen(seed + 1))
    x[torch.arange(T, device=DEV), y] += 5.0
    return _laid(x.to(dtype), layout), y


def _run_logprob(B, x, y, top, stream=None):
    T = x.shape[0]
    o = {"logp": torch.full((T,), 9.0, device=DEV), "entropy": torch.full((T,), 9.0, device=DEV), "lse": torch.full((T, 2), 9.0, device=DEV)}
    ids, lp = (torch.full((T, top), -9, dtype=torch.int64, device=DEV), torch.full((T, top), 9.0, device=DEV)) if top else (None, None)
    B.def_logprob_forward(x, y, o["logp"], o["entropy"], o["lse"], ids, lp, stream=stream)
    return dict(o, top_ids=ids, top_logp=lp)


def _check_logprob(x, y, top, o):
    f = R.logprob(x, y, top)
    V = x.shape[1]
    # a term's exponent is off by 2 |x - m| 2^-24, its exponential by 2^-22; a thread adds V / 512 of them
    n = V / 128 + 64
    one = torch.ones_like(f["entropy"])
    poisoned = torch.isnan(f["lse"][:, 1])                       # the maximum of a row with a NaN is not specified
    assert torch.equal(o["lse"][~poisoned, 0].double(), f["lse"][~poisoned, 0]), "the maximum is exact"
    _close(o["lse"][:, 1], f["lse"][:, 1], one + f["lse"][:, 1].nan_to_num(0).abs(), F32, n=n)
    _close(o["entropy"], f["entropy"], one * 2 * (1 + f["entropy"].nan_to_num(0)), F32, n=2 * n)
    _close(o["logp"], f["logp"], one + f["logp"].nan_to_num(0, 0, 0).abs(), F32, n=n)
    if top:
        assert torch.equal(o["top_ids"].cpu(), f["top_ids"].cpu())
        _close(o["top_logp"], f["top_logp"], 1 + f["top_logp"].nan_to_num(0, 0, 0).abs(), F32, n=n)
    return f


def _check_gradient(B, x, y, top, o, f, dtype, seed=0, in_place=False, parts="all"):
    T, V = x.shape
    dl = _normal((T,), F32, seed + 50, 1.0) if parts in ("all", "logp") else None
    dH = _normal((T,), F32, seed + 51, 0.3) if parts in ("all", "entropy") else None
    dt = _normal((T, top), F32, seed + 52, 0.5) if top and parts in ("all", "top") else None
    want, mag = R.logprob_backward(f, y, dl, dH, f["top_ids"], dt)
    dx = x if in_place else _laid(torch.full_like(x, 9.0), "rows" if x.is_contiguous() else "off")
    B.def_logprob_backward(x, y, o["lse"], o["entropy"], dx, dl, dH, o["top_ids"], dt)
    # p from x - lse: off by |x - lse| 2^-23 and by what lse and the entropy are off
    off = (f["lp"].nan_to_num(0, 0, 0).abs() + f["lse"].nan_to_num(0, 0, 0).sum(1).abs()[:, None]).clamp(max=200)
    _close(dx, want, mag * (1 + off), dtype, n=V / 64 + 128 + 33)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("layout", ["rows", "padded", "off"])
def test_logprob(B, dtype, layout):
    for i, (T, V, top) in enumerate(LOGIT_SHAPES):
        x, y = _logit_inputs(T, V, dtype, 20 * i, layout)
        if T > 2:
            y[1] = -100
        o = _run_logprob(B, x, y, top)
        f = _check_logprob(x, y, top, o)
        for parts in ("all", "logp", "entropy", "top"):
            _check_gradient(B, x, y, top, o, f, dtype, i, parts=parts)
        _check_gradient(B, x, y, top, o, f, dtype, i, in_place=True)


@pytest.mark.parametrize("dtype", TYPES)
def test_logprob_gradient_with_other_alignment(B, dtype):
    """Logits and their gradient that do not start alike within 16 bytes."""
    for T, V in ((5, 777), (3, 30011)):
        x, y = _logit_inputs(T, V, dtype, 3)
        o = _run_logprob(B, x, y, 8)
        f = _check_logprob(x, y, 8, o)
        dl = _normal((T,), F32, 9)
        want, mag = R.logprob_backward(f, y, dl, None, f["top_ids"], None)
        dx = _out(T, V, dtype, "off")
        B.def_logprob_backward(x, y, o["lse"], o["entropy"], dx, dl)
        off = (f["lp"].nan_to_num(0, 0, 0).abs() + f["lse"].sum(1).abs()[:, None]).clamp(max=200)
        _close(dx, want, mag * (1 + off), dtype, n=V / 64 + 128 + 33)


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("V", [40, 264, 4099, 33000])
def test_logprob_masks_ties_and_specials(B, dtype, V):
    low = torch.finfo(dtype).min
    T, top = 16, min(V, 32)
    x = _normal((T, V), dtype, V, std=2.0)
    y = torch.arange(T, device=DEV) * 2
    x[0] = -math.inf                                        # nothing left
    x[1, 1:] = -math.inf                                    # one token left; the target is masked
    x[2] = low if dtype != F16 else -math.inf               # nothing left, by the lowest value
    x[3, 5:] = low                                          # five left
    x[4] = 1.25                                             # all equal
    x[5] = 0.0
    x[5, ::2] = -0.0                                        # zeros of both signs tie
    x[6, 3] = math.nan
    x[7, 7] = math.inf
    x[8] = torch.arange(V, device=DEV).to(dtype).flip(0) * 0.01   # descending: many of the best in few lists
    x[9, V // 2:] = -math.inf
    x[10] = -math.inf
    x[10, V - 1] = -3.0                                     # the last one only
    x[11] = math.nan
    x[12] = x[12].float().round().to(dtype)                 # few values, many ties
    x[13] = -40.0
    x[13, ::max(1, V // 200)] = 8.0                         # many equal maxima, far apart
    y[9], y[14], y[15] = V - 1, -1, V
    o = _run_logprob(B, x, y, top)
    f = _check_logprob(x, y, top, o)
    _check_gradient(B, x, y, top, o, f, dtype)
    again = _run_logprob(B, x, y, top)
    for k in o:
        assert torch.equal(o[k].nan_to_num(0), again[k].nan_to_num(0))
    assert float(o["entropy"][0]) == 0 and float(o["lse"][0, 0]) == -math.inf and float(o["logp"][14]) == 0


def test_logprob_best_in_one_list(B):
    """All large logits in places that one thread, or few, read: every element of a list is among the best."""
    for V in (8 * 512 * 40, 512 * 40 + 1):
        for stride in (4096, 2048, 512, 8):
            x = _normal((2, V), F32, 1)
            x[:, 3::stride] += 50
            y = torch.zeros(2, dtype=torch.int64, device=DEV)
            _check_logprob(x, y, 32, _run_logprob(B, x, y, 32))


def test_differences(B):
    """Gradients against central differences of the forward calls themselves, along random directions.  fp32: with
    step 1e-2 the difference is off by (1e-2)^2 of the third derivative (inputs and slopes are of order one) and by
    2^-24 |L| / 1e-2: 2e-3 of the slope's scale covers both."""
    T, C, eps = 6, 40, 1e-2

    def slope(f, at, d):
        return (f(at + eps * d) - f(at - eps * d)) / (2 * eps)

    # norm
    h, b, w_post, gate, w_pre = _norm_inputs(T, C, F32, "rows", 2, 77)
    cn, ch = _normal((T, C), F32, 1), _normal((T, C), F32, 2)

    def loss(h=h, b=b, w_post=w_post, gate=gate, w_pre=w_pre):
        ho, n, r2, r1 = torch.empty_like(h), torch.empty_like(h), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        B.def_norm_forward(h, b, w_post, gate, w_pre, ho, n, r2, r1, res_scale=0.75)
        return float((n.double() * cn.double()).sum() + (ho.double() * ch.double()).sum()), ho, r2, r1

    _, ho, r2, r1 = loss()
    g = {"h": torch.empty_like(h), "b": torch.empty_like(h), "w_post": torch.empty(C, device=DEV), "gate": torch.empty(2, C, device=DEV), "w_pre": torch.empty(C, device=DEV)}
    work = torch.empty(B.def_norm_backward_workspace(T, C, 2), dtype=torch.uint8, device=DEV)
    B.def_norm_backward(cn, ch, ho, b, w_post, gate, w_pre, r2, r1, g["h"], g["b"], g["w_post"], g["gate"], g["w_pre"], work, res_scale=0.75)
    for name, at in (("h", h), ("b", b), ("w_post", w_post), ("gate", gate), ("w_pre", w_pre)):
        d = _normal(at.shape, F32, 9)
        got = float((g[name].double() * d.double()).sum())
        want = slope(lambda v: loss(**{name: v})[0], at, d)
        scale = float((g[name].double() * d.double()).abs().sum())
        assert abs(got - want) <= 2e-3 * scale, (name, got, want)

    # log probabilities
    x, y = _logit_inputs(T, C, F32, 5)
    x = x / 3
    cl, cH = _normal((T,), F32, 3), _normal((T,), F32, 4)
    o = _run_logprob(B, x, y, 0)
    dx = torch.empty_like(x)
    B.def_logprob_backward(x, y, o["lse"], o["entropy"], dx, cl, cH)
    d = _normal(x.shape, F32, 11)

    def total(v):
        o = _run_logprob(B, v, y, 0)
        return float((o["logp"].double() * cl.double()).sum() + (o["entropy"].double() * cH.double()).sum())

    assert abs(float((dx.double() * d.double()).sum()) - slope(total, x, d)) <= 2e-3 * float((dx * d).abs().sum())

    # gated: the checkpoint's values are where the slope is taken, so they are the inputs
    ck = [_checkpoint(B, _normal((T, C), F32, 20 + k)) for k in (0, 1)]
    gh, uh = torch.empty((T, C), device=DEV), torch.empty((T, C), device=DEV)
    B.def_checkpoint_unpack(ck[0], gh)
    B.def_checkpoint_unpack(ck[1], uh)
    dg, du = torch.empty_like(gh), torch.empty_like(gh)
    B.def_gated_backward(cn, ck[0], ck[1], dg, du)
    for grad, f in ((dg, lambda v: (v, uh)), (du, lambda v: (gh, v))):
        def out(v):
            h = torch.empty_like(gh)
            B.def_gated_forward(*f(v), h)
            return float((h.double() * cn.double()).sum())
        at = gh if grad is dg else uh
        d = _normal(at.shape, F32, 31)
        assert abs(float((grad.double() * d.double()).sum()) - slope(out, at, d)) <= 2e-3 * float((grad * d).abs().sum())


# --- streams, long offsets -----------------------------------------------------------------------------------------------

def test_side_stream(B):
    side = torch.cuda.Stream()
    x, y = _logit_inputs(64, 3000, BF16, 1)
    want = _run_logprob(B, x, y, 8)
    h, b, w_post, gate, w_pre = _norm_inputs(64, 512, BF16, "rows", 1, 2)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(2_000_000)
        x2 = (x.float() * 1.0).to(BF16)                       # made on the side stream, after the sleep
        got = _run_logprob(B, x2, y, 8, stream=side)
        ck = B.def_checkpoint_alloc(64, 3000, DEV)
        B.def_checkpoint_pack(x2, ck, stream=side)
        back = torch.empty_like(x2)
        B.def_checkpoint_unpack(ck, back, stream=side)
        h2 = h * 1.0
        ho, n, r2, r1 = torch.empty_like(h), torch.empty_like(h), torch.empty(64, device=DEV), torch.empty(64, device=DEV)
        B.def_norm_forward(h2, b, w_post, gate, w_pre, ho, n, r2, r1, stream=side)
    side.synchronize()
    for k in want:
        assert torch.equal(want[k], got[k])
    wq, we = R.pack(x)
    assert torch.equal(back.cpu(), R.held(wq, we).to(BF16))
    f = R.norm_forward(h, b, w_post, gate, w_pre, 1.0, 1e-6)
    _close(ho, f["h"], f["scale_h"], BF16)


def test_offsets_past_32_bits(B):
    """Rows more than 2^31 elements apart, and a gradient row beyond 2^32 bytes."""
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free device memory")
    C, ld = 520, (1 << 31) + 8
    buf = torch.zeros(2 * ld + C, dtype=BF16, device=DEV)
    x = torch.as_strided(buf, (3, C), (ld, 1))
    x.copy_(_normal((3, C), BF16, 1))
    small = x.contiguous()
    out = torch.as_strided(torch.zeros(2 * ld + C, dtype=BF16, device=DEV), (3, C), (ld, 1))
    ck = _checkpoint(B, x)
    B.def_checkpoint_unpack(ck, out)
    assert torch.equal(out.contiguous().cpu(), R.read(ck, C).to(BF16))
    wq, we = R.pack(small)
    assert torch.equal(ck[0][:, :C].long().cpu(), wq)
    y = torch.tensor([1, 2, 3], device=DEV)
    f = _check_logprob(small, y, 8, _run_logprob(B, x, y, 8))
    B.def_logprob_backward(x, y, f["lse"].float(), f["entropy"].float(), out, torch.ones(3, device=DEV))
    dense = torch.empty_like(small)
    B.def_logprob_backward(small, y, f["lse"].float(), f["entropy"].float(), dense, torch.ones(3, device=DEV))
    assert torch.equal(out.contiguous(), dense)
    w = torch.ones(C, device=DEV)
    r1, r2, n, ho = torch.empty(3, device=DEV), torch.empty(3, device=DEV), torch.empty_like(small), torch.empty_like(small)
    B.def_norm_forward(x, x, w, None, w, out, n, r2, r1)
    B.def_norm_forward(small, small.clone(), w, None, w, ho, n, r2, r1)
    assert torch.equal(out.contiguous(), ho)
