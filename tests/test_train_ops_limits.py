"""Limits that include/def_train.h promises: the least aligned checkpoints, the largest magnitudes, calls from several
host threads, the longest runs of rows and of tokens.  Bounds as in test_train_ops_gpu.py."""
import ctypes
import threading
import time

import pytest
import torch

import train_ref as R
from test_train_ops_gpu import (B, BF16, DEV, F16, F32, _check_gradient, _check_logprob, _checkpoint, _close, _norm_inputs, _normal,  # noqa: F401
                                _out, _run_logprob)


def _moved(ck, off):
    """The same checkpoint with its exponents `off` bytes into a buffer of their own."""
    q, e = ck
    buf = torch.full((e.numel() + off + 64,), 77, dtype=torch.uint8, device=DEV)
    moved = buf[off:off + e.numel()].view(e.shape)
    moved.copy_(e)
    assert moved.data_ptr() % 16 == off % 16
    return q, moved


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F32])
@pytest.mark.parametrize("T,C", [(900, 512), (1000, 1000), (450, 4096), (6, 512)])
@pytest.mark.parametrize("off_h,off_b", [(4, 0), (0, 8), (12, 4)])
def test_exponents_at_any_multiple_of_4(B, dtype, T, C, off_h, off_b):  # noqa: F811
    """Rows of exponents that are whole 16-byte words, from a base that is not on a 16-byte boundary."""
    assert B.def_checkpoint_layout(C)[1] % 16 == 0
    h, b, w_post, gate, w_pre = _norm_inputs(T, C, dtype, "rows", 2, 61)
    dn, dh_in = (_normal((T, C), dtype, 63 + k, std=0.1) for k in (0, 1))
    r2, r1 = (torch.rsqrt(v.float().square().mean(1) + 1e-5) for v in (b, h))
    hs, bs = _checkpoint(B, h), _checkpoint(B, b)
    hv, bv = R.read(hs, C).to(DEV), R.read(bs, C).to(DEV)
    hs, bs = _moved(hs, off_h), _moved(bs, off_b)
    dh, db = _out(T, C, dtype), _out(T, C, dtype)
    dwp, dg, dw = torch.empty(C, device=DEV), torch.empty(2, C, device=DEV), torch.empty(C, device=DEV)
    work = torch.empty(B.def_norm_backward_workspace(T, C, 2), dtype=torch.uint8, device=DEV)
    B.def_norm_backward(dn, dh_in, hs, bs, w_post, gate, w_pre, r2, r1, dh, db, dwp, dg, dw, work, res_scale=0.75)
    want, mag = R.norm_backward(dn, dh_in, hv, bv, w_post, gate, w_pre, 0.75, r2, r1)
    _close(dh, want["dh"], mag["dh"], dtype, n=128)
    _close(db, want["db"], mag["db"], dtype, n=256)
    for name, got in (("dw_pre", dw), ("dw_post", dwp), ("dgate", dg)):
        _close(got, want[name], mag[name], F32, n=T + 128)
    B.def_norm_backward(dn, None, hs, None, None, None, w_pre, None, r1, dh, None, None, None, dw, work)
    want, mag = R.norm_backward(dn, None, hv, None, None, None, w_pre, 1.0, None, r1)
    _close(dh, want["dh"], mag["dh"], dtype, n=128)
    _close(dw, want["dw_pre"], mag["dw_pre"], F32, n=T + 128)
    # the other calls that read or write exponents
    out, same = _out(T, C, dtype), _moved((hs[0], torch.zeros_like(hs[1])), off_h)
    B.def_checkpoint_unpack(hs, out)
    assert torch.equal(out.double(), hv.to(dtype).double())
    B.def_checkpoint_pack(h, same)
    assert torch.equal(same[1][:, :C // 32], hs[1][:, :C // 32])
    grad = torch.empty((40, C), device=DEV)
    dy = _normal((T, 40), dtype, 70, std=0.1)
    work = torch.empty(max(1, B.def_checkpoint_weight_grad_workspace(dy, C)), dtype=torch.uint8, device=DEV)
    B.def_checkpoint_weight_grad(dy, hs, grad, work)
    _close(grad, dy.double().t() @ hv, dy.double().abs().t() @ hv.abs(), F32, n=2 * (T + 16))


FILLS = [-1e9, -1e10, -1e12, -1e15, -1e20, -7e29, -8e29, -9e29]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [F32, BF16])
@pytest.mark.parametrize("V", [40, 264, 4099, 33000])
@pytest.mark.parametrize("target", ["given", "ignored"])
def test_logits_of_any_size(B, dtype, V, target):  # noqa: F811
    """Rows filled, or partly filled, with finite masks; maxima far from 0; differences that count beside a large maximum."""
    few = torch.randperm(V, generator=torch.Generator().manual_seed(V))[:5].to(DEV)
    step = {F32: 2.0 ** -24, BF16: 2.0 ** -8}[dtype]
    rows = []

    def row(fill=None, where=slice(None)):
        r = _normal((V,), F32, V + len(rows), std=2.0)
        if fill is not None:
            r[where] = fill
        rows.append(r)
        return r

    for f in FILLS:
        row(f)                                                          # nothing else
        row(f, slice(0, V // 2))                                        # what the first threads read
        row(f, slice(V - V // 2, V))
        row(f, slice(0, V, 2))
        keep = row()
        rows[-1] = torch.full_like(keep, f).index_copy(0, few, keep[few])   # five left
        r = row(f)
        r[:8] = 2 * f if f > -4e29 else f                               # two masks
        r[V // 2] = f / 2
    for m in (1e10, 1e20, -1e10, 3e38):
        row(m, V - 1)
        row(m, slice(0, V, 3))                                          # equal maxima
        row(m, slice(0, V))
    for m in (2.0 ** 17, 1e6, 2.0 ** 20 - 1, 2.0 ** 20, 1.1e6, 2.0 ** 22, -2.0 ** 20, -2.0 ** 20 + 1, -1e6, 1e9):
        r = row()                                                       # neighbours of the type around a large number
        r.mul_(4).round_().mul_(max(2 * abs(m) * step, 0.25)).add_(m)
    x = torch.stack(rows).to(dtype)
    T = x.shape[0]
    y = torch.full((T,), -1, device=DEV) if target == "ignored" else (torch.arange(T, device=DEV) * 7) % V
    top = min(V, 32)
    o = _run_logprob(B, x, y, top)
    f = _check_logprob(x, y, top, o)
    assert bool(torch.isfinite(o["entropy"]).all()) and bool(torch.isfinite(o["lse"]).all())
    for parts in ("all", "logp"):
        _check_gradient(B, x, y, top, o, f, dtype, V, parts=parts)


@pytest.mark.gpu
def test_norms_from_many_host_threads(B):  # noqa: F811
    """Threads with a stream each call the same kernels on rows of different length, three seconds long: as if each were alone."""
    T, failures, calls = 900, [], []

    def work(C):
        h, b, w_post, _, w_pre = _norm_inputs(T, C, BF16, "rows", 0, C)
        ho, n, r2, r1 = _out(T, C, BF16), _out(T, C, BF16), torch.empty(T, device=DEV), torch.empty(T, device=DEV)
        dh, db, dwp, dw = _out(T, C, BF16), _out(T, C, BF16), torch.empty(C, device=DEV), torch.empty(C, device=DEV)
        space = torch.empty(B.def_norm_backward_workspace(T, C), dtype=torch.uint8, device=DEV)
        p = [v.data_ptr() for v in (h, b, w_post, w_pre, ho, n, r2, r1, dh, db, dwp, dw, space)]

        def both(stream):                                               # the library's own calls: no lock is held inside them
            rc = B.lib.def_norm_forward(1, T, C, p[0], C, p[1], C, p[2], None, 1, p[3], 1.0, 1e-6, p[4], C, p[5], C, p[6], p[7], None, None, None,
                                        None, None, None, stream)
            return rc or B.lib.def_norm_backward(1, T, C, p[5], C, None, 0, p[4], C, None, None, p[1], C, None, None, p[2], None, 1, p[3], 1.0,
                                                 p[6], p[7], p[8], C, p[9], C, p[10], None, p[11], 0, p[12], space.numel(), stream)
        return both, (ho, n, r2, r1, dh, db, dwp, dw), (h, b, w_post, w_pre, space)

    jobs = [work(C) for C in (4096, 2056, 4088, 2064) for _ in (0, 1)]
    alone = []
    for both, outs, _ in jobs:
        assert both(0) == B.DEF_OK
        torch.cuda.synchronize()
        alone.append([o.clone() for o in outs])
    streams = [torch.cuda.Stream() for _ in jobs]
    stop = time.monotonic() + 3

    def loop(both, stream):
        done = 0
        while time.monotonic() < stop and not failures:
            for _ in range(50):
                if both(stream.cuda_stream) != B.DEF_OK:
                    failures.append(B.def_last_error())
                    return
            done += 50
            stream.synchronize()
        calls.append(done)

    threads = [threading.Thread(target=loop, args=(job[0], stream)) for job, stream in zip(jobs, streams)]
    for t in threads:
        t.start()
    for t in threads:
        t.join()
    torch.cuda.synchronize()
    assert not failures, failures[0]
    assert len(calls) == len(jobs) and min(calls) > 0
    for (_, outs, _), want in zip(jobs, alone):
        assert all(torch.equal(o, w) for o, w in zip(outs, want))


@pytest.mark.gpu
def test_norm_of_more_groups_than_a_grid_holds(B):  # noqa: F811
    """More than 2^32 rows, each a group of its own."""
    T = (1 << 32) + 5
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB of free device memory")
    h = torch.empty((T, 1), dtype=BF16, device=DEV)
    h.normal_(generator=torch.Generator(device=DEV).manual_seed(1))
    n = torch.full((T, 1), float("nan"), dtype=BF16, device=DEV)
    r1, w = torch.full((T,), float("nan"), device=DEV), torch.full((1,), 1.5, device=DEV)
    rc = B.lib.def_norm_forward(B.DEF_DTYPE_BF16, T, 1, h.data_ptr(), 1, None, 0, None, None, T, w.data_ptr(), 1.0, 1e-5, None, 0,
                                n.data_ptr(), 1, None, r1.data_ptr(), None, None, None, None, None, None, None)
    assert rc == B.DEF_OK, B.def_last_error()
    for at in range(0, T, 1 << 28):
        x = h[at:at + (1 << 28), 0].float()
        want = torch.rsqrt(x * x + 1e-5)
        got = r1[at:at + (1 << 28)]
        assert bool(((got - want).abs() <= 8 * R.U32 * want).all())
        want = want.mul_(x).mul_(1.5)
        assert bool(((n[at:at + (1 << 28), 0].float() - want).abs() <= 1.01 * R.UNIT[BF16] * want.abs()).all())


def test_norm_backward_refuses_more_groups_than_a_grid_holds():
    from paper_2004_05298_b200 import binding

    def at(i):
        return 0x1000_0000_0000 + i * (1 << 36)                           # made up, never dereferenced

    T = 1 << 32
    need = ctypes.c_int64(0)
    assert binding.lib.def_norm_backward_workspace(T, 1, T, ctypes.byref(need)) == binding.DEF_OK
    rc = binding.lib.def_norm_backward(1, T, 1, at(0), 1, None, 0, at(1), 1, None, None, None, 0, None, None, None, None, T, at(2), 1.0, None,
                                       at(3), at(4), 1, None, 0, None, None, at(5), 0, at(6), need.value, None)
    assert rc == binding.DEF_ERR_ARG and "groups" in binding.def_last_error()


@pytest.mark.gpu
@pytest.mark.parametrize("O", [40, 4000])
def test_weight_grad_of_one_row_of_any_stride(B, O):  # noqa: F811
    """One token's row stride means nothing, not even to a tensor map (whose strides end at 2^40 bytes)."""
    I = 520
    dy, ck = _normal((1, O), BF16, 1), _checkpoint(B, _normal((1, I), BF16, 2))
    want = torch.empty((O, I), device=DEV)
    space = torch.empty((68 << 20) + 8 * O * I + 6 * (O + 7), dtype=torch.uint8, device=DEV)
    B.def_checkpoint_weight_grad(dy, ck, want, space)
    for ld in (O, 1 << 39, (1 << 59) + 8):
        dw = torch.full((O, I), 5.0, device=DEV)
        rc = B.lib.def_checkpoint_weight_grad(B.DEF_DTYPE_BF16, 1, O, I, dy.data_ptr(), ld, ck[0].data_ptr(), ck[1].data_ptr(), dw.data_ptr(), 0,
                                              space.data_ptr(), space.numel(), None)
        assert rc == B.DEF_OK, B.def_last_error()
        assert torch.equal(dw, want)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF16, F16, F32])
def test_weight_grad_of_many_tokens_of_one_sign(B, dtype):  # noqa: F811
    """16384 tokens in whole tiles, all products positive: nothing cancels, and a chain of sums is as long as they get.

    The matrix unit may drop up to a unit, 2^-23 of the running sum, each time it adds 16 products: 64 times until the
    accumulator is handed over, to a sum that grows linearly, 32.5 2^-23 = 3.9e-6 of the whole at most.  The 16 (fp32: 48)
    hand-overs round to nearest, 2^-24 each: 8.5 (40.5) more of those.  One chain over all tokens drops up to 6e-5; an fp32
    dy without its third piece is off by 2e-5, since here every number's last 8 bits are ones."""
    T, O, I = 16384, 2048, 2304                                          # 72 tiles, one for (nearly) each pair of CTAs
    dy = torch.empty((T, O), device=DEV).uniform_(1, 2, generator=torch.Generator(device=DEV).manual_seed(1))
    if dtype == F32:
        dy = (dy.view(torch.int32) | 0x80ff).view(F32)
    dy = dy.to(dtype)
    ck = _checkpoint(B, torch.empty((T, I), device=DEV).uniform_(1, 2, generator=torch.Generator(device=DEV).manual_seed(2)).to(BF16))
    space = torch.empty(B.def_checkpoint_weight_grad_workspace(dy, I), dtype=torch.uint8, device=DEV)
    dw = torch.empty((O, I), device=DEV)
    B.def_checkpoint_weight_grad(dy, ck, dw, space)
    want = dy.double().t() @ R.read(ck, I).to(DEV)
    bound = 32.5 * 2.0 ** -23 + (40.5 if dtype == F32 else 8.5) * R.U32 + R.U32
    assert float(((dw.double() - want) / want).abs().max()) <= bound


@pytest.mark.gpu
def test_alternatives_gradient_needs_their_ids(B):  # noqa: F811
    x = _normal((3, 40), F32, 1)
    y = torch.zeros(3, dtype=torch.int64, device=DEV)
    o = _run_logprob(B, x, y, 4)
    dx = torch.full_like(x, 9.0)
    with pytest.raises(B.DefError):
        B.def_logprob_backward(x, y, o["lse"], o["entropy"], dx, dtop_logp=torch.ones(3, 4, device=DEV))
    with pytest.raises(ValueError):
        B.def_logprob_backward(x, y, o["lse"], o["entropy"], dx, top_ids=o["top_ids"], dtop_logp=torch.ones(3, 5, device=DEV))
    assert bool((dx == 9).all())
    B.def_logprob_backward(x, y, o["lse"], o["entropy"], dx, top_ids=o["top_ids"])
    assert bool((dx == 0).all())
