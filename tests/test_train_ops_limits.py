"""Limits that include/def_train.h promises: the least aligned checkpoints, the largest magnitudes, calls from several
host threads, the longest runs of rows and of tokens.  Bounds as in test_train_ops_gpu.py."""
import pytest
import torch

import train_ref as R
from test_train_ops_gpu import B, BF16, DEV, F16, F32, _checkpoint, _close, _norm_inputs, _normal, _out  # noqa: F401


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
