"""Thin ctypes binding of libdef_b200.so: the same entry points as include/def.h and include/def_train.h,
taking torch tensors.  It checks dtype / contiguity / device / shape and passes data pointers;
every step of the method runs inside the library's CUDA kernels.  There is no CPU or
eager fallback: if the library cannot be built or loaded, importing fails loudly."""
import ctypes
import os

import torch

from . import build as _build

DEF_VARIANT_DEF, DEF_VARIANT_DEF_A, DEF_VARIANT_EF = 0, 1, 2
DEF_OK = 0
DEF_ERR_ARG, DEF_ERR_NULL, DEF_ERR_ALIGN, DEF_ERR_ALIAS = -1, -2, -3, -4
DEF_ERR_DEVICE, DEF_ERR_CUDA, DEF_ERR_UNSUPPORTED = -5, -6, -7
DEF_MAX_WORKERS = 64
DEF_KERNEL_STREAM, DEF_KERNEL_BLOCK, DEF_KERNEL_GENERAL = 0, 1, 2
DEF_COMPRESSOR_RBGS, DEF_COMPRESSOR_SCALE = 0, 1

_i64, _u64, _i32, _f32, _ptr = (ctypes.c_int64, ctypes.c_uint64, ctypes.c_int32, ctypes.c_float,
                                ctypes.c_void_p)

DEF_DTYPE_F32, DEF_DTYPE_BF16, DEF_DTYPE_F16 = 0, 1, 2
DEF_CHECKPOINT_GROUP = 32
DEF_NORM_MAX_C = 16384
DEF_LOGPROB_MAX_TOP = 32

# name -> (restype, argtypes): every symbol include/def.h and include/def_train.h declare
SIGNATURES = {
    "def_create": (_ptr, [_i64, _i32, _i64, _i32, _f32, _f32, _ptr]),
    "def_destroy": (ctypes.c_int, [_ptr]),
    "def_step": (ctypes.c_int, [_ptr, _ptr, _ptr, _ptr, _ptr, _u64, _u64]),
    "def_step_columns": (ctypes.c_int, [_ptr, _i64, _i64, _i64, _ptr, _ptr, _ptr, _ptr, _u64, _u64]),
    "def_step_detach": (ctypes.c_int, [_ptr, _ptr, _ptr, _ptr, _ptr, _ptr, _u64, _u64]),
    "def_step_columns_detach": (ctypes.c_int, [_ptr, _i64, _i64, _i64, _ptr, _ptr, _ptr, _ptr, _ptr, _u64, _u64]),
    "def_step_rows_local": (ctypes.c_int, [_ptr, _ptr, _ptr, _ptr, _ptr, _u64, _u64]),
    "def_step_rows_apply": (ctypes.c_int, [_ptr, _ptr, _ptr, _i32, _u64, _u64]),
    "def_step_rows_local_detach": (ctypes.c_int, [_ptr, _ptr, _ptr, _ptr, _ptr, _ptr, _ptr, _u64, _u64]),
    "def_step_rows_apply_detach": (ctypes.c_int, [_ptr, _ptr, _ptr, _i32, _ptr, _u64, _u64]),
    "def_set_rows_stream": (ctypes.c_int, [_ptr, _ptr]),
    "def_step_host": (ctypes.c_int, [_ptr, _ptr, _ptr, _ptr, _ptr, _u64, _u64]),
    "def_step_columns_host": (ctypes.c_int, [_ptr, _i64, _i64, _i64, _ptr, _ptr, _ptr, _ptr, _u64, _u64]),
    "def_detach": (ctypes.c_int, [_ptr, _i64, _i64, _ptr, _ptr, _ptr]),
    "def_output": (ctypes.c_int, [_ptr, _i64, _i64, _ptr, _ptr, _ptr]),
    "def_stats": (ctypes.c_int, [_ptr, _i64, _i64, _ptr, _ptr]),
    "def_stats_static": (ctypes.c_int, [_ptr, _i64, _i64, _i32, _f32, _ptr, _ptr]),
    "def_set_stream": (ctypes.c_int, [_ptr, _ptr]),
    "def_set_lr": (ctypes.c_int, [_ptr, _f32]),
    "def_set_small_step_bytes": (ctypes.c_int, [_ptr, _i64]),
    "def_set_compressor": (ctypes.c_int, [_ptr, _i32, _f32]),
    "def_set_pair_overlap": (ctypes.c_int, [_ptr, _i32]),
    "def_block_start": (ctypes.c_int, [_ptr, _u64, _u64, _ptr]),
    "def_block_start_device": (ctypes.c_int, [_ptr, _ptr, _ptr, _i64, _ptr, _ptr]),
    "def_launch_count": (ctypes.c_int, [_ptr, _ptr]),
    "def_tile_plan": (ctypes.c_int, [_ptr, _i64, _i64, _u64, _u64, _ptr]),
    "def_set_kernel_timing": (ctypes.c_int, [_ptr, ctypes.c_int]),
    "def_kernel_time": (ctypes.c_int, [_ptr, ctypes.c_int, _ptr, _ptr]),
    "def_last_error": (ctypes.c_char_p, []),
    "def_checkpoint_layout": (ctypes.c_int, [_i64, _ptr, _ptr]),
    "def_checkpoint_pack": (ctypes.c_int, [_i32, _i64, _i64, _ptr, _i64, _ptr, _ptr, _ptr]),
    "def_checkpoint_unpack": (ctypes.c_int, [_i32, _i64, _i64, _ptr, _ptr, _ptr, _i64, _ptr]),
    "def_checkpoint_weight_grad": (ctypes.c_int, [_i32, _i64, _i64, _i64, _ptr, _i64, _ptr, _ptr, _ptr, _i32, _ptr, _i64, _ptr]),
    "def_checkpoint_weight_grad_workspace": (ctypes.c_int, [_i32, _i64, _i64, _i64, _ptr, _i64, _ptr]),
    "def_gated_forward": (ctypes.c_int, [_i32, _i64, _i64] + [_ptr, _i64] * 3 + [_ptr] * 5),
    "def_gated_backward": (ctypes.c_int, [_i32, _i64, _i64, _ptr, _i64] + [_ptr] * 4 + [_ptr, _i64] * 3 + [_ptr] * 3),
    "def_norm_forward": (ctypes.c_int, [_i32, _i64, _i64] + [_ptr, _i64] * 2 + [_ptr, _ptr, _i64, _ptr, _f32, _f32]
                         + [_ptr, _i64] * 2 + [_ptr] * 9),
    "def_norm_backward": (ctypes.c_int, [_i32, _i64, _i64] + [_ptr, _i64] * 2 + [_ptr, _i64, _ptr, _ptr] * 2
                          + [_ptr, _ptr, _i64, _ptr, _f32, _ptr, _ptr] + [_ptr, _i64] * 2 + [_ptr] * 3 + [_i32, _ptr, _i64, _ptr]),
    "def_norm_backward_workspace": (ctypes.c_int, [_i64, _i64, _i64, _ptr]),
    "def_logprob_forward": (ctypes.c_int, [_i32, _i64, _i64, _ptr, _i64] + [_ptr] * 4 + [_i32] + [_ptr] * 3),
    "def_logprob_backward": (ctypes.c_int, [_i32, _i64, _i64, _ptr, _i64] + [_ptr] * 5 + [_i32] + [_ptr] * 3 + [_i64, _ptr]),
}


class DefError(RuntimeError):
    def __init__(self, code, message):
        super().__init__("def error %d: %s" % (code, message))
        self.code = code


def _load():
    path = _build.build()
    if not os.path.exists(path):
        raise ImportError("libdef_b200.so is missing and could not be built")
    lib = ctypes.CDLL(path)
    for name, (restype, argtypes) in SIGNATURES.items():
        fn = getattr(lib, name)          # AttributeError if the library lacks a declared symbol
        fn.restype = restype
        fn.argtypes = argtypes
    return lib


lib = _load()
LIB_PATH = _build.LIB


def def_last_error():
    return lib.def_last_error().decode()


def _check(rc):
    if rc != DEF_OK:
        raise DefError(rc, def_last_error())


def _dev(t, name, shape=None, dtype=torch.float32, optional=False):
    if t is None:
        if optional:
            return None
        raise DefError(DEF_ERR_NULL, "%s is None" % name)
    if not isinstance(t, torch.Tensor) or t.dtype != dtype or not t.is_contiguous():
        raise TypeError("%s must be a contiguous %s torch tensor" % (name, dtype))
    if not t.is_cuda:
        raise TypeError("%s must live on the GPU" % name)
    if shape is not None and tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    return t.data_ptr()


def _host(t, name, shape, optional=False):
    if t is None:
        if optional:
            return None
        raise DefError(DEF_ERR_NULL, "%s is None" % name)
    if not isinstance(t, torch.Tensor) or t.dtype != torch.float32 or not t.is_contiguous() or t.is_cuda:
        raise TypeError("%s must be a contiguous float32 CPU tensor" % name)
    if tuple(t.shape) != tuple(shape):
        raise ValueError("%s has shape %s, expected %s" % (name, tuple(t.shape), tuple(shape)))
    return t.data_ptr()


class DefCtx:
    """Owner of one def_ctx handle (freed by def_destroy or when collected)."""

    def __init__(self, handle, d, W, k, variant, lr, momentum):
        self.handle = handle
        self.d, self.W, self.k, self.variant, self.lr, self.momentum = d, W, k, variant, lr, momentum

    def __del__(self):
        if getattr(self, "handle", None):
            lib.def_destroy(self.handle)
            self.handle = None


def def_create(d, W, k, variant, lr, momentum, coeffs=None):
    arr = None
    if coeffs is not None:
        arr = (ctypes.c_float * 2)(float(coeffs[0]), float(coeffs[1]))
    handle = lib.def_create(int(d), int(W), int(k), int(variant), float(lr), float(momentum), arr)
    if not handle:
        msg = def_last_error()
        raise DefError(DEF_ERR_UNSUPPORTED if "weight decay" in msg else DEF_ERR_ARG, msg)
    return DefCtx(handle, int(d), int(W), int(k), int(variant), float(lr), float(momentum))


def def_destroy(ctx):
    if ctx.handle:
        rc = lib.def_destroy(ctx.handle)
        ctx.handle = None
        _check(rc)


def def_set_stream(ctx, stream):
    """stream: a torch.cuda.Stream, a raw cudaStream_t integer, or None (legacy default)."""
    raw = stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else (stream or 0)
    _check(lib.def_set_stream(ctx.handle, ctypes.c_void_p(raw)))


def def_set_lr(ctx, lr):
    _check(lib.def_set_lr(ctx.handle, float(lr)))
    ctx.lr = float(lr)


def def_step(ctx, params, grads, errors, mom, step, seed):
    d, W = ctx.d, ctx.W
    _check(lib.def_step(ctx.handle, _dev(params, "params", (d,)), _dev(grads, "grads", (W, d)),
                        _dev(errors, "errors", (W, d)), _dev(mom, "mom", (W, d), optional=True),
                        int(step), int(seed)))


def def_step_columns(ctx, j0, n, ld, params, grads, errors, mom, step, seed):
    """params: [n]; grads / errors / mom: [W, ld] (a rank's local column shard)."""
    W = ctx.W
    _check(lib.def_step_columns(ctx.handle, int(j0), int(n), int(ld), _dev(params, "params", (n,)),
                                _dev(grads, "grads", (W, ld)), _dev(errors, "errors", (W, ld)),
                                _dev(mom, "mom", (W, ld), optional=True), int(step), int(seed)))


def def_step_host(ctx, params, grads, errors, mom, step, seed):
    d, W = ctx.d, ctx.W
    _check(lib.def_step_host(ctx.handle, _host(params, "params", (d,)), _host(grads, "grads", (W, d)),
                             _host(errors, "errors", (W, d)), _host(mom, "mom", (W, d), optional=True),
                             int(step), int(seed)))


def def_step_columns_host(ctx, j0, n, ld, params, grads, errors, mom, step, seed):
    W = ctx.W
    _check(lib.def_step_columns_host(ctx.handle, int(j0), int(n), int(ld), _host(params, "params", (n,)),
                                     _host(grads, "grads", (W, ld)), _host(errors, "errors", (W, ld)),
                                     _host(mom, "mom", (W, ld), optional=True), int(step), int(seed)))


def def_block_start(ctx, step, seed):
    out = ctypes.c_int64(-1)
    _check(lib.def_block_start(ctx.handle, int(step), int(seed), ctypes.byref(out)))
    return int(out.value)


def def_block_start_device(seeds, steps, ds, starts_out, stream=None):
    """seeds, steps: uint64 bit patterns held in int64 CUDA tensors; ds, starts_out: int64."""
    n = seeds.numel()
    raw = stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else (stream or 0)
    _check(lib.def_block_start_device(_dev(seeds, "seeds", (n,), torch.int64),
                                      _dev(steps, "steps", (n,), torch.int64),
                                      _dev(ds, "ds", (n,), torch.int64), n,
                                      _dev(starts_out, "starts_out", (n,), torch.int64),
                                      ctypes.c_void_p(raw)))


def def_tile_plan(ctx, j0, n, step, seed):
    """(first tile of run A, its tiles, tiles of run B from tile 0, tiles left to the stream kernel)."""
    out = (ctypes.c_int64 * 4)()
    _check(lib.def_tile_plan(ctx.handle, int(j0), int(n), int(step), int(seed), out))
    return tuple(int(v) for v in out)


def def_launch_count(ctx):
    out = ctypes.c_int64(0)
    _check(lib.def_launch_count(ctx.handle, ctypes.byref(out)))
    return int(out.value)


def def_set_kernel_timing(ctx, enable):
    _check(lib.def_set_kernel_timing(ctx.handle, 1 if enable else 0))


def def_kernel_time(ctx, kernel):
    """(total device milliseconds, launches) of one kernel kind since def_create."""
    ms, n = ctypes.c_double(0.0), ctypes.c_int64(0)
    _check(lib.def_kernel_time(ctx.handle, int(kernel), ctypes.byref(ms), ctypes.byref(n)))
    return float(ms.value), int(n.value)


def def_detach(ctx, params, errors, detached_out, n=None, ld=None):
    """detached_out[w] = params - lambda * errors[w]; whole model unless n / ld name a column view."""
    n = ctx.d if n is None else int(n)
    ld = n if ld is None else int(ld)
    _check(lib.def_detach(ctx.handle, n, ld, _dev(params, "params", (n,)), _dev(errors, "errors", (ctx.W, ld)),
                          _dev(detached_out, "detached_out", (ctx.W, ld))))


def def_output(ctx, params, errors, model_out, n=None, ld=None):
    """The model Algorithm 1 returns: y_T for DEF, x_T for DEF-A and EF."""
    n = ctx.d if n is None else int(n)
    ld = n if ld is None else int(ld)
    _check(lib.def_output(ctx.handle, n, ld, _dev(params, "params", (n,)),
                          _dev(errors, "errors", (ctx.W, ld), optional=True), _dev(model_out, "model_out", (n,))))


def def_stats(ctx, errors, stats_out, n=None, ld=None):
    """stats_out: 3 float64 on the GPU (see include/def.h)."""
    n = ctx.d if n is None else int(n)
    ld = n if ld is None else int(ld)
    _check(lib.def_stats(ctx.handle, n, ld, _dev(errors, "errors", (ctx.W, ld)),
                         _dev(stats_out, "stats_out", (3,), torch.float64)))


DEF_STATS_STATIC_SLOTS = 2048
DEF_STATS_STATIC_MAX_N = 1 << 31


def def_stats_static(errors, lam, stats_out, n=None, ld=None, stream=None):
    """def_stats without any allocation and without a context: the scratch is a fixed array in
    the library's device image (see include/def.h for who needs this and for its rules).
    errors: [W, ld] float32 on the GPU; stats_out: 3 float64 on the GPU."""
    W = errors.shape[0]
    ld = errors.shape[1] if ld is None else int(ld)
    n = ld if n is None else int(n)
    raw = stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else (stream or 0)
    _check(lib.def_stats_static(_dev(errors, "errors", (W, ld)), n, ld, int(W), float(lam),
                                _dev(stats_out, "stats_out", (3,), torch.float64), ctypes.c_void_p(raw)))


def def_step_detach(ctx, params, grads, errors, mom, detached_out, step, seed):
    d, W = ctx.d, ctx.W
    _check(lib.def_step_detach(ctx.handle, _dev(params, "params", (d,)), _dev(grads, "grads", (W, d)),
                               _dev(errors, "errors", (W, d)), _dev(mom, "mom", (W, d), optional=True),
                               _dev(detached_out, "detached_out", (W, d)), int(step), int(seed)))


def def_step_columns_detach(ctx, j0, n, ld, params, grads, errors, mom, detached_out, step, seed):
    W = ctx.W
    _check(lib.def_step_columns_detach(ctx.handle, int(j0), int(n), int(ld), _dev(params, "params", (n,)),
                                       _dev(grads, "grads", (W, ld)), _dev(errors, "errors", (W, ld)),
                                       _dev(mom, "mom", (W, ld), optional=True),
                                       _dev(detached_out, "detached_out", (W, ld)), int(step), int(seed)))


def def_set_small_step_bytes(ctx, nbytes):
    _check(lib.def_set_small_step_bytes(ctx.handle, int(nbytes)))


DEF_OVERLAP_AUTO, DEF_OVERLAP_NEVER, DEF_OVERLAP_ALWAYS = 0, 1, 2


def def_set_pair_overlap(ctx, mode):
    _check(lib.def_set_pair_overlap(ctx.handle, int(mode)))


def def_set_compressor(ctx, compressor, delta=0.0):
    _check(lib.def_set_compressor(ctx.handle, int(compressor), float(delta)))


def def_step_rows_local(ctx, grads, errors, mom, block_sum_out, step, seed):
    d, W = ctx.d, ctx.W
    _check(lib.def_step_rows_local(ctx.handle, _dev(grads, "grads", (W, d)), _dev(errors, "errors", (W, d)),
                                   _dev(mom, "mom", (W, d), optional=True),
                                   _dev(block_sum_out, "block_sum_out", (ctx.k,)), int(step), int(seed)))


def def_step_rows_apply(ctx, params, block_sum, W_total, step, seed):
    _check(lib.def_step_rows_apply(ctx.handle, _dev(params, "params", (ctx.d,)),
                                   _dev(block_sum, "block_sum", (ctx.k,)), int(W_total), int(step), int(seed)))


def def_step_rows_local_detach(ctx, params, grads, errors, mom, block_sum_out, detached_out, step, seed):
    d, W = ctx.d, ctx.W
    _check(lib.def_step_rows_local_detach(ctx.handle, _dev(params, "params", (d,)), _dev(grads, "grads", (W, d)),
                                          _dev(errors, "errors", (W, d)), _dev(mom, "mom", (W, d), optional=True),
                                          _dev(block_sum_out, "block_sum_out", (ctx.k,)),
                                          _dev(detached_out, "detached_out", (W, d)), int(step), int(seed)))


def def_step_rows_apply_detach(ctx, params, block_sum, W_total, detached_out, step, seed):
    _check(lib.def_step_rows_apply_detach(ctx.handle, _dev(params, "params", (ctx.d,)),
                                          _dev(block_sum, "block_sum", (ctx.k,)), int(W_total),
                                          _dev(detached_out, "detached_out", (ctx.W, ctx.d)), int(step), int(seed)))


def def_set_rows_stream(ctx, stream):
    """Side stream of the row-sharded step (a torch.cuda.Stream, or None to switch it off): the
    block kernel, the all-reduce and the update run there, beside the streaming kernel."""
    raw = stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else (stream or 0)
    _check(lib.def_set_rows_stream(ctx.handle, ctypes.c_void_p(raw)))
    ctx.rows_stream = stream if isinstance(stream, torch.cuda.Stream) else None


def def_step_rows(ctx, params, grads, errors, mom, block_sum, step, seed, group=None, detached_out=None):
    """One row-sharded step: local half, all-reduce of the k block sums over `group` (NCCL through
    torch.distributed), apply.  W_total = local W times the group size.  After def_set_rows_stream
    the all-reduce is issued on that side stream, where the library has put the block kernel and
    puts the update, so that it overlaps the streaming kernel on the context's stream."""
    import torch.distributed as dist
    if detached_out is None:
        def_step_rows_local(ctx, grads, errors, mom, block_sum, step, seed)
    else:
        def_step_rows_local_detach(ctx, params, grads, errors, mom, block_sum, detached_out, step, seed)
    side = getattr(ctx, "rows_stream", None)
    if side is not None:
        with torch.cuda.stream(side):
            dist.all_reduce(block_sum, op=dist.ReduceOp.SUM, group=group)
    else:
        dist.all_reduce(block_sum, op=dist.ReduceOp.SUM, group=group)
    W_total = ctx.W * dist.get_world_size(group)
    if detached_out is None:
        def_step_rows_apply(ctx, params, block_sum, W_total, step, seed)
    else:
        def_step_rows_apply_detach(ctx, params, block_sum, W_total, detached_out, step, seed)


# --- operators of the training step around def_step (include/def_train.h) ------------------------------------------
#
# Activations are [T, C] tensors of float32, bfloat16 or float16 with consecutive columns and any row stride; a
# checkpoint is a pair (q, e) made by def_checkpoint_alloc.  `stream`: as in def_block_start_device.

_DTYPES = {torch.float32: DEF_DTYPE_F32, torch.bfloat16: DEF_DTYPE_BF16, torch.float16: DEF_DTYPE_F16}


def _stream(stream):
    return stream.cuda_stream if isinstance(stream, torch.cuda.Stream) else (stream or 0)


def _act(t, name, like=None):
    """(dtype code, T, C, pointer, row stride) of an activation; `like`: another's, to agree with."""
    try:
        code = _DTYPES[t.dtype]
        T, C = t.shape
        ld, inner = t.stride()
    except (AttributeError, KeyError, ValueError, TypeError):
        raise TypeError("%s must be a two-dimensional float32, bfloat16 or float16 torch tensor" % name) from None
    if not t.is_cuda:
        raise TypeError("%s must live on the GPU" % name)
    if inner != 1 and C > 1:
        raise ValueError("the columns of %s must be consecutive" % name)
    if T <= 1:
        ld = C
    if like is not None and (code != like[0] or T != like[1] or C != like[2]):
        raise ValueError("%s is %s of %s, expected type %d and shape %s" % (name, t.dtype, (T, C), like[0], like[1:3]))
    return code, T, C, t.data_ptr(), ld


def _opt_act(t, name, like):
    return (None, 0) if t is None else _act(t, name, like)[3:]


def _held(ck, name, T, C):
    """(q pointer, e pointer) of a checkpoint of [T, C], or of None."""
    if ck is None:
        return None, None
    q, e = ck
    return (_param(q, name, (T, (C + 15) // 16 * 16), torch.int8), _param(e, name, (T, (C + 127) // 128 * 4), torch.uint8))


def _param(t, name, shape, dtype=torch.float32):
    """Pointer of a contiguous tensor of this shape, or of None; _dev says what is wrong where something is."""
    if t is None:
        return None
    try:
        if t.dtype is dtype and t.shape == shape and t.is_cuda and t.is_contiguous():
            return t.data_ptr()
    except AttributeError:
        pass
    return _dev(t, name, shape, dtype)


def _need(t, name, shape, dtype=torch.float32):
    return _dev(t, name, shape, dtype) if t is None else _param(t, name, shape, dtype)


def _work(t, name):
    if t is None:
        return None, 0
    return _dev(t, name, None, torch.uint8), t.numel()


def def_checkpoint_layout(C):
    """(bytes per row of the 8-bit integers, bytes per row of the exponents) of a checkpoint of [T, C]."""
    ldq, lde = ctypes.c_int64(0), ctypes.c_int64(0)
    _check(lib.def_checkpoint_layout(int(C), ctypes.byref(ldq), ctypes.byref(lde)))
    return int(ldq.value), int(lde.value)


def def_checkpoint_alloc(T, C, device):
    """An uninitialised checkpoint (q, e) of [T, C] from torch's allocator."""
    ldq, lde = def_checkpoint_layout(C)
    return torch.empty((T, ldq), dtype=torch.int8, device=device), torch.empty((T, lde), dtype=torch.uint8, device=device)


def def_checkpoint_pack(x, ck, stream=None):
    dt, T, C, p, ld = _act(x, "x")
    q, e = _held(ck, "checkpoint", T, C)
    _check(lib.def_checkpoint_pack(dt, T, C, p, ld, q, e, _stream(stream)))


def def_checkpoint_unpack(ck, out, stream=None):
    dt, T, C, p, ld = _act(out, "out")
    q, e = _held(ck, "checkpoint", T, C)
    _check(lib.def_checkpoint_unpack(dt, T, C, q, e, p, ld, _stream(stream)))


def def_checkpoint_weight_grad_workspace(dy, I):
    dt, T, O, p, ld = _act(dy, "dy")
    out = ctypes.c_int64(0)
    _check(lib.def_checkpoint_weight_grad_workspace(dt, T, O, int(I), p, ld, ctypes.byref(out)))
    return int(out.value)


def def_checkpoint_weight_grad(dy, ck, dw, workspace=None, accumulate=False, stream=None):
    """dw [O, I] (float32) (+)= dy^T times the [T, I] checkpoint."""
    dt, T, O, p, ld = _act(dy, "dy")
    if not isinstance(dw, torch.Tensor) or dw.dim() != 2:
        raise TypeError("dw must be a two-dimensional torch tensor")
    I = dw.shape[1]
    q, e = _held(ck, "checkpoint", T, I)
    w, nw = _work(workspace, "workspace")
    _check(lib.def_checkpoint_weight_grad(dt, T, O, I, p, ld, q, e, _need(dw, "dw", (O, I)), 1 if accumulate else 0, w, nw, _stream(stream)))


def def_gated_forward(gate, up, h, gate_ck=None, up_ck=None, stream=None):
    g = _act(gate, "gate")
    dt, T, F = g[:3]
    gq, ge = _held(gate_ck, "gate checkpoint", T, F)
    uq, ue = _held(up_ck, "up checkpoint", T, F)
    _check(lib.def_gated_forward(dt, T, F, *g[3:], *_act(up, "up", g)[3:], *_act(h, "h", g)[3:], gq, ge, uq, ue, _stream(stream)))


def def_gated_backward(dh, gate_ck, up_ck, dgate, dup, h_out=None, h_ck=None, stream=None):
    d = _act(dh, "dh")
    dt, T, F = d[:3]
    gq, ge = _held(gate_ck, "gate checkpoint", T, F)
    uq, ue = _held(up_ck, "up checkpoint", T, F)
    hq, he = _held(h_ck, "h checkpoint", T, F)
    _check(lib.def_gated_backward(dt, T, F, *d[3:], gq, ge, uq, ue, *_act(dgate, "dgate", d)[3:], *_act(dup, "dup", d)[3:],
                                  *_opt_act(h_out, "h_out", d), hq, he, _stream(stream)))


def def_norm_forward(h, b, w_post, gate, w_pre, h_out, n_out, rstd_post, rstd_pre, res_scale=1.0, eps=1e-6, b_ck=None, h_ck=None,
                     n_ck=None, stream=None):
    """h_out = res_scale h + gate norm(b) w_post, n_out = norm(h_out) w_pre; with b (and w_post, gate, h_out, rstd_post)
    None: n_out = norm(h) w_pre.  gate: [groups, C] or None."""
    a = _act(h, "h")
    dt, T, C = a[:3]
    groups = 1 if gate is None else gate.shape[0]
    bq, be = _held(b_ck, "b checkpoint", T, C)
    hq, he = _held(h_ck, "h checkpoint", T, C)
    nq, ne = _held(n_ck, "n checkpoint", T, C)
    _check(lib.def_norm_forward(dt, T, C, *a[3:], *_opt_act(b, "b", a), _param(w_post, "w_post", (C,)), _param(gate, "gate", (groups, C)),
                                groups, _param(w_pre, "w_pre", (C,)), res_scale, eps, *_opt_act(h_out, "h_out", a),
                                *_act(n_out, "n_out", a)[3:], _param(rstd_post, "rstd_post", (T,)), _param(rstd_pre, "rstd_pre", (T,)),
                                bq, be, hq, he, nq, ne, _stream(stream)))


def def_norm_backward_workspace(T, C, groups=1):
    out = ctypes.c_int64(0)
    _check(lib.def_norm_backward_workspace(int(T), int(C), int(groups), ctypes.byref(out)))
    return int(out.value)


def def_norm_backward(dn, dh_in, h, b, w_post, gate, w_pre, rstd_post, rstd_pre, dh, db, dw_post, dgate, dw_pre, workspace,
                      res_scale=1.0, accumulate=False, stream=None):
    """h and b: the stored tensors, or checkpoints (q, e) of them; dh_in None: zero."""
    a = _act(dn, "dn")
    dt, T, C = a[:3]
    groups = 1 if gate is None else gate.shape[0]
    hq, he = _held(h, "h checkpoint", T, C) if isinstance(h, tuple) else (None, None)
    bq, be = _held(b, "b checkpoint", T, C) if isinstance(b, tuple) else (None, None)
    hp = _opt_act(None if hq is not None else h, "h", a)
    bp = _opt_act(None if bq is not None else b, "b", a)
    w, nw = _work(workspace, "workspace")
    _check(lib.def_norm_backward(dt, T, C, *a[3:], *_opt_act(dh_in, "dh_in", a), *hp, hq, he, *bp, bq, be,
                                 _param(w_post, "w_post", (C,)), _param(gate, "gate", (groups, C)), groups, _param(w_pre, "w_pre", (C,)),
                                 res_scale, _param(rstd_post, "rstd_post", (T,)), _param(rstd_pre, "rstd_pre", (T,)),
                                 *_act(dh, "dh", a)[3:], *_opt_act(db, "db", a), _param(dw_post, "dw_post", (C,)),
                                 _param(dgate, "dgate", (groups, C)), _param(dw_pre, "dw_pre", (C,)), 1 if accumulate else 0,
                                 w, nw, _stream(stream)))


def def_logprob_forward(logits, targets, logp, entropy, lse, top_ids=None, top_logp=None, stream=None):
    """targets: int64 [T]; lse: float32 [T, 2] (maximum, log of the sum relative to it); top_ids: int64 [T, top]."""
    dt, T, V, p, ld = _act(logits, "logits")
    top = 0 if top_ids is None else top_ids.shape[1]
    _check(lib.def_logprob_forward(dt, T, V, p, ld, _need(targets, "targets", (T,), torch.int64), _need(logp, "logp", (T,)),
                                   _need(entropy, "entropy", (T,)), _need(lse, "lse", (T, 2)), top,
                                   _param(top_ids, "top_ids", (T, top), torch.int64), _param(top_logp, "top_logp", (T, top)),
                                   _stream(stream)))


def def_logprob_backward(logits, targets, lse, entropy, dlogits, dlogp=None, dentropy=None, top_ids=None, dtop_logp=None, stream=None):
    """dtop_logp needs top_ids; top_ids without it is not looked at."""
    a = _act(logits, "logits")
    dt, T, V, p, ld = a
    if top_ids is None and dtop_logp is not None:
        raise DefError(DEF_ERR_NULL, "top_ids is None, but dtop_logp is given")
    top = 0 if dtop_logp is None else top_ids.shape[1]
    if top == 0:
        top_ids = dtop_logp = None
    _check(lib.def_logprob_backward(dt, T, V, p, ld, _need(targets, "targets", (T,), torch.int64), _need(lse, "lse", (T, 2)),
                                    _need(entropy, "entropy", (T,)), _param(dlogp, "dlogp", (T,)), _param(dentropy, "dentropy", (T,)), top,
                                    _param(top_ids, "top_ids", (T, top), torch.int64), _param(dtop_logp, "dtop_logp", (T, top)),
                                    *_act(dlogits, "dlogits", a)[3:], _stream(stream)))
