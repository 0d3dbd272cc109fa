// C boundary of the operators around the step (see include/def_train.h): argument validation, kernel selection, launch.
#include "../../include/def_train.h"
#include "def_checkpoint_kernels.cuh"
#include "def_error.cuh"
#include "def_logprob_kernels.cuh"
#include "def_norm_kernels.cuh"
#include "def_weight_grad_kernels.cuh"

#include <atomic>
#include <cstring>

#include <cuda.h>

namespace {

using defk::cuda_fail;
using defk::fail;

constexpr int kMaxDevices = 64;

// SMs of the current device; negative (an error code) if it cannot run these kernels.  The answer is looked up once
// per device.
int sm_count() {
    static std::atomic<int> known[kMaxDevices];
    int dev = -1;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess || dev < 0 || dev >= kMaxDevices) {
        cudaGetLastError();
        return fail(DEF_ERR_DEVICE, "no usable CUDA device: %s", cudaGetErrorString(err));
    }
    int sms = known[dev].load(std::memory_order_relaxed);
    if (sms > 0) return sms;
    int major = 0;
    if ((err = cudaDeviceGetAttribute(&major, cudaDevAttrComputeCapabilityMajor, dev)) != cudaSuccess ||
        (err = cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev)) != cudaSuccess) {
        cudaGetLastError();
        return fail(DEF_ERR_DEVICE, "cannot query device %d: %s", dev, cudaGetErrorString(err));
    }
    if (major != 10) return fail(DEF_ERR_DEVICE, "device %d is compute capability %d.x; this library is built for 10.x (sm_100a)", dev, major);
    known[dev].store(sms, std::memory_order_relaxed);
    return sms;
}

int element_size(int32_t dtype) { return dtype == DEF_DTYPE_F32 ? 4 : dtype == DEF_DTYPE_BF16 || dtype == DEF_DTYPE_F16 ? 2 : 0; }

int64_t ceil_div(int64_t a, int64_t b) { return (a + b - 1) / b; }
int64_t q_stride(int64_t C) { return ceil_div(C, 16) * 16; }
int64_t e_stride(int64_t C) { return ceil_div(ceil_div(C, deft::kGroup), 4) * 4; }

// One tensor argument: `rows` runs of `width` bytes, `stride` bytes apart.
struct View {
    const void *p;
    const char *name;
    int64_t rows, width, stride;
    unsigned align;
    bool written;
};

bool share_bytes(const View &a, const View &b) {
    if (!a.p || !b.p || a.rows == 0 || b.rows == 0) return false;
    const uint64_t a0 = (uint64_t)(uintptr_t)a.p, b0 = (uint64_t)(uintptr_t)b.p;
    const uint64_t a1 = a0 + (uint64_t)(a.rows - 1) * a.stride + a.width, b1 = b0 + (uint64_t)(b.rows - 1) * b.stride + b.width;
    if (a1 <= b0 || b1 <= a0) return false;
    if (a.stride != b.stride || a.width > a.stride || b.width > b.stride) return true;
    const uint64_t s = (uint64_t)a.stride;           // how far b's columns start behind a's, in [0, s)
    const int64_t d = (int64_t)(b0 >= a0 ? (b0 - a0) % s : (s - (a0 - b0) % s) % s);
    return !(d >= a.width && d + b.width <= a.stride);      // column ranges of one buffer are apart
}

// Alignment, and that nothing written shares memory with another argument, except that the output `out` may be the
// input `in`, row for row.
template <int N> int check_views(const View (&v)[N], int in = -1, int out = -1) {
    for (const View &a : v)
        if (a.p && ((uintptr_t)a.p & (a.align - 1))) return fail(DEF_ERR_ALIGN, "%s is not %u-byte aligned", a.name, a.align);
    for (int i = 0; i < N; ++i)
        for (int j = i + 1; j < N; ++j)
            if ((v[i].written || v[j].written) && share_bytes(v[i], v[j])) {
                if (i == in && j == out && v[i].p == v[j].p && (v[i].stride == v[j].stride || v[i].rows == 1)) continue;
                return fail(DEF_ERR_ALIAS, "%s and %s overlap", v[i].name, v[j].name);
            }
    return DEF_OK;
}

int check_rows(int32_t dtype, int64_t T, int64_t C, const char *width) {
    if (!element_size(dtype)) return fail(DEF_ERR_ARG, "dtype must be one of DEF_DTYPE_F32, _BF16, _F16 (got %d)", dtype);
    if (T < 0) return fail(DEF_ERR_ARG, "T must not be negative (got %lld)", (long long)T);
    if (C < 1) return fail(DEF_ERR_ARG, "%s must be at least 1 (got %lld)", width, (long long)C);
    if (T > ((int64_t)1 << 40) || C > (int64_t)1 << 30) return fail(DEF_ERR_ARG, "T or %s is too large", width);
    return DEF_OK;
}
int check_stride(const void *p, int64_t ld, int64_t C, int64_t T, const char *name) {
    if (p && ld < C) return fail(DEF_ERR_ARG, "the row stride of %s must be at least its width (got %lld)", name, (long long)ld);
    if (p && ld > ((int64_t)1 << 60) / (T > 0 ? T : 1)) return fail(DEF_ERR_ARG, "the rows of %s reach too far", name);
    return DEF_OK;
}
int check_pair(const void *q, const void *e, const char *name) {
    if (!q != !e) return fail(DEF_ERR_NULL, "%s_q and %s_e must both be given or both be NULL", name, name);
    return DEF_OK;
}
#define DEF_TRY(call) do { const int rc_ = (call); if (rc_ != DEF_OK) return rc_; } while (0)

View rows_view(const void *p, const char *name, int64_t T, int64_t C, int64_t ld, int64_t es, bool written) {
    return {p, name, T, C * es, ld * es, (unsigned)es, written};
}
View q_view(const void *p, const char *name, int64_t T, int64_t C, bool written) { return {p, name, T, C, q_stride(C), 16, written}; }
View e_view(const void *p, const char *name, int64_t T, int64_t C, bool written) {
    return {p, name, T, ceil_div(C, deft::kGroup), e_stride(C), 4, written};
}
View floats_view(const void *p, const char *name, int64_t n, bool written) { return {p, name, p ? 1 : 0, n * 4, n * 4, 4, written}; }

// Whether rows of C elements at p, stride ld, can be read and written 8 elements at a time.
bool wide(const void *p, int64_t ld, int64_t es) { return !p || (((uintptr_t)p & 15u) == 0 && ld * es % 16 == 0); }

int launched(const char *what) {
    const cudaError_t err = cudaGetLastError();
    return err == cudaSuccess ? DEF_OK : cuda_fail(err, what);
}

// Calls f with a value of the element type.
template <typename F> void by_dtype(int32_t dtype, F f) {
    if (dtype == DEF_DTYPE_F32) f(float());
    else if (dtype == DEF_DTYPE_BF16) f(__nv_bfloat16());
    else f(__half());
}

constexpr int kUsualSms = 148;      // what launches and workspaces are sized for before a device is looked at

template <bool B> struct Is { static constexpr bool value = B; };
template <typename F> void by_alignment(bool aligned, F f) {
    if (aligned) f(Is<true>());
    else f(Is<false>());
}

// Rows of its columns that a CTA of these kernels walks, where that leaves enough CTAs.  1, 2, 4, 8 of them, us: 16384 x 8192
// bf16 pack 85, 76, 73, 73, unpack 96, 79, 76, 76, gated backward 239, 216, 208, 208; 16384 x 4097 bf16 pack 80, 68, 63, 62;
// 8192 x 4096 fp32 pack 27 each, gated forward 76, 76, 78, 78.
constexpr int kPlaneRows = 4;
// Launch of a kernel that works on rows by columns without sums: a warp lies in one row.  f(aligned, grid, block).
template <typename F> void on_plane(bool aligned, int64_t T, int64_t C, F f) {
    const int64_t lanes = ceil_div(C, 8);
    unsigned bx = 32;
    while (bx < 256 && bx < lanes) bx *= 2;
    const dim3 block(bx, 256 / bx);
    // Several rows per CTA: fewer instructions go into addresses.
    const int64_t gx = ceil_div(lanes, bx), all = ceil_div(T, block.y);
    int64_t gy = ceil_div(all, kPlaneRows);
    if (gx * gy < 32 * kUsualSms) gy = ceil_div(32 * kUsualSms, gx) < all ? ceil_div(32 * kUsualSms, gx) : all;
    const dim3 grid((unsigned)gx, (unsigned)(gy < 65535 ? gy : 65535));
    by_alignment(aligned, [&](auto is_aligned) { f(is_aligned, grid, block); });
}

}  // namespace

extern "C" int def_checkpoint_layout(int64_t C, int64_t *ldq_out, int64_t *lde_out) {
    if (!ldq_out || !lde_out) return fail(DEF_ERR_NULL, "ldq_out and lde_out must not be NULL");
    if (C < 1 || C > (int64_t)1 << 30) return fail(DEF_ERR_ARG, "C must be in [1, 2^30] (got %lld)", (long long)C);
    *ldq_out = q_stride(C);
    *lde_out = e_stride(C);
    return DEF_OK;
}

extern "C" int def_checkpoint_pack(int32_t dtype, int64_t T, int64_t C, const void *x, int64_t ldx, int8_t *q, uint8_t *e,
                                   void *cuda_stream) {
    DEF_TRY(check_rows(dtype, T, C, "C"));
    if (T == 0) return DEF_OK;
    if (!x || !q || !e) return fail(DEF_ERR_NULL, "x, q and e must not be NULL");
    DEF_TRY(check_stride(x, ldx, C, T, "x"));
    const int es = element_size(dtype);
    const View views[] = {rows_view(x, "x", T, C, ldx, es, false), q_view(q, "q", T, C, true), e_view(e, "e", T, C, true)};
    DEF_TRY(check_views(views));
    if (const int sms = sm_count(); sms < 0) return sms;
    const bool aligned_rows = C % 8 == 0 && wide(x, ldx, es);
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        on_plane(aligned_rows, T, C, [&](auto v, dim3 grid, dim3 block) {
            deft::pack_kernel<E, v.value><<<grid, block, 0, (cudaStream_t)cuda_stream>>>((const E *)x, ldx, T, (int)C, q, e, q_stride(C), e_stride(C));
        });
    });
    return launched("def_checkpoint_pack");
}

extern "C" int def_checkpoint_unpack(int32_t dtype, int64_t T, int64_t C, const int8_t *q, const uint8_t *e, void *out,
                                     int64_t ldout, void *cuda_stream) {
    DEF_TRY(check_rows(dtype, T, C, "C"));
    if (T == 0) return DEF_OK;
    if (!out || !q || !e) return fail(DEF_ERR_NULL, "q, e and out must not be NULL");
    DEF_TRY(check_stride(out, ldout, C, T, "out"));
    const int es = element_size(dtype);
    const View views[] = {rows_view(out, "out", T, C, ldout, es, true), q_view(q, "q", T, C, false), e_view(e, "e", T, C, false)};
    DEF_TRY(check_views(views));
    if (const int sms = sm_count(); sms < 0) return sms;
    const bool aligned_rows = C % 8 == 0 && wide(out, ldout, es);
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        on_plane(aligned_rows, T, C, [&](auto v, dim3 grid, dim3 block) {
            deft::unpack_kernel<E, v.value><<<grid, block, 0, (cudaStream_t)cuda_stream>>>(q, e, q_stride(C), e_stride(C), T, (int)C, (E *)out, ldout);
        });
    });
    return launched("def_checkpoint_unpack");
}

extern "C" int def_gated_forward(int32_t dtype, int64_t T, int64_t F, const void *gate, int64_t ldg, const void *up, int64_t ldu,
                                 void *h, int64_t ldh, int8_t *gate_q, uint8_t *gate_e, int8_t *up_q, uint8_t *up_e,
                                 void *cuda_stream) {
    DEF_TRY(check_rows(dtype, T, F, "F"));
    if (T == 0) return DEF_OK;
    if (!gate || !up || !h) return fail(DEF_ERR_NULL, "gate, up and h must not be NULL");
    DEF_TRY(check_pair(gate_q, gate_e, "gate"));
    DEF_TRY(check_pair(up_q, up_e, "up"));
    DEF_TRY(check_stride(gate, ldg, F, T, "gate"));
    DEF_TRY(check_stride(up, ldu, F, T, "up"));
    DEF_TRY(check_stride(h, ldh, F, T, "h"));
    const int es = element_size(dtype);
    const View views[] = {rows_view(gate, "gate", T, F, ldg, es, false), rows_view(up, "up", T, F, ldu, es, false),
                          rows_view(h, "h", T, F, ldh, es, true), q_view(gate_q, "gate_q", T, F, true), e_view(gate_e, "gate_e", T, F, true),
                          q_view(up_q, "up_q", T, F, true), e_view(up_e, "up_e", T, F, true)};
    DEF_TRY(check_views(views));
    if (const int sms = sm_count(); sms < 0) return sms;
    deft::GatedForward a = {gate, up, h, ldg, ldu, ldh, gate_q, up_q, gate_e, up_e, T, F, q_stride(F), e_stride(F)};
    const bool aligned_rows = F % 8 == 0 && wide(gate, ldg, es) && wide(up, ldu, es) && wide(h, ldh, es);
    by_dtype(dtype, [&](auto type) {
        on_plane(aligned_rows, T, F, [&](auto v, dim3 grid, dim3 block) {
            deft::gated_forward_kernel<decltype(type), v.value><<<grid, block, 0, (cudaStream_t)cuda_stream>>>(a);
        });
    });
    return launched("def_gated_forward");
}

extern "C" int def_gated_backward(int32_t dtype, int64_t T, int64_t F, const void *dh, int64_t lddh, const int8_t *gate_q,
                                  const uint8_t *gate_e, const int8_t *up_q, const uint8_t *up_e, void *dgate, int64_t lddg,
                                  void *dup, int64_t lddu, void *h_out, int64_t ldh, int8_t *h_q, uint8_t *h_e, void *cuda_stream) {
    DEF_TRY(check_rows(dtype, T, F, "F"));
    if (T == 0) return DEF_OK;
    if (!dh || !gate_q || !gate_e || !up_q || !up_e || !dgate || !dup)
        return fail(DEF_ERR_NULL, "dh, the checkpoints of gate and up, dgate and dup must not be NULL");
    DEF_TRY(check_pair(h_q, h_e, "h"));
    DEF_TRY(check_stride(dh, lddh, F, T, "dh"));
    DEF_TRY(check_stride(dgate, lddg, F, T, "dgate"));
    DEF_TRY(check_stride(dup, lddu, F, T, "dup"));
    DEF_TRY(check_stride(h_out, ldh, F, T, "h_out"));
    const int es = element_size(dtype);
    const View views[] = {rows_view(dh, "dh", T, F, lddh, es, false), q_view(gate_q, "gate_q", T, F, false), e_view(gate_e, "gate_e", T, F, false),
                          q_view(up_q, "up_q", T, F, false), e_view(up_e, "up_e", T, F, false), rows_view(dgate, "dgate", T, F, lddg, es, true),
                          rows_view(dup, "dup", T, F, lddu, es, true), rows_view(h_out, "h_out", T, F, ldh, es, true),
                          q_view(h_q, "h_q", T, F, true), e_view(h_e, "h_e", T, F, true)};
    DEF_TRY(check_views(views));
    if (const int sms = sm_count(); sms < 0) return sms;
    deft::GatedBackward a = {dh, gate_q, up_q, gate_e, up_e, dgate, dup, h_out, lddh, lddg, lddu, ldh, h_q, h_e, T, F, q_stride(F), e_stride(F)};
    const bool aligned_rows = F % 8 == 0 && wide(dh, lddh, es) && wide(dgate, lddg, es) && wide(dup, lddu, es) && wide(h_out, ldh, es);
    by_dtype(dtype, [&](auto type) {
        on_plane(aligned_rows, T, F, [&](auto v, dim3 grid, dim3 block) {
            deft::gated_backward_kernel<decltype(type), v.value><<<grid, block, 0, (cudaStream_t)cuda_stream>>>(a);
        });
    });
    return launched("def_gated_backward");
}

// ---------------------------------------------------------------------------
// Norms
// ---------------------------------------------------------------------------
namespace {

// Most threads per CTA that a kernel is compiled for, runs of 8 columns per thread, CTAs per SM that its registers are for.
template <int MOST, int ITERS> struct Shape {
    static constexpr int most = MOST, iters = ITERS;
    // as few threads as cover the row
    static int threads(int64_t C) { return (int)(ceil_div(ceil_div(C, 8 * ITERS), 32) * 32); }
};
template <int MOST, int ITERS, int MINB> struct StreamShape : Shape<MOST, ITERS> { static constexpr int min_ctas = MINB; };
template <typename F> void by_row_shape(int64_t C, F f) {
    const int64_t n = ceil_div(C, 8);
    if (n <= 256) f(Shape<256, 1>());
    else if (n <= 512) f(Shape<256, 2>());
    else if (n <= 1024) f(Shape<512, 2>());
    else f(Shape<1024, 2>());
}
// 288 threads rather than 512 for the widths that 256 just miss, us: 16384 x 4352 bf16 forward 99 against 158, backward 148
// against 193 (8-bit saves 194 against 282); 4097 forward 199 against 288, backward 370 against 402; fp32 4352 196 against
// 232, 267 against 271.  The other way round in fp32 off alignment, backward: 4097, 559 against 475.
template <typename F> void by_stream_shape(int64_t C, F f) {
    const int64_t n = ceil_div(C, 8);
    if (n <= 128) f(StreamShape<128, 1, 6>());
    else if (n <= 256) f(StreamShape<128, 2, 4>());
    else if (n <= 512) f(StreamShape<256, 2, 2>());
    else if (n <= 576) f(StreamShape<288, 2, 2>());
    else if (n <= 1024) f(StreamShape<512, 2, 1>());
    else f(StreamShape<1024, 2, 1>());
}
// CTAs of a stream kernel per SM: as many of `threads` as the registers of min_ctas full ones hold, 13 at most.
template <typename S> int stream_ctas(int threads) {
    const int n = S::min_ctas * S::most / threads;
    return n < 13 ? n : 13;
}
// Stages of a stream kernel's ring: as many as fit beside the parameters with `ctas` on an SM (below 2: not for it).
constexpr int kStreamSmem = 224 * 1024, kStreamOwn = 2048;            // shared memory of an SM; what a CTA needs besides
int stream_stages(int64_t params, int64_t stage, int ctas) {
    const int64_t n = ((int64_t)kStreamSmem / ctas - kStreamOwn - params) / stage;
    return (int)(n < deft::kMaxStages ? n : deft::kMaxStages);
}
// The limit belongs to the kernel, not to the launch: every call sets the same one, the most that any call needs, so that
// no thread lowers it under another's launch.
template <typename K> cudaError_t allow_stream_smem(K kernel) {
    return cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kStreamSmem - kStreamOwn);
}

int check_groups(int64_t T, int64_t groups) {
    if (groups < 1 || T % groups) return fail(DEF_ERR_ARG, "groups must divide T (got %lld groups, %lld rows)", (long long)groups, (long long)T);
    return DEF_OK;
}

// Slices per group that rows are cut into (each: one CTA, and in the backward pass one row of partial sums): about `want`
// in all, at most one per row.
constexpr int64_t kNormParts = 13 * kUsualSms;    // the most in all, which the workspace is sized for
constexpr int64_t kMostCtas = 0x7fffffff;         // of a grid
int64_t norm_parts(int64_t T, int64_t groups, int64_t want) {
    const int64_t rows = T / groups, each = ceil_div(want, groups);
    return rows < each ? rows : each;
}
// A stream kernel pays off from this many rows per slice on.  It against one row per CTA at 1, 2, 3, 4 and 6 rows, us:
//   forward   2048 bf16   11, 11, 11.2, 11.8, 15 against 11, 11, 12.8, 14.9, 21     4096 fp32  11, 13, 15, 19, 27 against 11, 13, 17, 21, 27
//             4097 bf16   12, 15, 19, 22, 29 against 11, 13, 19, 23, 33             1111 fp16  14, 17, 22, 25, 34 against 11, 13, 17, 21, 29
//   backward  512 bf16    21, 21, 23, 26, 27 against 19, 21, 26, 28, 34             4096 bf16  17, 19, 21, 22, 28 against 30, 52, 58, 70, 87
//             4097 bf16   38, 44, 49, 54, 68 against 34, 52, 71, 83, 146            1111 fp16  30, 34, 41, 46, 58 against 25, 33, 40, 50, 79
// Short unaligned rows would rather have a higher bound forward (513 to 1111 columns lose up to 5 us), long ones a lower one
// backward.
constexpr int64_t kStreamRows = 3, kStreamRowsAlignedBackward = 1;

}  // namespace

extern "C" int def_norm_forward(int32_t dtype, int64_t T, int64_t C, const void *h, int64_t ldh, const void *b, int64_t ldb,
                                const float *w_post, const float *gate, int64_t groups, const float *w_pre, float res_scale,
                                float eps, void *h_out, int64_t ldho, void *n_out, int64_t ldn, float *rstd_post, float *rstd_pre,
                                int8_t *b_q, uint8_t *b_e, int8_t *h_q, uint8_t *h_e, int8_t *n_q, uint8_t *n_e, void *cuda_stream) {
    DEF_TRY(check_rows(dtype, T, C, "C"));
    if (C > DEF_NORM_MAX_C) return fail(DEF_ERR_ARG, "C must be at most %d (got %lld)", DEF_NORM_MAX_C, (long long)C);
    if (T == 0) return DEF_OK;
    if (!h || !w_pre || !n_out || !rstd_pre) return fail(DEF_ERR_NULL, "h, w_pre, n_out and rstd_pre must not be NULL");
    if (b && (!w_post || !h_out || !rstd_post)) return fail(DEF_ERR_NULL, "w_post, h_out and rstd_post must not be NULL where b is given");
    if (!b && (w_post || gate || h_out || rstd_post || b_q || b_e))
        return fail(DEF_ERR_ARG, "w_post, gate, h_out, rstd_post, b_q and b_e must be NULL where b is");
    DEF_TRY(check_pair(b_q, b_e, "b"));
    DEF_TRY(check_pair(h_q, h_e, "h"));
    DEF_TRY(check_pair(n_q, n_e, "n"));
    DEF_TRY(check_groups(T, groups));
    if (!(eps >= 0.f) || !(eps <= 1e30f)) return fail(DEF_ERR_ARG, "eps must be a finite number that is not negative");
    DEF_TRY(check_stride(h, ldh, C, T, "h"));
    DEF_TRY(check_stride(b, ldb, C, T, "b"));
    DEF_TRY(check_stride(h_out, ldho, C, T, "h_out"));
    DEF_TRY(check_stride(n_out, ldn, C, T, "n_out"));
    const int es = element_size(dtype);
    const View views[] = {rows_view(h, "h", T, C, ldh, es, false), rows_view(b, "b", T, C, ldb, es, false),
                          floats_view(w_post, "w_post", C, false), floats_view(gate, "gate", groups * C, false), floats_view(w_pre, "w_pre", C, false),
                          rows_view(h_out, "h_out", T, C, ldho, es, true), rows_view(n_out, "n_out", T, C, ldn, es, true),
                          floats_view(rstd_post, "rstd_post", T, true), floats_view(rstd_pre, "rstd_pre", T, true),
                          q_view(b_q, "b_q", T, C, true), e_view(b_e, "b_e", T, C, true), q_view(h_q, "h_q", T, C, true), e_view(h_e, "h_e", T, C, true),
                          q_view(n_q, "n_q", T, C, true), e_view(n_e, "n_e", T, C, true)};
    DEF_TRY(check_views(views, 0, 5));
    if (const int sms = sm_count(); sms < 0) return sms;
    deft::NormForward a;
    a.h = h; a.b = b; a.h_out = h_out; a.n_out = n_out;
    a.ldh = ldh; a.ldb = ldb; a.ldho = ldho; a.ldn = ldn;
    a.w_post = w_post; a.gate = gate; a.w_pre = w_pre; a.rstd_post = rstd_post; a.rstd_pre = rstd_pre;
    a.hb = {b_q, b_e}; a.hh = {h_q, h_e}; a.hn = {n_q, n_e};
    a.T = T; a.C = C; a.rows_per_group = T / groups; a.ldq = q_stride(C); a.lde = e_stride(C);
    a.res_scale = res_scale; a.eps = eps; a.inv_C = 1.f / (float)C;
    const bool aligned_rows = C % 8 == 0 && wide(h, ldh, es) && wide(b, ldb, es) && wide(h_out, ldho, es) && wide(n_out, ldn, es);
    cudaError_t err = cudaSuccess;
    bool streamed = false;
    // Bytes of a row in a stream kernel's ring; parameters are padded to 8 columns there.
    const int64_t slot = aligned_rows ? C * es : ceil_div(C * es, 32) * 32 + 16, padded = ceil_div(C, 8) * 8;
    by_stream_shape(C, [&](auto shape) {
            using S = decltype(shape);
            const int64_t params = (b ? 8 : 4) * padded, stage = (b ? 2 : 1) * slot;
            const int threads = aligned_rows ? S::most : S::threads(C);
            int ctas = stream_ctas<S>(threads), stages = 0;
            while ((stages = stream_stages(params, stage, ctas)) < 2 && ctas > 1) --ctas;
            const int64_t want = (int64_t)ctas * kUsualSms;
            a.parts_per_group = norm_parts(T, groups, want);
            if (stages < 2 || T < want * kStreamRows || groups * a.parts_per_group > kMostCtas) return;
            streamed = true;
            const unsigned grid = (unsigned)(groups * a.parts_per_group);
            const int smem = (int)(params + stages * stage);
            by_dtype(dtype, [&](auto type) {
                using E = decltype(type);
                const auto kernel = aligned_rows ? deft::norm_forward_stream_kernel<E, true, S::most, S::iters, S::min_ctas>
                                                 : deft::norm_forward_stream_kernel<E, false, S::most, S::iters, S::min_ctas>;
                if ((err = allow_stream_smem(kernel)) != cudaSuccess) return;
                kernel<<<grid, threads, smem, (cudaStream_t)cuda_stream>>>(a, stages);
            });
        });
    if (err != cudaSuccess) return cuda_fail(err, "def_norm_forward");
    if (streamed) return launched("def_norm_forward");
    by_dtype(dtype, [&](auto type) {
        by_alignment(aligned_rows, [&](auto aligned) {
            by_row_shape(C, [&](auto shape) {
                using S = decltype(shape);
                const unsigned grid = (unsigned)(T < kMostCtas ? T : kMostCtas);
                deft::norm_forward_kernel<decltype(type), aligned.value, S::most, S::iters><<<grid, S::threads(C), 0, (cudaStream_t)cuda_stream>>>(a);
            });
        });
    });
    return launched("def_norm_forward");
}

extern "C" int def_norm_backward_workspace(int64_t T, int64_t C, int64_t groups, int64_t *bytes_out) {
    if (!bytes_out) return fail(DEF_ERR_NULL, "bytes_out must not be NULL");
    DEF_TRY(check_rows(DEF_DTYPE_F32, T, C, "C"));
    if (C > DEF_NORM_MAX_C) return fail(DEF_ERR_ARG, "C must be at most %d (got %lld)", DEF_NORM_MAX_C, (long long)C);
    DEF_TRY(check_groups(T, groups));
    *bytes_out = groups * norm_parts(T, groups, kNormParts) * 2 * C * (int64_t)sizeof(float);
    return DEF_OK;
}

extern "C" int def_norm_backward(int32_t dtype, int64_t T, int64_t C, const void *dn, int64_t lddn, const void *dh_in, int64_t lddhi,
                                 const void *h, int64_t ldh, const int8_t *h_q, const uint8_t *h_e, const void *b, int64_t ldb,
                                 const int8_t *b_q, const uint8_t *b_e, const float *w_post, const float *gate, int64_t groups,
                                 const float *w_pre, float res_scale, const float *rstd_post, const float *rstd_pre, void *dh,
                                 int64_t lddh, void *db, int64_t lddb, float *dw_post, float *dgate, float *dw_pre, int32_t accumulate,
                                 void *workspace, int64_t workspace_bytes, void *cuda_stream) {
    int64_t need = 0;
    if (!element_size(dtype)) return fail(DEF_ERR_ARG, "dtype must be one of DEF_DTYPE_F32, _BF16, _F16 (got %d)", dtype);
    DEF_TRY(def_norm_backward_workspace(T, C, groups, &need));
    if (T > 0 && groups * norm_parts(T, groups, kNormParts) > kMostCtas) return fail(DEF_ERR_ARG, "groups must be below 2^31 (got %lld)", (long long)groups);
    DEF_TRY(check_pair(h_q, h_e, "h"));
    DEF_TRY(check_pair(b_q, b_e, "b"));
    const bool has_b = b || b_q;
    if (!w_pre || !dw_pre) return fail(DEF_ERR_NULL, "w_pre and dw_pre must not be NULL");
    if (T > 0 && (!dn || (!h && !h_q) || !rstd_pre || !dh)) return fail(DEF_ERR_NULL, "dn, h (or its checkpoint), rstd_pre and dh must not be NULL");
    if ((h && h_q) || (b && b_q)) return fail(DEF_ERR_ARG, "h and b are given as values or as a checkpoint, not both");
    if (has_b && (!w_post || !rstd_post || !db || !dw_post)) return fail(DEF_ERR_NULL, "w_post, rstd_post, db and dw_post must not be NULL where b is given");
    if (has_b && !gate != !dgate) return fail(DEF_ERR_NULL, "gate and dgate must both be given or both be NULL");
    if (!has_b && T > 0 && (w_post || gate || rstd_post || db || dw_post || dgate))
        return fail(DEF_ERR_ARG, "w_post, gate, rstd_post, db, dw_post and dgate must be NULL where b is");
    if (T > 0 && !workspace) return fail(DEF_ERR_NULL, "workspace must not be NULL");
    if (workspace_bytes < need) return fail(DEF_ERR_ARG, "the workspace must have %lld bytes (got %lld)", (long long)need, (long long)workspace_bytes);
    DEF_TRY(check_stride(dn, lddn, C, T, "dn"));
    DEF_TRY(check_stride(dh_in, lddhi, C, T, "dh_in"));
    DEF_TRY(check_stride(h, ldh, C, T, "h"));
    DEF_TRY(check_stride(b, ldb, C, T, "b"));
    DEF_TRY(check_stride(dh, lddh, C, T, "dh"));
    DEF_TRY(check_stride(db, lddb, C, T, "db"));
    const int es = element_size(dtype);
    const View views[] = {rows_view(dn, "dn", T, C, lddn, es, false), rows_view(dh_in, "dh_in", T, C, lddhi, es, false),
                          rows_view(h, "h", T, C, ldh, es, false), rows_view(b, "b", T, C, ldb, es, false),
                          q_view(h_q, "h_q", T, C, false), e_view(h_e, "h_e", T, C, false), q_view(b_q, "b_q", T, C, false), e_view(b_e, "b_e", T, C, false),
                          floats_view(w_post, "w_post", C, false), floats_view(gate, "gate", groups * C, false), floats_view(w_pre, "w_pre", C, false),
                          floats_view(rstd_post, "rstd_post", T, false), floats_view(rstd_pre, "rstd_pre", T, false),
                          rows_view(dh, "dh", T, C, lddh, es, true), rows_view(db, "db", T, C, lddb, es, true),
                          floats_view(dw_post, "dw_post", C, true), floats_view(dgate, "dgate", groups * C, true), floats_view(dw_pre, "dw_pre", C, true),
                          {workspace, "workspace", workspace ? 1 : 0, need, need, 16, true}};
    DEF_TRY(check_views(views, 1, 13));
    if (const int sms = sm_count(); sms < 0) return sms;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (T == 0) {
        cudaError_t err = cudaSuccess;
        if (!accumulate) {
            err = cudaMemsetAsync(dw_pre, 0, (size_t)C * 4, stream);
            if (err == cudaSuccess && dw_post) err = cudaMemsetAsync(dw_post, 0, (size_t)C * 4, stream);
            if (err == cudaSuccess && dgate) err = cudaMemsetAsync(dgate, 0, (size_t)(groups * C) * 4, stream);
        }
        return err == cudaSuccess ? DEF_OK : cuda_fail(err, "def_norm_backward");
    }
    deft::NormBackward a;
    a.dn = dn; a.dh_in = dh_in; a.h = h; a.b = b; a.hh = {h_q, h_e}; a.hb = {b_q, b_e}; a.dh = dh; a.db = db;
    a.lddn = lddn; a.lddhi = lddhi; a.ldh = ldh; a.ldb = ldb; a.lddh = lddh; a.lddb = lddb;
    a.w_post = w_post; a.gate = gate; a.w_pre = w_pre; a.rstd_post = rstd_post; a.rstd_pre = rstd_pre;
    a.partial = (float *)workspace;
    a.T = T; a.C = C; a.rows_per_group = T / groups; a.ldq = q_stride(C); a.lde = e_stride(C);
    a.res_scale = res_scale; a.inv_C = 1.f / (float)C;
    const bool aligned_rows = C % 8 == 0 && wide(dn, lddn, es) && wide(dh_in, lddhi, es) && wide(h, ldh, es) && wide(b, ldb, es) && wide(dh, lddh, es) && wide(db, lddb, es);
    a.ring_e = wide(h_e, a.lde, 1) && wide(b_e, a.lde, 1);           // bulk copies start on 16-byte boundaries
    cudaError_t err = cudaSuccess;
    bool streamed = false;
    const int64_t slot = aligned_rows ? C * es : ceil_div(C * es, 32) * 32 + 16, padded = ceil_div(C, 8) * 8;
    by_stream_shape(C, [&](auto shape) {
            using S = decltype(shape);
            const int64_t params = (has_b ? 8 : 4) * padded;
            const int64_t held = a.ldq + (a.ring_e ? a.lde : 0);
            const int64_t stage = slot * (dh_in ? 2 : 1) + (h_q ? held : slot) + (!has_b ? 0 : b_q ? held : slot);
            const int threads = aligned_rows ? S::most : S::threads(C);
            int ctas = stream_ctas<S>(threads), stages = 0;
            while ((stages = stream_stages(params, stage, ctas)) < 2 && ctas > 1) --ctas;
            const int64_t want = (int64_t)ctas * kUsualSms;
            if (stages < 2 || T < want * (aligned_rows ? kStreamRowsAlignedBackward : kStreamRows) || (has_b && !h_q != !b_q)) return;
            streamed = true;
            a.parts_per_group = norm_parts(T, groups, want);
            const int smem = (int)(params + stages * stage);
            by_dtype(dtype, [&](auto type) {
                using E = decltype(type);
                const auto pick = [&](auto aligned) {
                    return h_q ? deft::norm_backward_stream_kernel<E, aligned.value, S::most, S::iters, S::min_ctas, true>
                               : deft::norm_backward_stream_kernel<E, aligned.value, S::most, S::iters, S::min_ctas, false>;
                };
                const auto kernel = aligned_rows ? pick(Is<true>()) : pick(Is<false>());
                if ((err = allow_stream_smem(kernel)) != cudaSuccess) return;
                kernel<<<(unsigned)(groups * a.parts_per_group), threads, smem, stream>>>(a, stages);
            });
        });
    if (err != cudaSuccess) return cuda_fail(err, "def_norm_backward");
    if (!streamed)
        by_dtype(dtype, [&](auto type) {
            by_alignment(aligned_rows, [&](auto aligned) {
                by_row_shape(C, [&](auto shape) {
                    using S = decltype(shape);
                    // 4, 3 or 1 CTAs per SM.  At 1, 2, 3, 4, 6 of them, us: 1500 x 513 fp16 (96 threads) 40, 28, 25, 23, 26; 1000 x 257
                    // bf16 (64) 28, 21, 20, 19, 21; 1533 x 1111 fp16 (160) 46, 32, 30, 40, 38; 1533 x 1001 bf16 (128) 44, 32,
                    // 28, 28, 36; 400 x 4097 bf16 (288) 42, 58, 58, 58, 58; 300 x 8191 bf16 (512) 61, 88, 84, 85, 85.  The
                    // exception: 800 x 2047 bf16 (256) 34, 30, 40, 42, 48.
                    a.parts_per_group = norm_parts(T, groups, S::threads(C) <= 128 ? 4 * kUsualSms : S::threads(C) <= 256 ? 3 * kUsualSms : kUsualSms);
                    deft::norm_backward_kernel<decltype(type), aligned.value, S::most, S::iters><<<(unsigned)(groups * a.parts_per_group), S::threads(C), 0, stream>>>(a);
                });
            });
        });
    DEF_TRY(launched("def_norm_backward"));
    // The sums' kernel may be set up while the other still runs; it waits for it before it reads.
    const int64_t jobs_gate = gate ? groups : 0, jobs = jobs_gate + (has_b ? 2 : 1);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)ceil_div(C, 32), (unsigned)(jobs < 1024 ? jobs : 1024));
    cfg.blockDim = C % 4 == 0 ? dim3(8, 32) : dim3(32, 32);
    cfg.stream = stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
    attr[0].val.programmaticStreamSerializationAllowed = 1;
    cfg.attrs = attr;
    cfg.numAttrs = 1;
    err = cudaLaunchKernelEx(&cfg, C % 4 == 0 ? deft::norm_reduce_kernel<4> : deft::norm_reduce_kernel<1>, (const float *)workspace, w_post, gate, (int)C, groups, a.parts_per_group, jobs_gate, (int)accumulate,
                             has_b ? dw_post : (float *)nullptr, dgate, dw_pre);
    if (err != cudaSuccess) {
        cudaGetLastError();
        return cuda_fail(err, "def_norm_backward (sums)");
    }
    return DEF_OK;
}

// ---------------------------------------------------------------------------
// Weight gradient
// ---------------------------------------------------------------------------
namespace {

// What a call launches and keeps in its workspace: partial tiles first, then the 16-bit pieces of dy, then x^ in 16 bits.
struct GradPlan {
    bool copy_dy, copy_x;
    int planes, pairs;
    int64_t ld_dy, ld_planes, ld_x, partial_bytes, plane_bytes, x_bytes;
    int64_t tiles_i, tiles_o, blocks, whole;
};
GradPlan grad_plan(int32_t dtype, int64_t T, int64_t O, int64_t I, const void *dy, int64_t lddy, int sms) {
    GradPlan p;
    const int es = element_size(dtype);
    // One row has no stride; rows that a tensor map cannot reach (its strides end at 2^40 bytes) are copied like unaligned ones.
    p.ld_dy = T > 1 ? lddy : ceil_div(O, 8) * 8;
    p.copy_dy = es == 4 || !wide(dy, p.ld_dy, es) || p.ld_dy >= ((int64_t)1 << 40) / es;
    p.planes = es == 4 ? 3 : 1;
    p.ld_planes = ceil_div(O, 8) * 8;
    p.ld_x = ceil_div(I, 8) * 8;
    p.plane_bytes = p.copy_dy ? p.planes * T * p.ld_planes * 2 : 0;
    p.tiles_i = ceil_div(I, deft::kPairI);
    p.tiles_o = ceil_div(O, deft::kTileO);
    p.blocks = ceil_div(T, deft::kTileT);
    // A pair of CTAs per pair of SMs.  Rounds of whole tiles; the tiles of a last round that would leave a tenth of the
    // pairs idle or more are cut by tokens into equal runs instead, which costs a pass over their partial sums.  Whole against
    // cut, 8192 tokens, I = 4096, bf16, us: 16 tiles of a round of 74 66 against 29, 32 67 against 44, 48 67 against 58, 64
    // 68 against 73; a round and 6 tiles 131 against 82, one and 54 129 against 128, two and 12 223 against 171.  The partial sums
    // weigh more where tokens are few, and a tenth is then too little: 64 tiles of 512 tokens 19 against 33.
    const int64_t tiles = p.tiles_i * p.tiles_o, workers = sms / 2, rest = tiles % workers, per_tile = p.blocks * p.planes;
    p.whole = rest * 10 >= workers * 9 || per_tile == 1 ? tiles : tiles - rest;
    const int64_t most = p.whole == 0 ? tiles * per_tile : tiles;
    p.pairs = (int)(most < workers ? most : workers);
    p.partial_bytes = p.whole < tiles ? (int64_t)p.pairs * 4 * deft::kTileO * deft::kTileI * 4 : 0;
    // A tile of x^ is widened once for each tile of dw along o (and each piece of dy).  From kWidenOnce of them on it is
    // cheaper to widen x^ to memory first, as long as that keeps to the documented size of the workspace.
    p.x_bytes = T * p.ld_x * 2;
    p.copy_x = p.tiles_o * p.planes >= deft::kWidenOnce &&
               p.partial_bytes + p.plane_bytes + p.x_bytes <= ((int64_t)68 << 20) + 8 * O * I + 6 * T * O;
    if (!p.copy_x) p.x_bytes = 0;
    return p;
}

// The driver's entry point for tensor maps, found at run time: the library itself does not link the driver.
using EncodeTiled = CUresult (*)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *,
                                 const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave, CUtensorMapSwizzle, CUtensorMapL2promotion,
                                 CUtensorMapFloatOOBfill);
EncodeTiled encode_tiled() {
    static std::atomic<void *> known{nullptr};
    void *f = known.load();
    if (f) return (EncodeTiled)f;
    cudaDriverEntryPointQueryResult found;
    if (cudaGetDriverEntryPointByVersion("cuTensorMapEncodeTiled", &f, 12000, cudaEnableDefault, &found) != cudaSuccess ||
        found != cudaDriverEntryPointSuccess)
        return nullptr;
    known.store(f);
    return (EncodeTiled)f;
}

}  // namespace

extern "C" int def_checkpoint_weight_grad_workspace(int32_t dtype, int64_t T, int64_t O, int64_t I, const void *dy, int64_t lddy,
                                                    int64_t *bytes_out) {
    if (!bytes_out) return fail(DEF_ERR_NULL, "bytes_out must not be NULL");
    DEF_TRY(check_rows(dtype, T, O, "O"));
    DEF_TRY(check_rows(dtype, T, I, "I"));
    DEF_TRY(check_stride(dy, lddy, O, T, "dy"));
    if (T >= (int64_t)1 << 31) return fail(DEF_ERR_ARG, "T must be below 2^31 (got %lld)", (long long)T);
    const GradPlan p = grad_plan(dtype, T, O, I, dy, lddy, kUsualSms);
    *bytes_out = p.partial_bytes + p.plane_bytes + p.x_bytes;
    return DEF_OK;
}

extern "C" int def_checkpoint_weight_grad(int32_t dtype, int64_t T, int64_t O, int64_t I, const void *dy, int64_t lddy, const int8_t *q,
                                          const uint8_t *e, float *dw, int32_t accumulate, void *workspace, int64_t workspace_bytes,
                                          void *cuda_stream) {
    int64_t need = 0;
    DEF_TRY(def_checkpoint_weight_grad_workspace(dtype, T, O, I, dy, lddy, &need));
    if (!dw || (T > 0 && (!dy || !q || !e))) return fail(DEF_ERR_NULL, "dy, q, e and dw must not be NULL");
    if (need > 0 && !workspace) return fail(DEF_ERR_NULL, "workspace must not be NULL");
    if (workspace_bytes < need) return fail(DEF_ERR_ARG, "the workspace must have %lld bytes (got %lld)", (long long)need, (long long)workspace_bytes);
    const int es = element_size(dtype);
    const View views[] = {rows_view(dy, "dy", T, O, lddy, es, false), q_view(q, "q", T, I, false), e_view(e, "e", T, I, false),
                          floats_view(dw, "dw", O * I, true), {workspace, "workspace", need > 0 ? 1 : 0, need, need, 16, true}};
    DEF_TRY(check_views(views));
    if (const int sms = sm_count(); sms < 0) return sms;
    const cudaStream_t stream = (cudaStream_t)cuda_stream;
    if (T == 0) {
        if (accumulate) return DEF_OK;
        const cudaError_t err = cudaMemsetAsync(dw, 0, (size_t)(O * I) * 4, stream);
        return err == cudaSuccess ? DEF_OK : cuda_fail(err, "def_checkpoint_weight_grad");
    }
    const EncodeTiled encode = encode_tiled();
    if (!encode) return fail(DEF_ERR_CUDA, "the driver does not offer tensor maps");
    // The plan the workspace was sized by, on as many CTAs.
    GradPlan p = grad_plan(dtype, T, O, I, dy, lddy, kUsualSms);
    const bool half = dtype == DEF_DTYPE_F16;
    uint4 *planes = (uint4 *)((char *)workspace + p.partial_bytes);
    void *wide_x = (char *)workspace + p.partial_bytes + p.plane_bytes;
    const void *rows = p.copy_dy ? planes : dy, *xs = p.copy_x ? wide_x : (const void *)q;
    const int64_t ld = p.copy_dy ? p.ld_planes : p.ld_dy;
    // The maps first: nothing is launched where the driver refuses one.
    CUtensorMap map_y, map_x, map_e = {};
    const cuuint64_t dim_y[3] = {(cuuint64_t)O, (cuuint64_t)T, (cuuint64_t)p.planes}, stride_y[2] = {(cuuint64_t)ld * 2, (cuuint64_t)ld * 2 * (cuuint64_t)(p.planes > 1 ? T : 1)};
    const cuuint32_t box_y[3] = {64, deft::kTileT, 1}, one[3] = {1, 1, 1};
    const cuuint64_t dim_x[2] = {(cuuint64_t)I, (cuuint64_t)T}, stride_x[1] = {(cuuint64_t)(p.copy_x ? p.ld_x * 2 : q_stride(I))};
    const cuuint32_t box_x[2] = {p.copy_x ? 64u : (cuuint32_t)deft::kTileI, deft::kTileT};
    const CUtensorMapDataType type16 = half ? CU_TENSOR_MAP_DATA_TYPE_FLOAT16 : CU_TENSOR_MAP_DATA_TYPE_BFLOAT16;
    if (encode(&map_y, type16, 3, const_cast<void *>(rows), dim_y, stride_y, box_y, one, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
               CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS ||
        encode(&map_x, p.copy_x ? type16 : CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<void *>(xs), dim_x, stride_x, box_x, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
               p.copy_x ? CU_TENSOR_MAP_SWIZZLE_128B : CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B,
               CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
        return fail(DEF_ERR_CUDA, "the driver refused a tensor map of dy or x");
    const bool wide_e = !p.copy_x && e_stride(I) % 16 == 0 && ((uintptr_t)e & 15u) == 0;
    if (wide_e) {
        const cuuint64_t dim_e[2] = {(cuuint64_t)e_stride(I), (cuuint64_t)T}, stride_e[1] = {(cuuint64_t)e_stride(I)};
        const cuuint32_t box_e[2] = {16, deft::kTileT};
        if (encode(&map_e, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<uint8_t *>(e), dim_e, stride_e, box_e, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                   CU_TENSOR_MAP_SWIZZLE_NONE, CU_TENSOR_MAP_L2_PROMOTION_L2_128B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) != CUDA_SUCCESS)
            return fail(DEF_ERR_CUDA, "the driver refused a tensor map of e");
    }
    if (p.copy_dy) {
        on_plane(false, T, O, [&](auto, dim3 grid, dim3 block) {
            if (es == 4) deft::weight_grad_planes_kernel<float><<<grid, block, 0, stream>>>((const float *)dy, lddy, T, (int)O, planes, p.ld_planes);
            else deft::weight_grad_planes_kernel<__half><<<grid, block, 0, stream>>>((const __half *)dy, lddy, T, (int)O, planes, p.ld_planes);
        });
        DEF_TRY(launched("def_checkpoint_weight_grad (copy)"));
    }
    if (p.copy_x) {
        on_plane(I % 8 == 0, T, I, [&](auto v, dim3 grid, dim3 block) {
            if (half)
                deft::unpack_kernel<__half, v.value><<<grid, block, 0, stream>>>(q, e, q_stride(I), e_stride(I), T, (int)I, (__half *)wide_x, p.ld_x);
            else
                deft::unpack_kernel<__nv_bfloat16, v.value><<<grid, block, 0, stream>>>(q, e, q_stride(I), e_stride(I), T, (int)I, (__nv_bfloat16 *)wide_x, p.ld_x);
        });
        DEF_TRY(launched("def_checkpoint_weight_grad (widen)"));
    }
    deft::WeightGrad a = {e, dw, (float *)workspace, T, O, I, e_stride(I), (int)p.tiles_i, (int)p.tiles_o, (int)p.blocks, p.planes, accumulate, p.whole};
    cudaError_t err = cudaSuccess;
    auto launch = [&](auto kernel, auto shape) {
        using S = decltype(shape);
        if ((err = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, S::smem)) != cudaSuccess) return;
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)p.pairs * 2);
        cfg.blockDim = dim3(S::threads);
        cfg.dynamicSmemBytes = S::smem;
        cfg.stream = stream;
        cudaLaunchAttribute attr[2];
        attr[0].id = cudaLaunchAttributeClusterDimension;
        attr[0].val.clusterDim.x = 2;
        attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
        attr[1].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[1].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 2;
        err = cudaLaunchKernelEx(&cfg, kernel, a, map_y, map_x, map_e);
    };
    auto by_operand = [&](auto type) {
        using E = decltype(type);
        if (p.copy_x) launch(deft::weight_grad_kernel<E, false, false>, deft::GradShape<false>());
        else if (wide_e) launch(deft::weight_grad_kernel<E, true, true>, deft::GradShape<true>());
        else launch(deft::weight_grad_kernel<E, true, false>, deft::GradShape<true>());
    };
    if (half) by_operand(__half());
    else by_operand(__nv_bfloat16());
    if (err != cudaSuccess) {
        cudaGetLastError();
        return cuda_fail(err, "def_checkpoint_weight_grad");
    }
    if (const int64_t cut = p.tiles_i * p.tiles_o - p.whole; cut > 0) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3((unsigned)(cut * 2 * (deft::kTileO / 8)));
        cfg.blockDim = dim3(256);
        cfg.stream = stream;
        cudaLaunchAttribute attr[1];
        attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[0].val.programmaticStreamSerializationAllowed = 1;
        cfg.attrs = attr;
        cfg.numAttrs = 1;
        if ((err = cudaLaunchKernelEx(&cfg, deft::weight_grad_join_kernel, a, p.pairs)) != cudaSuccess) {
            cudaGetLastError();
            return cuda_fail(err, "def_checkpoint_weight_grad (join)");
        }
    }
    return DEF_OK;
}

// ---------------------------------------------------------------------------
// Log probabilities
// ---------------------------------------------------------------------------
namespace {
constexpr int64_t kLogprobNarrow = 24576;  // rows up to this go to CTAs of 128 threads, longer ones to CTAs of 512 (8192 rows of 20000:
                                           // 68 against 99 us; of 32000 fp32, top = 8: 203 against 186)
// Least columns per CTA of a row that is cut, and what cutting gives, us: one row of 128000 bf16 forward 11.2 against 15.1 whole,
// backward 8.2 against 12.3; 64 such rows 14.4 against 16.6, 8.3 against 14.4; one row of 20000 10.3 and 8.1 either way; 16
// rows of 50001 bf16 12.3 against 10.3, 8.2 either way.
constexpr int64_t kLogprobLeast = 4096;
}  // namespace

extern "C" int def_logprob_forward(int32_t dtype, int64_t T, int64_t V, const void *logits, int64_t ldx, const int64_t *targets,
                                   float *logp, float *entropy, float *lse, int32_t top, int64_t *top_ids, float *top_logp,
                                   void *cuda_stream) {
    DEF_TRY(check_rows(dtype, T, V, "V"));
    if (top < 0 || top > DEF_LOGPROB_MAX_TOP || top > V) return fail(DEF_ERR_ARG, "top must be in [0, min(V, %d)] (got %d)", DEF_LOGPROB_MAX_TOP, top);
    if (T == 0) return DEF_OK;
    if (!logits || !targets || !logp || !entropy || !lse) return fail(DEF_ERR_NULL, "logits, targets, logp, entropy and lse must not be NULL");
    if ((top > 0) != (top_ids != nullptr) || (top > 0) != (top_logp != nullptr)) return fail(DEF_ERR_NULL, "top_ids and top_logp must be given if and only if top > 0");
    DEF_TRY(check_stride(logits, ldx, V, T, "logits"));
    const int es = element_size(dtype);
    const View views[] = {rows_view(logits, "logits", T, V, ldx, es, false), {targets, "targets", 1, T * 8, T * 8, 8, false},
                          floats_view(logp, "logp", T, true), floats_view(entropy, "entropy", T, true), floats_view(lse, "lse", 2 * T, true),
                          {top_ids, "top_ids", top_ids ? 1 : 0, T * top * 8, T * top * 8, 8, true}, floats_view(top_logp, "top_logp", T * top, true)};
    DEF_TRY(check_views(views));
    if (const int sms = sm_count(); sms < 0) return sms;
    deft::LogprobForward a = {logits, ldx, T, V, targets, logp, entropy, lse, top_ids, top_logp, top};
    // A row is cut over up to 8 CTAs while that leaves each SM no more than one and each CTA kLogprobLeast elements.
    const bool narrow = V <= kLogprobNarrow;
    int split = 1;
    while (split < 8 && T * split * 2 <= kUsualSms && V >= kLogprobLeast * split * 2) split *= 2;
    if (T * split > 0x7fffffff) return fail(DEF_ERR_ARG, "T is too large (got %lld)", (long long)T);
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(T * split));
    cfg.blockDim = dim3(narrow ? 128 : 512);
    cfg.stream = (cudaStream_t)cuda_stream;
    cudaLaunchAttribute attr[1];
    attr[0].id = cudaLaunchAttributeClusterDimension;
    attr[0].val.clusterDim.x = (unsigned)split;
    attr[0].val.clusterDim.y = attr[0].val.clusterDim.z = 1;
    cfg.attrs = attr;
    cfg.numAttrs = split > 1 ? 1 : 0;
    cudaError_t err = cudaSuccess;
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        err = narrow ? cudaLaunchKernelEx(&cfg, deft::logprob_forward_kernel<E, 128>, a, split) : cudaLaunchKernelEx(&cfg, deft::logprob_forward_kernel<E, 512>, a, split);
    });
    if (err != cudaSuccess) {
        cudaGetLastError();
        return cuda_fail(err, "def_logprob_forward");
    }
    return DEF_OK;
}

extern "C" int def_logprob_backward(int32_t dtype, int64_t T, int64_t V, const void *logits, int64_t ldx, const int64_t *targets,
                                    const float *lse, const float *entropy, const float *dlogp, const float *dentropy, int32_t top,
                                    const int64_t *top_ids, const float *dtop_logp, void *dlogits, int64_t lddx, void *cuda_stream) {
    DEF_TRY(check_rows(dtype, T, V, "V"));
    if (top < 0 || top > DEF_LOGPROB_MAX_TOP || top > V) return fail(DEF_ERR_ARG, "top must be in [0, min(V, %d)] (got %d)", DEF_LOGPROB_MAX_TOP, top);
    if (T == 0) return DEF_OK;
    if (!logits || !targets || !lse || !entropy || !dlogits) return fail(DEF_ERR_NULL, "logits, targets, lse, entropy and dlogits must not be NULL");
    if ((top > 0) != (top_ids != nullptr) || (top > 0) != (dtop_logp != nullptr)) return fail(DEF_ERR_NULL, "top_ids and dtop_logp must be given if and only if top > 0");
    DEF_TRY(check_stride(logits, ldx, V, T, "logits"));
    DEF_TRY(check_stride(dlogits, lddx, V, T, "dlogits"));
    const int es = element_size(dtype);
    const View views[] = {rows_view(logits, "logits", T, V, ldx, es, false), rows_view(dlogits, "dlogits", T, V, lddx, es, true),
                          {targets, "targets", 1, T * 8, T * 8, 8, false}, floats_view(lse, "lse", 2 * T, false), floats_view(entropy, "entropy", T, false),
                          floats_view(dlogp, "dlogp", T, false), floats_view(dentropy, "dentropy", T, false),
                          {top_ids, "top_ids", top_ids ? 1 : 0, T * top * 8, T * top * 8, 8, false}, floats_view(dtop_logp, "dtop_logp", T * top, false)};
    DEF_TRY(check_views(views, 0, 1));
    if (const int sms = sm_count(); sms < 0) return sms;
    deft::LogprobBackward a = {logits, dlogits, ldx, lddx, T, V, targets, top_ids, lse, entropy, dlogp, dentropy, dtop_logp, top};
    const bool narrow = V <= kLogprobNarrow;
    int split = 1;
    while (split < 8 && T * split * 2 <= 2 * kUsualSms && V >= kLogprobLeast * split * 2) split *= 2;
    if (T * split > 0x7fffffff) return fail(DEF_ERR_ARG, "T is too large (got %lld)", (long long)T);
    by_dtype(dtype, [&](auto type) {
        using E = decltype(type);
        const unsigned grid = (unsigned)(T * split);
        if (narrow) deft::logprob_backward_kernel<E, 128><<<grid, 128, 0, (cudaStream_t)cuda_stream>>>(a, split);
        else deft::logprob_backward_kernel<E, 512><<<grid, 512, 0, (cudaStream_t)cuda_stream>>>(a, split);
    });
    return launched("def_logprob_backward");
}
