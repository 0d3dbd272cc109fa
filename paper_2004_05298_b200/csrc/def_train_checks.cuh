// What the C entry points of the operators around the step share: argument checks, views, launch shapes, tensor maps.
#pragma once

#include <atomic>
#include <cstring>

#include <cuda.h>

#include "../../include/def_train.h"
#include "def_error.cuh"
#include "def_train_common.cuh"

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

// A kernel's limit of dynamic shared memory, raised once per kernel and device (every call of a kernel asks for the same).  K is the
// kernel itself, so that each has a record of its own.
template <auto K> cudaError_t allow_smem(int bytes) {
    static std::atomic<uint64_t> raised{0};
    static_assert(kMaxDevices <= 64);
    int dev = 0;
    cudaError_t err = cudaGetDevice(&dev);
    if (err != cudaSuccess || (raised.load(std::memory_order_acquire) >> dev & 1)) return err;
    if ((err = cudaFuncSetAttribute(K, cudaFuncAttributeMaxDynamicSharedMemorySize, bytes)) == cudaSuccess) raised.fetch_or((uint64_t)1 << dev, std::memory_order_release);
    return err;
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
