// What the kernels around the step share: element types, 8-element accesses, reductions, and the 8-bit
// checkpoint's group of 32 columns.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace deft {

constexpr int kGroup = 32;            // columns of a row that share one exponent (DEF_CHECKPOINT_GROUP)

template <typename T> __device__ __forceinline__ float to_float(T v);
template <> __device__ __forceinline__ float to_float(float v) { return v; }
template <> __device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
template <> __device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float(float v) { return v; }
template <> __device__ __forceinline__ __nv_bfloat16 from_float(float v) { return __float2bfloat16_rn(v); }
template <> __device__ __forceinline__ __half from_float(float v) { return __float2half_rn(v); }

// V consecutive elements as they lie in memory: V = 8 on 16-byte aligned rows, V = 1 on others.
template <typename T, int V> struct alignas(V == 1 ? sizeof(T) : 16) Frag { T v[V]; };

// Streams that are read once bypass the L1, which is left to what CTAs share (weights).
template <typename T, int V> __device__ __forceinline__ Frag<T, V> load_frag(const T *p) {
    Frag<T, V> f;
    if constexpr (V == 1) {
        f.v[0] = *p;
    } else {
        static_assert(V == 8, "");
        constexpr int kWords = sizeof(T) * V / 16;
        uint4 w[kWords];
#pragma unroll
        for (int i = 0; i < kWords; ++i)
            asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                         : "=r"(w[i].x), "=r"(w[i].y), "=r"(w[i].z), "=r"(w[i].w)
                         : "l"(reinterpret_cast<const uint4 *>(p) + i));
        memcpy(&f, w, sizeof(f));
    }
    return f;
}
template <typename T, int V> __device__ __forceinline__ void to_floats(const Frag<T, V> &f, float (&out)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = to_float<T>(f.v[i]);
}
template <typename T, int V> __device__ __forceinline__ void load_floats(const T *p, float (&out)[V]) {
    to_floats<T, V>(load_frag<T, V>(p), out);
}
template <typename T, int V> __device__ __forceinline__ void store_floats(T *p, const float (&in)[V]) {
    Frag<T, V> f;
#pragma unroll
    for (int i = 0; i < V; ++i) f.v[i] = from_float<T>(in[i]);
    if constexpr (V == 1) {
        *p = f.v[0];
    } else {
        constexpr int kWords = sizeof(T) * V / 16;
        uint4 w[kWords];
        memcpy(w, &f, sizeof(f));
#pragma unroll
        for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4 *>(p)[i] = w[i];
    }
}
// fp32 parameters, read by every row: cached.
template <int V> __device__ __forceinline__ void load_params(const float *p, float (&out)[V]) {
    if constexpr (V == 1) {
        out[0] = __ldg(p);
    } else if ((reinterpret_cast<uintptr_t>(p) & 15u) == 0) {   // the same for all threads
#pragma unroll
        for (int i = 0; i < V / 4; ++i) {
            const float4 t = __ldg(reinterpret_cast<const float4 *>(p) + i);
            out[4 * i] = t.x; out[4 * i + 1] = t.y; out[4 * i + 2] = t.z; out[4 * i + 3] = t.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) out[i] = __ldg(p + i);
    }
}

// ---------------------------------------------------------------------------
// Checkpoint group: 32 consecutive columns of a row, held by 32 / V consecutive lanes of a warp (V columns each).
// k = max(floor(log2 amax) - 6, -126) is read off the exponent bits of amax: the steps are powers of two, so x 2^-k
// is exact and the only rounding is the one to an integer; q 2^k has at most 7 bits of magnitude and is exact in
// bf16 and fp32.
// ---------------------------------------------------------------------------
template <int V> __device__ __forceinline__ uint32_t group_exponent(const float (&x)[V]) {
    // Magnitudes as integers: ordered like the magnitudes, and an infinity or NaN (>= 0x7f800000) wins.
    uint32_t top = 0;
#pragma unroll
    for (int i = 0; i < V; ++i) top = max(top, __float_as_uint(x[i]) & 0x7fffffffu);
#pragma unroll
    for (int s = 1; s < kGroup / V; s <<= 1) top = max(top, __shfl_xor_sync(0xffffffffu, top, s));
    const int biased = (int)(top >> 23);            // floor(log2 amax) + 127; 0 for zero and subnormals
    return biased == 255 ? 255u : (uint32_t)max(biased - 6, 1);
}
template <int V> __device__ __forceinline__ void quantise(const float (&x)[V], uint32_t e, int8_t (&q)[V]) {
    const float inv = e == 255 ? 0.f : __uint_as_float((254u - e) << 23);   // 2^-k, e in [1, 248]
#pragma unroll
    for (int i = 0; i < V; ++i) {
        const int r = e == 255 ? 0 : __float2int_rn(x[i] * inv);
        q[i] = (int8_t)max(-127, min(127, r));
    }
}
// 2^k; +infinity for e = 255, which makes q e NaN because q is 0 there.
__device__ __forceinline__ float group_scale(uint32_t e) { return __uint_as_float(e << 23); }

template <int V> __device__ __forceinline__ void store_q(int8_t *p, const int8_t (&q)[V]) {
    if constexpr (V == 1) {
        *p = q[0];
    } else {
        uint2 w;
        memcpy(&w, q, sizeof(w));
        *reinterpret_cast<uint2 *>(p) = w;
    }
}
template <int V> __device__ __forceinline__ void load_held(const int8_t *q, const uint8_t *e, int64_t col, float (&x)[V]) {
    int8_t v[V];
    if constexpr (V == 1) {
        v[0] = q[col];
    } else {
        uint2 w;
        asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(w.x), "=r"(w.y) : "l"(q + col));
        memcpy(v, &w, sizeof(w));
    }
    const float scale = group_scale(e[col / kGroup]);
#pragma unroll
    for (int i = 0; i < V; ++i) x[i] = (float)v[i] * scale;
}

// Writes the checkpoint of V columns at `col`; every lane of the warp calls it, `valid` where the columns exist
// (the others pass zeros).
template <int V>
__device__ __forceinline__ void store_held(int8_t *q, uint8_t *e, int64_t col, bool valid, const float (&x)[V]) {
    const uint32_t ex = group_exponent<V>(x);
    int8_t v[V];
    quantise<V>(x, ex, v);
    if (valid) {
        store_q<V>(q + col, v);
        if (col % kGroup == 0) e[col / kGroup] = (uint8_t)ex;
    }
}

// ---------------------------------------------------------------------------
// Sums over a CTA.  `scratch` has room for one value per warp and is not reused by the caller before its next
// __syncthreads().
// ---------------------------------------------------------------------------
__device__ __forceinline__ float warp_sum(float v) {
#pragma unroll
    for (int s = 16; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    return v;
}
template <int THREADS> __device__ __forceinline__ float cta_sum(float v, float *scratch) {
    v = warp_sum(v);
    if constexpr (THREADS == 32) return v;
    constexpr int kWarps = THREADS / 32;
    if ((threadIdx.x & 31) == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = (threadIdx.x & 31) < kWarps ? scratch[threadIdx.x & 31] : 0.f;
#pragma unroll
    for (int s = kWarps / 2; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
    return kWarps == 32 ? v : __shfl_sync(0xffffffffu, v, 0);
}

}  // namespace deft
