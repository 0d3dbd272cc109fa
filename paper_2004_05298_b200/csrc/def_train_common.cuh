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
template <typename T, int V> __device__ __forceinline__ Frag<T, V> zeros() {
    Frag<T, V> f;
    memset(&f, 0, sizeof(f));
    return f;
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

// Two fp32 operations in one instruction.
struct Pair { uint64_t bits; };
__device__ __forceinline__ Pair make_pair(float a, float b) {
    Pair p;
    asm("mov.b64 %0, {%1, %2};" : "=l"(p.bits) : "f"(a), "f"(b));
    return p;
}
__device__ __forceinline__ void split_pair(Pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p.bits)); }
__device__ __forceinline__ Pair pair_fma(Pair a, Pair b, Pair c) {
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d.bits) : "l"(a.bits), "l"(b.bits), "l"(c.bits));
    return d;
}
__device__ __forceinline__ Pair pair_add(Pair a, Pair b) {
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d.bits) : "l"(a.bits), "l"(b.bits));
    return d;
}
__device__ __forceinline__ Pair pair_mul(Pair a, Pair b) {
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.bits) : "l"(a.bits), "l"(b.bits));
    return d;
}
__device__ __forceinline__ Pair both(float a) { return make_pair(a, a); }
// ---------------------------------------------------------------------------
// Checkpoint group: 32 consecutive columns of a row, held by 32 / V consecutive lanes of a warp (V columns each).
// k = max(floor(log2 amax) - 6, -126) is read off the exponent bits of amax: the steps are powers of two, so x 2^-k
// is exact and the only rounding is the one to an integer; q 2^k has at most 7 bits of magnitude and is exact in
// bf16 and fp32.
// ---------------------------------------------------------------------------
__device__ __forceinline__ float max_nan(float a, float b) {       // keeps a NaN (fmaxf drops it)
    float y;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}
// Bits of the group's largest magnitude; at least 0x7f800000 if it holds an infinity or a NaN.
template <int V> __device__ __forceinline__ uint32_t group_top(float top) {
    uint32_t bits = __float_as_uint(top) & 0x7fffffffu;
#pragma unroll
    for (int s = 1; s < kGroup / V; s <<= 1) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, s));
    return bits;
}
template <int V> __device__ __forceinline__ uint32_t group_top(const float (&x)[V]) {
    float top = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < V; ++i) top = max_nan(top, fabsf(x[i]));
    return group_top<V>(top);
}
// The same from 16-bit values as loaded: magnitudes of either type order like the integers they are held in.
template <typename T, int V> __device__ __forceinline__ uint32_t group_top(const Frag<T, V> &f) {
    if constexpr (sizeof(T) == 2 && V == 8) {
        uint32_t w[4];
        memcpy(w, &f, sizeof(w));
        const uint32_t m = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
        const uint16_t top = (uint16_t)max(m & 0xffffu, m >> 16);
        T t;
        memcpy(&t, &top, sizeof(t));
        return group_top<V>(to_float<T>(t));
    } else {
        float x[V];
        to_floats<T, V>(f, x);
        return group_top<V>(x);
    }
}
__device__ __forceinline__ uint32_t group_exponent(uint32_t top) {
    const int biased = (int)(top >> 23);            // floor(log2 amax) + 127; 0 for zero and subnormals
    return biased == 255 ? 255u : (uint32_t)max(biased - 6, 1);
}
// x 2^-k is rounded to the nearest integer by adding 1.5 2^23 in the same operation: the sum's last bits are the integer,
// in two's complement (a conversion instruction runs at an eighth of that rate).  Only a group whose largest magnitude
// rounds to 128 steps is clamped, and only one with an infinity or a NaN is cleared.
template <int V> __device__ __forceinline__ void quantise(const float (&x)[V], uint32_t top, uint32_t e, uint32_t (&q)[V]) {
    const float inv = __uint_as_float((254u - e) << 23);                    // 2^-k, e in [1, 248]; -infinity for 255
#pragma unroll
    for (int i = 0; i < V; ++i) q[i] = __float_as_uint(fmaf(x[i], inv, 12582912.f));
    if (!(fabsf(__uint_as_float(top) * inv) < 127.5f)) {
#pragma unroll
        for (int i = 0; i < V; ++i) q[i] = e == 255 ? 0u : min(max(q[i], 0x4b400000u - 127u), 0x4b400000u + 127u);
    }
}
// 2^k; +infinity for e = 255, which makes q e NaN because q is 0 there.
__device__ __forceinline__ float group_scale(uint32_t e) { return __uint_as_float(e << 23); }

// Stores the low bytes of q.
template <int V> __device__ __forceinline__ void store_q(int8_t *p, const uint32_t (&q)[V]) {
    if constexpr (V == 1) {
        *p = (int8_t)q[0];
    } else {
        uint2 w;
        w.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
        w.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
        *reinterpret_cast<uint2 *>(p) = w;
    }
}
// V of a row's 8-bit integers as they lie in memory, and the values they stand for.
template <int V> struct RawQ { uint32_t w[V == 1 ? 1 : V / 4]; };
template <int V> __device__ __forceinline__ RawQ<V> load_q(const int8_t *p) {
    RawQ<V> r;
    if constexpr (V == 1) r.w[0] = (uint8_t)*p;
    else asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "l"(p));
    return r;
}
// q 2^k as the difference of 2^k (2^23 + q + 128), which the byte completes to a float's bits, and 2^k (2^23 + 128); both
// and the difference are exact.  Steps above 2^104 (and the marker 255) take the plain way.
template <int V> __device__ __forceinline__ void held_values(const RawQ<V> &q, uint32_t e, float (&x)[V]) {
    const uint32_t base = (e + 23u) << 23;
    const float zero = __uint_as_float(base | 128u);
    if (e < 232u) {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = __uint_as_float(__byte_perm(q.w[i / 4] ^ 0x80808080u, base, 0x7650 + i % 4)) - zero;
    } else {
#pragma unroll
        for (int i = 0; i < V; ++i) x[i] = (float)(int8_t)(q.w[i / 4] >> (i % 4 * 8)) * group_scale(e);
    }
}
template <int V> __device__ __forceinline__ void load_held(const int8_t *q, const uint8_t *e, int col, float (&x)[V]) {
    held_values<V>(load_q<V>(q + col), e[(unsigned)col / kGroup], x);
}

// Writes the checkpoint of V columns at `col`; every lane of the warp calls it, `valid` where the columns exist (the
// others pass zeros).  `top`: group_top of the same values.
template <int V>
__device__ __forceinline__ void store_held(int8_t *q, uint8_t *e, int col, bool valid, const float (&x)[V], uint32_t top) {
    const uint32_t ex = group_exponent(top);
    uint32_t v[V];
    quantise<V>(x, top, ex, v);
    if (valid) {
        store_q<V>(q + col, v);
        if (col % kGroup == 0) e[(unsigned)col / kGroup] = (uint8_t)ex;
    }
}
template <int V> __device__ __forceinline__ void store_held(int8_t *q, uint8_t *e, int col, bool valid, const float (&x)[V]) {
    store_held<V>(q, e, col, valid, x, group_top<V>(x));
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
