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

// V = 8 consecutive elements as they lie in memory.
template <typename T, int V> struct alignas(16) Frag { T v[V]; };

// Streams that are read once bypass the L1, which is left to what CTAs share (weights).
template <typename T, int V> __device__ __forceinline__ Frag<T, V> load_frag(const T *p) {
    Frag<T, V> f;
    constexpr int kWords = sizeof(T) * V / 16;
    uint4 w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i)
        asm volatile("ld.global.L1::no_allocate.v4.u32 {%0, %1, %2, %3}, [%4];"
                     : "=r"(w[i].x), "=r"(w[i].y), "=r"(w[i].z), "=r"(w[i].w)
                     : "l"(reinterpret_cast<const uint4 *>(p) + i));
    memcpy(&f, w, sizeof(f));
    return f;
}
template <typename T, int V> __device__ __forceinline__ void to_floats(const Frag<T, V> &f, float (&out)[V]) {
#pragma unroll
    for (int i = 0; i < V; ++i) out[i] = to_float<T>(f.v[i]);
}
template <typename T, int V> __device__ __forceinline__ void store_floats(T *p, const float (&in)[V]) {
    Frag<T, V> f;
#pragma unroll
    for (int i = 0; i < V; ++i) f.v[i] = from_float<T>(in[i]);
    constexpr int kWords = sizeof(T) * V / 16;
    uint4 w[kWords];
    memcpy(w, &f, sizeof(f));
#pragma unroll
    for (int i = 0; i < kWords; ++i) reinterpret_cast<uint4 *>(p)[i] = w[i];
}
template <typename T, int V> __device__ __forceinline__ Frag<T, V> zeros() {
    Frag<T, V> f;
    memset(&f, 0, sizeof(f));
    return f;
}
// fp32 parameters, read by every row: cached.  Columns from C on give 0.
__device__ __forceinline__ void load_params(const float *p, int col, int C, float (&out)[8]) {
    p += col;
    if (col + 8 <= C && (reinterpret_cast<uintptr_t>(p) & 15u) == 0) {
#pragma unroll
        for (int i = 0; i < 2; ++i) {
            const float4 t = __ldg(reinterpret_cast<const float4 *>(p) + i);
            out[4 * i] = t.x; out[4 * i + 1] = t.y; out[4 * i + 2] = t.z; out[4 * i + 3] = t.w;
        }
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) out[i] = col + i < C ? __ldg(p + i) : 0.f;
    }
}

// ---------------------------------------------------------------------------
// Rows that do not start on 16-byte boundaries, still 8 columns per lane.  A warp's lanes hold consecutive runs of 8 columns
// of one row, so all their addresses are off by the same number of bytes.  A run is read as the aligned words around it
// and shifted into place; to write, a lane takes the end of its neighbour's run and the beginning of its own, which fill
// aligned words.  Only what lies wholly inside the row is touched by words: the row's first and last columns and the ends
// of a warp go element by element.  (Element accesses alone: a fifth of this speed.)
// ---------------------------------------------------------------------------

// N words starting `off` bytes into w (off < 16; a multiple of 2, and of 4 for 32-bit elements).
template <int N> __device__ __forceinline__ void shift_words(uint32_t (&w)[N + 4], uint32_t off, uint32_t (&out)[N]) {
    if (off & 8) {
#pragma unroll
        for (int i = 0; i < N + 2; ++i) w[i] = w[i + 2];
    }
    if (off & 4) {
#pragma unroll
        for (int i = 0; i < N + 1; ++i) w[i] = w[i + 1];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) out[i] = __funnelshift_r(w[i], w[i + 1], (off & 2) * 8);
}
template <typename T> __device__ __forceinline__ Frag<T, 8> load_run(const T *row, int col, int C) {
    constexpr int kWords = 2 * (int)sizeof(T);        // 32-bit words of a run
    constexpr int kSize = (int)sizeof(T);
    Frag<T, 8> f;
    const T *p = row + col;
    const uint32_t off = (uint32_t)(uintptr_t)p & 15u;
    const int before = (int)off / kSize;              // elements of the first word that are not the run's
    const int reach = off ? 8 + 16 / kSize - before : 8;          // elements from `col` to the end of the last word
    if (col >= before && col + reach <= C) {
        uint32_t w[kWords + 4], out[kWords];
        const uint4 *q = reinterpret_cast<const uint4 *>(reinterpret_cast<uintptr_t>(p) - off);
#pragma unroll
        for (int i = 0; i < kWords / 4 + 1; ++i) {
            uint4 v = make_uint4(0, 0, 0, 0);
            if (i < kWords / 4 || off)
                asm volatile("ld.global.v4.u32 {%0, %1, %2, %3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "l"(q + i));
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
        shift_words<kWords>(w, off, out);
        memcpy(&f, out, sizeof(f));
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) f.v[i] = col + i < C ? p[i] : from_float<T>(0.f);
    }
    return f;
}
// Stores run [col, col + 8) given the last 16 bytes of the run before it.  `own`: this thread writes the words that begin
// with the neighbour's end; `next`: its neighbour writes those that begin with this run's end.  What neither covers goes
// element by element.
template <typename T> __device__ __forceinline__ void store_shifted(T *row, int col, int C, const Frag<T, 8> &f, const uint4 &neighbour, bool own, bool next) {
    constexpr int kWords = 2 * (int)sizeof(T), kSize = (int)sizeof(T);
    T *p = row + col;
    const uint32_t off = (uint32_t)(uintptr_t)p & 15u;
    const int before = (int)off / kSize;              // elements of the neighbour's run in this run's first word
    uint32_t w[kWords + 4], out[kWords];
    w[0] = neighbour.x; w[1] = neighbour.y; w[2] = neighbour.z; w[3] = neighbour.w;
    memcpy(w + 4, &f, sizeof(f));
    // the words start `before` elements before the run, that is 16 - off bytes into w
    if (off == 0) {
#pragma unroll
        for (int i = 0; i < kWords; ++i) out[i] = w[4 + i];
    } else {
        shift_words<kWords>(w, 16u - off, out);
    }
    own = (own || off == 0) && col - before + 8 <= C;
    next = next && col - before + 16 <= C;
    if (own) {
        uint4 *q = reinterpret_cast<uint4 *>(reinterpret_cast<uintptr_t>(p) - off);
#pragma unroll
        for (int i = 0; i < kWords / 4; ++i) q[i] = make_uint4(out[4 * i], out[4 * i + 1], out[4 * i + 2], out[4 * i + 3]);
    }
    const int from = own ? 8 - before : 0, to = next || (off == 0 && own) ? 8 - before : 8;
    const int exist = C - col < 8 ? C - col : 8;
    const uint32_t mask = exist > 0 ? ((1u << to) - 1u) & ~((1u << from) - 1u) & ((1u << exist) - 1u) : 0u;
    if (mask) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (mask >> i & 1u) p[i] = f.v[i];
    }
}
template <typename T> __device__ __forceinline__ Frag<T, 8> round_run(const float (&x)[8]) {
    Frag<T, 8> f;
#pragma unroll
    for (int i = 0; i < 8; ++i) f.v[i] = from_float<T>(x[i]);
    return f;
}
template <typename T> __device__ __forceinline__ uint4 end_of_run(const Frag<T, 8> &f) {
    uint4 w[sizeof(T) / 2];
    memcpy(w, &f, sizeof(f));
    return w[sizeof(T) / 2 - 1];
}
// Every lane of the warp calls it; lanes with col >= C store nothing.  The ends of the warp's columns go by element.
template <typename T> __device__ __forceinline__ void store_run(T *row, int col, int C, const float (&x)[8]) {
    const int lane = threadIdx.x & 31;
    const Frag<T, 8> f = round_run<T>(x);
    uint4 n = end_of_run<T>(f);
    n.x = __shfl_up_sync(0xffffffffu, n.x, 1);
    n.y = __shfl_up_sync(0xffffffffu, n.y, 1);
    n.z = __shfl_up_sync(0xffffffffu, n.z, 1);
    n.w = __shfl_up_sync(0xffffffffu, n.w, 1);
    store_shifted<T>(row, col, C, f, n, lane > 0, lane < 31);
}
// A whole row by a CTA, thread i holding runs i, i + threads, ...: warps hand their ends on in `ends` [ITERS * 32], so only
// the row's own ends go by element.  Every thread calls it; it waits for all of them once.
template <typename T, int ITERS> __device__ __forceinline__ void store_row(T *row, int threads, int C, const float (&x)[ITERS][8], uint4 *ends) {
    const int lane = threadIdx.x & 31, warps = threads >> 5;
    Frag<T, 8> f[ITERS];
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        f[it] = round_run<T>(x[it]);
        if (lane == 31) ends[it * warps + (threadIdx.x >> 5)] = end_of_run<T>(f[it]);
    }
    __syncthreads();
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        uint4 n = end_of_run<T>(f[it]);
        n.x = __shfl_up_sync(0xffffffffu, n.x, 1);
        n.y = __shfl_up_sync(0xffffffffu, n.y, 1);
        n.z = __shfl_up_sync(0xffffffffu, n.z, 1);
        n.w = __shfl_up_sync(0xffffffffu, n.w, 1);
        const int col = (it * threads + (int)threadIdx.x) * 8;
        if (lane == 0 && col > 0) n = ends[it * warps + (int)(threadIdx.x >> 5) - 1];
        store_shifted<T>(row, col, C, f[it], n, col > 0, true);
    }
}
// Columns [col, col + 8) of a row: whole words where rows are ALIGNED (C is then a multiple of 8), as above elsewhere.
template <typename T, bool ALIGNED> __device__ __forceinline__ Frag<T, 8> load_cols(const T *row, int col, int C) {
    if constexpr (ALIGNED) return load_frag<T, 8>(row + col);
    else return load_run<T>(row, col, C);
}
template <typename T, bool ALIGNED> __device__ __forceinline__ void store_cols(T *row, int col, int C, const float (&x)[8]) {
    if constexpr (ALIGNED) {
        if (col < C) store_floats<T, 8>(row + col, x);
    } else {
        store_run<T>(row, col, C, x);
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
// ---------------------------------------------------------------------------
// Checkpoint group: 32 consecutive columns of a row, held by 4 consecutive lanes of a warp (8 columns each).
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
__device__ __forceinline__ uint32_t group_top(float top) {
    uint32_t bits = __float_as_uint(top) & 0x7fffffffu;
#pragma unroll
    for (int s = 1; s < kGroup / 8; s <<= 1) bits = max(bits, __shfl_xor_sync(0xffffffffu, bits, s));
    return bits;
}
__device__ __forceinline__ uint32_t group_top(const float (&x)[8]) {
    float top = fabsf(x[0]);
#pragma unroll
    for (int i = 1; i < 8; ++i) top = max_nan(top, fabsf(x[i]));
    return group_top(top);
}
// The same from 16-bit values as loaded: magnitudes of either type order like the integers they are held in.
template <typename T> __device__ __forceinline__ uint32_t group_top(const Frag<T, 8> &f) {
    if constexpr (sizeof(T) == 2) {
        uint32_t w[4];
        memcpy(w, &f, sizeof(w));
        const uint32_t m = __vmaxu2(__vmaxu2(w[0] & 0x7fff7fffu, w[1] & 0x7fff7fffu), __vmaxu2(w[2] & 0x7fff7fffu, w[3] & 0x7fff7fffu));
        const uint16_t top = (uint16_t)max(m & 0xffffu, m >> 16);
        T t;
        memcpy(&t, &top, sizeof(t));
        return group_top(to_float<T>(t));
    } else {
        return group_top(f.v);
    }
}
__device__ __forceinline__ uint32_t group_exponent(uint32_t top) {
    const int biased = (int)(top >> 23);            // floor(log2 amax) + 127; 0 for zero and subnormals
    return biased == 255 ? 255u : (uint32_t)max(biased - 6, 1);
}
// x 2^-k is rounded to the nearest integer by adding 1.5 2^23 in the same operation: the sum's last bits are the integer,
// in two's complement (a conversion instruction runs at an eighth of that rate).  Only a group whose largest magnitude
// rounds to 128 steps is clamped, and only one with an infinity or a NaN is cleared.
__device__ __forceinline__ void quantise(const float (&x)[8], uint32_t top, uint32_t e, uint32_t (&q)[8]) {
    const float inv = __uint_as_float((254u - e) << 23);                    // 2^-k, e in [1, 248]; -infinity for 255
#pragma unroll
    for (int i = 0; i < 8; ++i) q[i] = __float_as_uint(fmaf(x[i], inv, 12582912.f));
    if (!(fabsf(__uint_as_float(top) * inv) < 127.5f)) {
#pragma unroll
        for (int i = 0; i < 8; ++i) q[i] = e == 255 ? 0u : min(max(q[i], 0x4b400000u - 127u), 0x4b400000u + 127u);
    }
}
// 2^k; +infinity for e = 255, which makes q e NaN because q is 0 there.
__device__ __forceinline__ float group_scale(uint32_t e) { return __uint_as_float(e << 23); }

// Stores the low bytes of q, the first n of them.
__device__ __forceinline__ void store_q(int8_t *p, int n, const uint32_t (&q)[8]) {
    if (n >= 8) {
        uint2 w;
        w.x = __byte_perm(__byte_perm(q[0], q[1], 0x0040), __byte_perm(q[2], q[3], 0x0040), 0x5410);
        w.y = __byte_perm(__byte_perm(q[4], q[5], 0x0040), __byte_perm(q[6], q[7], 0x0040), 0x5410);
        *reinterpret_cast<uint2 *>(p) = w;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (i < n) p[i] = (int8_t)q[i];
    }
}
// 8 of a row's 8-bit integers as they lie in memory (rows are padded to 16), and the values they stand for.
struct RawQ { uint32_t w[2]; };
__device__ __forceinline__ RawQ load_q(const int8_t *p) {
    RawQ r;
    asm volatile("ld.global.L1::no_allocate.v2.u32 {%0, %1}, [%2];" : "=r"(r.w[0]), "=r"(r.w[1]) : "l"(p));
    return r;
}
// q 2^k as the difference of 2^k (2^23 + q + 128), which the byte completes to a float's bits, and 2^k (2^23 + 128); both
// and the difference are exact.  Steps above 2^104 (and the marker 255) take the plain way.
__device__ __forceinline__ void held_values(const RawQ &q, uint32_t e, float (&x)[8]) {
    const uint32_t base = (e + 23u) << 23;
    const float zero = __uint_as_float(base | 128u);
    if (e < 232u) {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = __uint_as_float(__byte_perm(q.w[i / 4] ^ 0x80808080u, base, 0x7650 + i % 4)) - zero;
    } else {
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (float)(int8_t)(q.w[i / 4] >> (i % 4 * 8)) * group_scale(e);
    }
}
// The same of columns [col, col + 8), 0 for those from C on.
template <bool ALIGNED> __device__ __forceinline__ void held_cols(const RawQ &q, uint32_t e, int col, int C, float (&x)[8]) {
    held_values(q, e, x);
    if (!ALIGNED && col + 8 > C) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i >= C) x[i] = 0.f;
    }
}

// Writes the checkpoint of columns [col, min(col + 8, C)); every lane of the warp calls it, with zeros for columns that do
// not exist.  `top`: group_top of the same values.
template <bool ALIGNED> __device__ __forceinline__ void store_held(int8_t *q, uint8_t *e, int col, int C, const float (&x)[8], uint32_t top) {
    const uint32_t ex = group_exponent(top);
    uint32_t v[8];
    quantise(x, top, ex, v);
    if (col < C) {
        store_q(q + col, ALIGNED ? 8 : C - col, v);
        if (col % kGroup == 0) e[(unsigned)col / kGroup] = (uint8_t)ex;
    }
}
template <bool ALIGNED> __device__ __forceinline__ void store_held(int8_t *q, uint8_t *e, int col, int C, const float (&x)[8]) {
    store_held<ALIGNED>(q, e, col, C, x, group_top(x));
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
// What the CTA's threads accessed before is behind all of them afterwards, also where they are one warp.
// THREADS: those of the CTA, or 0 where only the launch knows.
template <int THREADS = 0> __device__ __forceinline__ float cta_sum(float v, float *scratch) {
    const int warps = (THREADS ? THREADS : (int)blockDim.x) >> 5, lane = threadIdx.x & 31;
    v = warp_sum(v);
    if (warps == 1) {
        __syncwarp();
        return v;
    }
    if (lane == 0) scratch[threadIdx.x >> 5] = v;
    __syncthreads();
    v = lane < warps ? scratch[lane] : 0.f;
    if constexpr (THREADS == 0 || THREADS == 1024 || (THREADS & (THREADS - 1)) != 0) {
        return warp_sum(v);
    } else {
#pragma unroll
        for (int s = THREADS / 64; s > 0; s >>= 1) v += __shfl_xor_sync(0xffffffffu, v, s);
        return __shfl_sync(0xffffffffu, v, 0);
    }
}

}  // namespace deft
