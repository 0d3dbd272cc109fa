// Gated feed-forward block (see include/def_train.h): what its two fused products do with their accumulators.
//
//     forward    [g | u] = x W_in^T,   h = g s u,  s = 1 / (1 + exp(-g));   checkpoints of g and u
//     backward   dh = dout W_down,     dg = dh u s (1 + g (1 - s)),  du = dh g s,  h^ = g s u  from the checkpoints
//
// The first product's tile is 128 columns of g beside the same 128 of u: the two CTAs of a pair bring one each, and a thread
// holds 64 of either, two groups of a checkpoint.  Nothing but h (or dg, du and h^) goes to memory in more than 8 bits.
#pragma once

#include "def_product_kernels.cuh"

namespace deft {

// A group of 32 columns that one thread holds, the first n of which exist.
__device__ __forceinline__ uint32_t held_top(const float (&x)[32], int n) {
    float top = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (i < n) top = max_nan(top, fabsf(x[i]));
    return __float_as_uint(top);
}
__device__ __forceinline__ void store_group(int8_t *q, uint8_t *e, const float (&x)[32], int n) {
    const uint32_t top = held_top(x, n), ex = group_exponent(top);
#pragma unroll
    for (int p = 0; p < 4; p += 2) {
        uint32_t w[4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float part[8];
            uint32_t v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) part[i] = x[8 * (p + r) + i];
            quantise(part, top, ex, v);
            if (n >= 32) {
                w[2 * r] = __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
                w[2 * r + 1] = __byte_perm(__byte_perm(v[4], v[5], 0x0040), __byte_perm(v[6], v[7], 0x0040), 0x5410);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (8 * (p + r) + i < n) q[8 * (p + r) + i] = (int8_t)v[i];
            }
        }
        if (n >= 32) *reinterpret_cast<uint4 *>(q + 8 * p) = make_uint4(w[0], w[1], w[2], w[3]);
    }
    *e = (uint8_t)ex;
}
// The values of a group (rows of q are padded to 16 bytes: words that begin inside a row lie inside it).
__device__ __forceinline__ void load_group(const int8_t *q, const uint8_t *e, float (&x)[32], int n) {
    uint4 w[2];
    w[0] = *reinterpret_cast<const uint4 *>(q);
    w[1] = n > 16 ? *reinterpret_cast<const uint4 *>(q + 16) : make_uint4(0, 0, 0, 0);
    const uint32_t ex = *e;
#pragma unroll
    for (int p = 0; p < 4; ++p) {
        RawQ r;
        r.w[0] = p % 2 ? w[p / 2].z : w[p / 2].x;
        r.w[1] = p % 2 ? w[p / 2].w : w[p / 2].y;
        float part[8];
        held_values(r, ex, part);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[8 * p + i] = part[i];
    }
}

template <typename T> __device__ __forceinline__ float logistic(float g) {
    if constexpr (sizeof(T) == 2) return __fdividef(1.f, 1.f + __expf(-g));
    else return 1.f / (1.f + expf(-g));
}

template <typename T> struct StoreGated {
    T *h;
    int64_t ldh, rows, F, ldq, lde;
    int8_t *gate_q, *up_q;
    uint8_t *gate_e, *up_e;
    int wide;
    static __device__ __forceinline__ uint32_t first(int half) { return half * 64; }
    static __device__ __forceinline__ uint32_t second(int half) { return 128 + half * 64; }
    __device__ __forceinline__ void store(const float (&acc)[128], int, int64_t row, int64_t col, int half, bool) const {
        if (row >= rows) return;
        col += half * 64;
#pragma unroll
        for (int part = 0; part < 2; ++part) {
            const int64_t c = col + 32 * part;
            if (c >= F) break;
            const int n = F - c < 32 ? (int)(F - c) : 32;
            float g[32], u[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                g[i] = acc[32 * part + i];
                u[i] = acc[64 + 32 * part + i];
            }
            if (gate_q) {
                store_group(gate_q + row * ldq + c, gate_e + row * lde + c / kGroup, g, n);
                store_group(up_q + row * ldq + c, up_e + row * lde + c / kGroup, u, n);
            }
#pragma unroll
            for (int i = 0; i < 32; ++i) g[i] = g[i] * logistic<T>(g[i]) * u[i];
            store_32<T>(h + row * ldh + c, n, wide, g);
        }
    }
};

template <typename T> struct StoreGatedBack {
    T *dgate, *dup, *h;
    int64_t ldd, ldh, rows, F, ldq, lde;
    const int8_t *gate_q, *up_q;
    const uint8_t *gate_e, *up_e;
    int8_t *h_q;
    uint8_t *h_e;
    int wide, wide_up, wide_h;
    static __device__ __forceinline__ uint32_t first(int half) { return half * 128; }
    static __device__ __forceinline__ uint32_t second(int half) { return half * 128 + 64; }
    __device__ __forceinline__ void store(const float (&acc)[128], int, int64_t row, int64_t col, int half, bool) const {
        if (row >= rows) return;
        col += half * 128;
#pragma unroll
        for (int part = 0; part < 4; ++part) {
            const int64_t c = col + 32 * part;
            if (c >= F) break;
            const int n = F - c < 32 ? (int)(F - c) : 32;
            float g[32], u[32], d[32];
            load_group(gate_q + row * ldq + c, gate_e + row * lde + c / kGroup, g, n);
            load_group(up_q + row * ldq + c, up_e + row * lde + c / kGroup, u, n);
#pragma unroll
            for (int i = 0; i < 32; ++i) {
                const float s = logistic<T>(g[i]), dh = acc[32 * part + i], gs = g[i] * s;
                d[i] = dh * u[i] * (s * (1.f + g[i] * (1.f - s)));
                u[i] = gs * u[i];                                   // h^
                g[i] = dh * gs;
            }
            store_32<T>(dgate + row * ldd + c, n, wide, d);
            store_32<T>(dup + row * ldd + c, n, wide_up, g);
            if (h) store_32<T>(h + row * ldh + c, n, wide_h, u);
            if (h_q) {
#pragma unroll
                for (int i = 0; i < 32; ++i) u[i] = to_float<T>(from_float<T>(u[i]));
                store_group(h_q + row * ldq + c, h_e + row * lde + c / kGroup, u, n);
            }
        }
    }
};

}  // namespace deft
