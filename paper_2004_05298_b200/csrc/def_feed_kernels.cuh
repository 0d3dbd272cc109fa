// Gated feed-forward block (see include/def_train.h): what its two fused products do with their accumulators.
//
//     forward    [g | u] = x W_in^T,   h = g s u,  s = 1 / (1 + exp(-g));   checkpoints of g and u
//     backward   dh = dout W_down,     dg = dh u s (1 + g (1 - s)),  du = dh g s,  h^ = g s u  from the checkpoints
//
// The first product's tile is 128 columns of g beside the same 128 of u: the two CTAs of a pair bring one each, and a thread
// holds 32 of either, a group of a checkpoint.  Nothing but h (or dg, du and h^) goes to memory in more than 8 bits.
#pragma once

#include "def_product_kernels.cuh"

namespace deft {

// Checkpoint of a group of 32 columns that one thread holds, the first n of which exist; whole groups are turned (32 bytes a
// row).  Whole warps call it.
template <typename V>
__device__ __forceinline__ void store_group(int8_t *q, int64_t ldq, uint8_t *e, const V (&x)[32], int n, bool there, uint8_t *turn) {
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (i < n) most = max_nan(most, fabsf(to_float<V>(x[i])));
    const uint32_t top = __float_as_uint(most), ex = group_exponent(top);
#pragma unroll
    for (int p = 0; p < 4; p += 2) {
        uint32_t w[4];
#pragma unroll
        for (int r = 0; r < 2; ++r) {
            float part[8];
            uint32_t v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) part[i] = to_float<V>(x[8 * (p + r) + i]);
            quantise(part, top, ex, v);
            if (n >= 32) {
                w[2 * r] = __byte_perm(__byte_perm(v[0], v[1], 0x0040), __byte_perm(v[2], v[3], 0x0040), 0x5410);
                w[2 * r + 1] = __byte_perm(__byte_perm(v[4], v[5], 0x0040), __byte_perm(v[6], v[7], 0x0040), 0x5410);
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i)
                    if (8 * (p + r) + i < n && there) q[8 * (p + r) + i] = (int8_t)v[i];
            }
        }
        if (n >= 32) turn_put_word<32>(turn, p / 2, make_uint4(w[0], w[1], w[2], w[3]));
    }
    if (n >= 32) turn_store_words<32>(turn, q, ldq, there);
    if (there) *e = (uint8_t)ex;
}

template <typename T> __device__ __forceinline__ float logistic(float g) {
    if constexpr (sizeof(T) == 2) return __fdividef(1.f, 1.f + expf(-g));
    else return 1.f / (1.f + expf(-g));
}

template <typename T> struct StoreGated {
    static constexpr bool kBoth = true;
    T *h;
    int64_t ldh, rows, F, ldq, lde;
    int8_t *gate_q, *up_q;
    uint8_t *gate_e, *up_e;
    int wide;
    __device__ __forceinline__ void store(float (&g)[32], float (&u)[32], int, int64_t row, int64_t c, uint8_t *turn) const {
        if (c >= F) return;
        const int n = F - c < 32 ? (int)(F - c) : 32;
        const bool there = row < rows;
        if (gate_q) {
            store_group(gate_q + row * ldq + c, ldq, gate_e + row * lde + c / kGroup, g, n, there, turn);
            store_group(up_q + row * ldq + c, ldq, up_e + row * lde + c / kGroup, u, n, there, turn);
        }
        T *p = h + row * ldh + c;
#pragma unroll
        for (int f = 0; f < 32; f += 8) {                          // 8 columns at a time, so that little is held at once
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = g[f + i] * logistic<T>(g[f + i]) * u[f + i];
            if (wide && n >= 32) {
                constexpr int W = kTurn<T>;
                turn_put_8<64, T>(turn, f % W, v);
                if (f % W + 8 == W) turn_store_words<64>(turn, p + f + 8 - W, ldh * (int64_t)sizeof(T), there);
            } else {
                constexpr int W = kTurn<T>;
                const int at = f % W;
#pragma unroll
                for (int i = 0; i < 8; ++i) turn_put<T, W>(turn, at + i, v[i]);
                if (at + 8 == W && f - at < n) turn_store<T, W>(turn, p + f - at, ldh, there, n - (f - at));
            }
        }
    }
};

template <typename T> struct StoreGatedBack {
    static constexpr bool kBoth = false;
    T *dgate, *dup, *h;
    int64_t ldd, ldh, rows, F, ldq, lde;
    const int8_t *gate_q, *up_q;
    const uint8_t *gate_e, *up_e;
    int8_t *h_q;
    uint8_t *h_e;
    int wide, wide_h;                     // of dgate and dup; of h
    // 8 columns at a time, so that little is held at once; only h^ is needed for the whole group.
    __device__ __forceinline__ void store(float (&dh)[32], float (&)[32], int, int64_t row, int64_t c, uint8_t *turn) const {
        if (c >= F) return;
        const int n = F - c < 32 ? (int)(F - c) : 32;
        const bool there = row < rows, direct = wide && n >= 32;
        const int8_t *q = gate_q + row * ldq + c, *r = up_q + row * ldq + c;
        const uint32_t eg = there ? gate_e[row * lde + c / kGroup] : 1u, eu = there ? up_e[row * lde + c / kGroup] : 1u;
        uint4 wg = {}, wu = {};                                    // 16 columns
        T *pg = dgate + row * ldd + c, *pu = dup + row * ldd + c;
        uint8_t *turn_up = turn + kTurnBytes / 2;
        T hv[32];
#pragma unroll
        for (int p = 0; p < 4; ++p) {
            if (p % 2 == 0 && there && 8 * p < n) {                // rows of q are padded to 16 bytes
                wg = *reinterpret_cast<const uint4 *>(q + 8 * p);
                wu = *reinterpret_cast<const uint4 *>(r + 8 * p);
            }
            const RawQ qg = {{p % 2 ? wg.z : wg.x, p % 2 ? wg.w : wg.y}}, qu = {{p % 2 ? wu.z : wu.x, p % 2 ? wu.w : wu.y}};
            float g[8], u[8], d[8];
            held_values(qg, eg, g);
            held_values(qu, eu, u);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float s = logistic<T>(g[i]), gs = g[i] * s, x = dh[8 * p + i];
                hv[8 * p + i] = from_float<T>(gs * u[i]);
                d[i] = x * u[i] * (s * fmaf(g[i], 1.f - s, 1.f));
                u[i] = x * gs;
            }
            constexpr int W = kTurn<T> / 2;                        // of either
            const int at = 8 * p % W, f = 8 * p - at;              // f: first column of the run that is put there
            if (direct) {
                turn_put_8<32, T>(turn, at, d);
                turn_put_8<32, T>(turn_up, at, u);
                if (at + 8 == W) {
                    turn_store_words<32>(turn, pg + f, ldd * (int64_t)sizeof(T), there);
                    turn_store_words<32>(turn_up, pu + f, ldd * (int64_t)sizeof(T), there);
                }
            } else {
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    turn_put<T, W>(turn, at + i, d[i]);
                    turn_put<T, W>(turn_up, at + i, u[i]);
                }
                if (at + 8 == W && f < n) {
                    turn_store<T, W>(turn, pg + f, ldd, there, n - f);
                    turn_store<T, W>(turn_up, pu + f, ldd, there, n - f);
                }
            }
        }
        if (h) store_32<T>(h + row * ldh + c, ldh, there, n, wide_h, hv, turn);
        if (h_q) store_group(h_q + row * ldq + c, ldq, h_e + row * lde + c / kGroup, hv, n, there, turn);
    }
};

}  // namespace deft
