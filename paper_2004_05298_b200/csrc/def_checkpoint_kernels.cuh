// 8-bit activation checkpoints and the gated activation that is kept in them (see include/def_train.h).
#pragma once

#include "def_train_common.cuh"

namespace deft {

// A CTA is blockDim.y rows by blockDim.x lanes of V columns; blockDim.x is a multiple of 32, so a warp lies in one row
// and the lanes that share an exponent are neighbours.  These kernels move bytes and little else: what counts is that
// few instructions go into an element and that an SM holds enough threads (32 registers: 2048 of them) to keep enough
// loads in flight.  Several rows per thread with all loads first cost more in registers than they gave.
template <int V> struct Place {
    int col;
    int64_t row, step;
    __device__ Place()
        : col((int)(blockIdx.x * blockDim.x + threadIdx.x) * V), row((int64_t)blockIdx.y * blockDim.y + threadIdx.y),
          step((int64_t)gridDim.y * blockDim.y) {}
};
template <typename T, int V>
__global__ void __launch_bounds__(256, 8) pack_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int C,
                                                      int8_t *__restrict__ q, uint8_t *__restrict__ e, int64_t ldq, int64_t lde) {
    const Place<V> at;
    const bool live = at.col < C;
    x += at.row * ldx + at.col;
    q += at.row * ldq;
    e += at.row * lde;
    for (int64_t t = at.row; t < rows; t += at.step) {
        Frag<T, V> f = zeros<T, V>();
        if (live) f = load_frag<T, V>(x);
        const uint32_t top = group_top<T, V>(f);
        float v[V];
        to_floats<T, V>(f, v);
        store_held<V>(q, e, at.col, live, v, top);
        x += at.step * ldx;
        q += at.step * ldq;
        e += at.step * lde;
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(256, 8) unpack_kernel(const int8_t *__restrict__ q, const uint8_t *__restrict__ e, int64_t ldq, int64_t lde,
                                                        int64_t rows, int C, T *__restrict__ out, int64_t ldout) {
    const Place<V> at;
    if (at.col >= C) return;
    q += at.row * ldq + at.col;
    e += at.row * lde + (unsigned)at.col / kGroup;
    out += at.row * ldout + at.col;
    for (int64_t t = at.row; t < rows; t += at.step) {
        float v[V];
        const RawQ<V> w = load_q<V>(q);
        held_values<V>(w, *e, v);
        store_floats<T, V>(out, v);
        q += at.step * ldq;
        e += at.step * lde;
        out += at.step * ldout;
    }
}

// 1 / (1 + exp(-g)).  16-bit activations: hardware exponential and reciprocal (2^-21 relative, far below their 2^-9 or
// 2^-12 rounding); fp32 activations: the accurate ones.
template <typename T> __device__ __forceinline__ float sigmoid(float g) {
    if constexpr (sizeof(T) == 2) return __fdividef(1.f, 1.f + __expf(-g));
    else return 1.f / (1.f + expf(-g));
}

struct GatedForward {
    const void *gate, *up;
    void *h;
    int64_t ldg, ldu, ldh;
    int8_t *gate_q, *up_q;
    uint8_t *gate_e, *up_e;
    int64_t T, F, ldq, lde;
};

template <typename T, int V>
__global__ void __launch_bounds__(256, 5) gated_forward_kernel(const GatedForward a) {
    const Place<V> at;
    const bool live = at.col < a.F;
    const T *gate = (const T *)a.gate + at.row * a.ldg + at.col, *up = (const T *)a.up + at.row * a.ldu + at.col;
    T *out = (T *)a.h + at.row * a.ldh + at.col;
    int64_t at_q = at.row * a.ldq, at_e = at.row * a.lde;
    for (int64_t t = at.row; t < a.T; t += at.step) {
        Frag<T, V> fg = zeros<T, V>(), fu = zeros<T, V>();
        if (live) {
            fg = load_frag<T, V>(gate);
            fu = load_frag<T, V>(up);
        }
        float g[V], u[V];
        to_floats<T, V>(fg, g);
        to_floats<T, V>(fu, u);
        if (a.gate_q) store_held<V>(a.gate_q + at_q, a.gate_e + at_e, at.col, live, g, group_top<T, V>(fg));
        if (a.up_q) store_held<V>(a.up_q + at_q, a.up_e + at_e, at.col, live, u, group_top<T, V>(fu));
        if (live) {
#pragma unroll
            for (int i = 0; i < V; ++i) g[i] = g[i] * sigmoid<T>(g[i]) * u[i];
            store_floats<T, V>(out, g);
        }
        gate += at.step * a.ldg;
        up += at.step * a.ldu;
        out += at.step * a.ldh;
        at_q += at.step * a.ldq;
        at_e += at.step * a.lde;
    }
}

struct GatedBackward {
    const void *dh;
    const int8_t *gate_q, *up_q;
    const uint8_t *gate_e, *up_e;
    void *dgate, *dup, *h;
    int64_t lddh, lddg, lddu, ldh;
    int8_t *h_q;
    uint8_t *h_e;
    int64_t T, F, ldq, lde;
};

template <typename T, int V>
__global__ void __launch_bounds__(256, sizeof(T) == 2 ? 5 : 4) gated_backward_kernel(const GatedBackward a) {
    const Place<V> at;
    const bool live = at.col < a.F;
    const T *dh = (const T *)a.dh + at.row * a.lddh + at.col;
    T *dgate = (T *)a.dgate + at.row * a.lddg + at.col, *dup = (T *)a.dup + at.row * a.lddu + at.col, *out = (T *)a.h + at.row * a.ldh + at.col;
    int64_t at_q = at.row * a.ldq, at_e = at.row * a.lde + (unsigned)at.col / kGroup;
    for (int64_t t = at.row; t < a.T; t += at.step) {
        float h[V];
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = 0.f;
        if (live) {
            const Frag<T, V> fd = load_frag<T, V>(dh);
            const RawQ<V> qg = load_q<V>(a.gate_q + at_q + at.col), qu = load_q<V>(a.up_q + at_q + at.col);
            const uint32_t eg = a.gate_e[at_e], eu = a.up_e[at_e];
            float g[V], u[V], d[V];
            to_floats<T, V>(fd, d);
            held_values<V>(qg, eg, g);
            held_values<V>(qu, eu, u);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float s = sigmoid<T>(g[i]), gs = g[i] * s, du = d[i] * gs;
                h[i] = gs * u[i];
                d[i] = d[i] * u[i] * (s * fmaf(g[i], 1.f - s, 1.f));
                u[i] = du;
            }
            store_floats<T, V>(dgate, d);
            store_floats<T, V>(dup, u);
            if (a.h) store_floats<T, V>(out, h);
        }
        if (a.h_q) {
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = to_float<T>(from_float<T>(h[i]));     // the values h_out holds
            store_held<V>(a.h_q + at_q, a.h_e + t * a.lde, at.col, live, h);
        }
        dh += at.step * a.lddh;
        dgate += at.step * a.lddg;
        dup += at.step * a.lddu;
        out += at.step * a.ldh;
        at_q += at.step * a.ldq;
        at_e += at.step * a.lde;
    }
}

}  // namespace deft
