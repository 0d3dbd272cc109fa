// 8-bit activation checkpoints and the gated activation that is kept in them (see include/def_train.h).
#pragma once

#include "def_train_common.cuh"

namespace deft {

// A CTA is blockDim.y rows by blockDim.x lanes of V columns; blockDim.x is a multiple of 32, so a warp lies in one row
// and the lanes that share an exponent are neighbours.
template <int V> struct Place {
    int64_t col;
    __device__ Place() : col(((int64_t)blockIdx.x * blockDim.x + threadIdx.x) * V) {}
};
__device__ __forceinline__ int64_t first_row() { return (int64_t)blockIdx.y * blockDim.y + threadIdx.y; }
__device__ __forceinline__ int64_t row_step() { return (int64_t)gridDim.y * blockDim.y; }

template <typename T, int V>
__global__ void __launch_bounds__(256) pack_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int64_t C,
                                                   int8_t *__restrict__ q, uint8_t *__restrict__ e, int64_t ldq, int64_t lde) {
    const int64_t col = Place<V>().col;
    for (int64_t t = first_row(); t < rows; t += row_step()) {
        float v[V];
#pragma unroll
        for (int i = 0; i < V; ++i) v[i] = 0.f;
        if (col < C) load_floats<T, V>(x + t * ldx + col, v);
        store_held<V>(q + t * ldq, e + t * lde, col, col < C, v);
    }
}

template <typename T, int V>
__global__ void __launch_bounds__(256) unpack_kernel(const int8_t *__restrict__ q, const uint8_t *__restrict__ e, int64_t ldq, int64_t lde,
                                                     int64_t rows, int64_t C, T *__restrict__ out, int64_t ldout) {
    const int64_t col = Place<V>().col;
    if (col >= C) return;
    for (int64_t t = first_row(); t < rows; t += row_step()) {
        float v[V];
        load_held<V>(q + t * ldq, e + t * lde, col, v);
        store_floats<T, V>(out + t * ldout + col, v);
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
__global__ void __launch_bounds__(256) gated_forward_kernel(const GatedForward a) {
    const int64_t col = Place<V>().col;
    for (int64_t t = first_row(); t < a.T; t += row_step()) {
        float g[V], u[V];
#pragma unroll
        for (int i = 0; i < V; ++i) g[i] = u[i] = 0.f;
        if (col < a.F) {
            load_floats<T, V>((const T *)a.gate + t * a.ldg + col, g);
            load_floats<T, V>((const T *)a.up + t * a.ldu + col, u);
            float h[V];
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = g[i] * sigmoid<T>(g[i]) * u[i];
            store_floats<T, V>((T *)a.h + t * a.ldh + col, h);
        }
        if (a.gate_q) store_held<V>(a.gate_q + t * a.ldq, a.gate_e + t * a.lde, col, col < a.F, g);
        if (a.up_q) store_held<V>(a.up_q + t * a.ldq, a.up_e + t * a.lde, col, col < a.F, u);
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
__global__ void __launch_bounds__(256) gated_backward_kernel(const GatedBackward a) {
    const int64_t col = Place<V>().col;
    for (int64_t t = first_row(); t < a.T; t += row_step()) {
        float h[V];
#pragma unroll
        for (int i = 0; i < V; ++i) h[i] = 0.f;
        if (col < a.F) {
            float g[V], u[V], d[V], dg[V], du[V];
            load_floats<T, V>((const T *)a.dh + t * a.lddh + col, d);
            load_held<V>(a.gate_q + t * a.ldq, a.gate_e + t * a.lde, col, g);
            load_held<V>(a.up_q + t * a.ldq, a.up_e + t * a.lde, col, u);
#pragma unroll
            for (int i = 0; i < V; ++i) {
                const float s = sigmoid<T>(g[i]), gs = g[i] * s;
                dg[i] = d[i] * u[i] * (s * fmaf(g[i], 1.f - s, 1.f));
                du[i] = d[i] * gs;
                h[i] = gs * u[i];
            }
            store_floats<T, V>((T *)a.dgate + t * a.lddg + col, dg);
            store_floats<T, V>((T *)a.dup + t * a.lddu + col, du);
            if (a.h) store_floats<T, V>((T *)a.h + t * a.ldh + col, h);
        }
        if (a.h_q) {
#pragma unroll
            for (int i = 0; i < V; ++i) h[i] = to_float<T>(from_float<T>(h[i]));     // the values h_out holds
            store_held<V>(a.h_q + t * a.ldq, a.h_e + t * a.lde, col, col < a.F, h);
        }
    }
}

}  // namespace deft
