// 8-bit activation checkpoints and the gated activation that is kept in them (see include/def_train.h).
#pragma once

#include "def_train_common.cuh"

namespace deft {

// A CTA is blockDim.y rows by blockDim.x lanes of 8 columns; blockDim.x is a multiple of 32, so a warp lies in one row
// and the lanes that share an exponent are neighbours.  These kernels move bytes and little else: what counts is that
// few instructions go into an element and that an SM holds enough threads (32 registers: 2048 of them) to keep enough
// loads in flight.  Several rows per thread with all loads first cost more in registers than they gave.
// 16384 x 8192 bf16: pack 73 us (407 MB), unpack 76; 8192 x 10240 gated: forward 122 us (676 MB), backward 145 (844 MB).
struct Place {
    int col;
    int64_t row, step;
    __device__ Place()
        : col((int)(blockIdx.x * blockDim.x + threadIdx.x) * 8), row((int64_t)blockIdx.y * blockDim.y + threadIdx.y),
          step((int64_t)gridDim.y * blockDim.y) {}
};

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256, ALIGNED ? 8 : 6) pack_kernel(const T *__restrict__ x, int64_t ldx, int64_t rows, int C,
                                                                    int8_t *__restrict__ q, uint8_t *__restrict__ e, int64_t ldq, int64_t lde) {
    const Place at;
    x += at.row * ldx;
    q += at.row * ldq;
    e += at.row * lde;
    for (int64_t t = at.row; t < rows; t += at.step) {
        Frag<T, 8> f = zeros<T, 8>();
        if (at.col < C) f = load_cols<T, ALIGNED>(x, at.col, C);
        const uint32_t top = group_top<T>(f);
        float v[8];
        to_floats<T, 8>(f, v);
        store_held<ALIGNED>(q, e, at.col, C, v, top);
        x += at.step * ldx;
        q += at.step * ldq;
        e += at.step * lde;
    }
}

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256, ALIGNED ? 8 : 6) unpack_kernel(const int8_t *__restrict__ q, const uint8_t *__restrict__ e, int64_t ldq, int64_t lde,
                                                                      int64_t rows, int C, T *__restrict__ out, int64_t ldout) {
    const Place at;
    q += at.row * ldq + at.col;
    e += at.row * lde + (unsigned)at.col / kGroup;
    out += at.row * ldout;
    for (int64_t t = at.row; t < rows; t += at.step) {
        float v[8];
        RawQ w = {{0, 0}};
        uint32_t ex = 1;
        if (at.col < C) {
            w = load_q(q);
            ex = *e;
        }
        held_values(w, ex, v);
        store_cols<T, ALIGNED>(out, at.col, C, v);
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

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256, ALIGNED ? 5 : 4) gated_forward_kernel(const GatedForward a) {
    const Place at;
    const int F = (int)a.F;
    const T *gate = (const T *)a.gate + at.row * a.ldg, *up = (const T *)a.up + at.row * a.ldu;
    T *out = (T *)a.h + at.row * a.ldh;
    int64_t at_q = at.row * a.ldq, at_e = at.row * a.lde;
    for (int64_t t = at.row; t < a.T; t += at.step) {
        Frag<T, 8> fg = zeros<T, 8>(), fu = zeros<T, 8>();
        if (at.col < F) {
            fg = load_cols<T, ALIGNED>(gate, at.col, F);
            fu = load_cols<T, ALIGNED>(up, at.col, F);
        }
        float g[8], u[8];
        to_floats<T, 8>(fg, g);
        to_floats<T, 8>(fu, u);
        if (a.gate_q) store_held<ALIGNED>(a.gate_q + at_q, a.gate_e + at_e, at.col, F, g, group_top<T>(fg));
        if (a.up_q) store_held<ALIGNED>(a.up_q + at_q, a.up_e + at_e, at.col, F, u, group_top<T>(fu));
#pragma unroll
        for (int i = 0; i < 8; ++i) g[i] = g[i] * sigmoid<T>(g[i]) * u[i];
        store_cols<T, ALIGNED>(out, at.col, F, g);
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

template <typename T, bool ALIGNED>
__global__ void __launch_bounds__(256, ALIGNED && sizeof(T) == 2 ? 5 : 4) gated_backward_kernel(const GatedBackward a) {
    const Place at;
    const int F = (int)a.F;
    const T *dh = (const T *)a.dh + at.row * a.lddh;
    T *dgate = (T *)a.dgate + at.row * a.lddg, *dup = (T *)a.dup + at.row * a.lddu, *out = (T *)a.h + at.row * a.ldh;
    int64_t at_q = at.row * a.ldq + at.col, at_e = at.row * a.lde + (unsigned)at.col / kGroup;
    for (int64_t t = at.row; t < a.T; t += at.step) {
        Frag<T, 8> fd = zeros<T, 8>();
        RawQ qg = {{0, 0}}, qu = {{0, 0}};
        uint32_t eg = 1, eu = 1;
        if (at.col < F) {
            fd = load_cols<T, ALIGNED>(dh, at.col, F);
            qg = load_q(a.gate_q + at_q);
            qu = load_q(a.up_q + at_q);
            eg = a.gate_e[at_e];
            eu = a.up_e[at_e];
        }
        float g[8], u[8], d[8], h[8];
        to_floats<T, 8>(fd, d);
        held_values(qg, eg, g);
        held_values(qu, eu, u);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const float s = sigmoid<T>(g[i]), gs = g[i] * s, du = d[i] * gs;
            h[i] = gs * u[i];
            d[i] = d[i] * u[i] * (s * fmaf(g[i], 1.f - s, 1.f));
            u[i] = du;
        }
        store_cols<T, ALIGNED>(dgate, at.col, F, d);
        store_cols<T, ALIGNED>(dup, at.col, F, u);
        if (a.h) store_cols<T, ALIGNED>(out, at.col, F, h);
        if (a.h_q) {
#pragma unroll
            for (int i = 0; i < 8; ++i) h[i] = at.col + i < F ? to_float<T>(from_float<T>(h[i])) : 0.f;     // the values h_out holds
            store_held<ALIGNED>(a.h_q + at_q - at.col, a.h_e + t * a.lde, at.col, F, h);
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
