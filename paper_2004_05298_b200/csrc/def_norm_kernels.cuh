// Norms before and after a block, fused with its gate and residual scale (see include/def_train.h).
#pragma once

#include "def_train_common.cuh"

namespace deft {

struct Held { int8_t *q; uint8_t *e; };                       // a checkpoint to write; q NULL: none
struct HeldIn { const int8_t *q; const uint8_t *e; };         // a checkpoint to read

struct NormForward {
    const void *h, *b;
    void *h_out, *n_out;
    int64_t ldh, ldb, ldho, ldn;         // in elements
    const float *w_post, *gate, *w_pre;
    float *rstd_post, *rstd_pre;
    Held hb, hh, hn;
    int64_t T, C, rows_per_group, ldq, lde;
    float res_scale, eps, inv_C;
};

// One CTA per row; the row stays in registers between its two norms.
template <typename T, int V, int THREADS, int ITERS>
__global__ void __launch_bounds__(THREADS) norm_forward_kernel(const NormForward a) {
    __shared__ float scratch[2][32];
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        float h[ITERS][V];
        const T *hr = (const T *)a.h + t * a.ldh;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * THREADS + (int)threadIdx.x) * V;
            if (col < a.C) load_floats<T, V>(hr + col, h[it]);
            else
                for (int i = 0; i < V; ++i) h[it][i] = 0.f;
        }
        float sum = 0.f;
        if (a.b) {
            float b[ITERS][V];
            const T *br = (const T *)a.b + t * a.ldb;
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int col = (it * THREADS + (int)threadIdx.x) * V;
                if (col < a.C) load_floats<T, V>(br + col, b[it]);
                else
                    for (int i = 0; i < V; ++i) b[it][i] = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) sum = fmaf(b[it][i], b[it][i], sum);
            }
            if (a.hb.q)
#pragma unroll
                for (int it = 0; it < ITERS; ++it) {
                    const int col = (it * THREADS + (int)threadIdx.x) * V;
                    store_held<V>(a.hb.q + t * a.ldq, a.hb.e + t * a.lde, col, col < a.C, b[it]);
                }
            sum = cta_sum<THREADS>(sum, scratch[0]);
            const float r = rsqrtf(fmaf(sum, a.inv_C, a.eps));
            if (threadIdx.x == 0) a.rstd_post[t] = r;
            const float *gate = a.gate ? a.gate + t / a.rows_per_group * a.C : nullptr;
            T *ho = (T *)a.h_out + t * a.ldho;
            sum = 0.f;
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int col = (it * THREADS + (int)threadIdx.x) * V;
                if (col < a.C) {
                    float w[V], g[V];
                    load_params<V>(a.w_post + col, w);
                    if (gate) {
                        load_params<V>(gate + col, g);
#pragma unroll
                        for (int i = 0; i < V; ++i) w[i] *= g[i];
                    }
#pragma unroll
                    for (int i = 0; i < V; ++i) h[it][i] = fmaf(b[it][i] * r, w[i], a.res_scale * h[it][i]);
                    store_floats<T, V>(ho + col, h[it]);
                }
#pragma unroll
                for (int i = 0; i < V; ++i) sum = fmaf(h[it][i], h[it][i], sum);
            }
            if (a.hh.q)
#pragma unroll
                for (int it = 0; it < ITERS; ++it) {
                    const int col = (it * THREADS + (int)threadIdx.x) * V;
                    float x[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) x[i] = to_float<T>(from_float<T>(h[it][i]));   // h' as stored
                    store_held<V>(a.hh.q + t * a.ldq, a.hh.e + t * a.lde, col, col < a.C, x);
                }
        } else {
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
#pragma unroll
                for (int i = 0; i < V; ++i) sum = fmaf(h[it][i], h[it][i], sum);
            if (a.hh.q)
#pragma unroll
                for (int it = 0; it < ITERS; ++it) {
                    const int col = (it * THREADS + (int)threadIdx.x) * V;
                    store_held<V>(a.hh.q + t * a.ldq, a.hh.e + t * a.lde, col, col < a.C, h[it]);
                }
        }
        sum = cta_sum<THREADS>(sum, scratch[1]);
        const float r = rsqrtf(fmaf(sum, a.inv_C, a.eps));
        if (threadIdx.x == 0) a.rstd_pre[t] = r;
        T *no = (T *)a.n_out + t * a.ldn;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * THREADS + (int)threadIdx.x) * V;
            float n[V];
#pragma unroll
            for (int i = 0; i < V; ++i) n[i] = 0.f;
            if (col < a.C) {
                float w[V];
                load_params<V>(a.w_pre + col, w);
#pragma unroll
                for (int i = 0; i < V; ++i) n[i] = h[it][i] * r * w[i];
                store_floats<T, V>(no + col, n);
            }
            if (a.hn.q) {
#pragma unroll
                for (int i = 0; i < V; ++i) n[i] = to_float<T>(from_float<T>(n[i]));           // n as stored
                store_held<V>(a.hn.q + t * a.ldq, a.hn.e + t * a.lde, col, col < a.C, n);
            }
        }
        if (THREADS > 32 && !a.b) __syncthreads();   // one sum per row: scratch[1] is rewritten by the next
    }
}

struct NormBackward {
    const void *dn, *dh_in, *h, *b;
    HeldIn hh, hb;                       // checkpoints in place of h and b
    void *dh, *db;
    int64_t lddn, lddhi, ldh, ldb, lddh, lddb;
    const float *w_post, *gate, *w_pre, *rstd_post, *rstd_pre;
    float *partial;                      // [parts][2][C]: sums of dn x and of D y over a part's rows
    int64_t T, C, rows_per_group, ldq, lde;
    int64_t parts_per_group;
    float res_scale, inv_C;
};

// Part p = (group, slice of the group's rows): one CTA walks the slice, the column sums stay in registers.
template <typename T, int V, int THREADS, int ITERS>
__global__ void __launch_bounds__(THREADS) norm_backward_kernel(const NormBackward a) {
    __shared__ float scratch[2][32];
    const int64_t group = blockIdx.x / a.parts_per_group, slice = blockIdx.x % a.parts_per_group;
    const int64_t first = group * a.rows_per_group + a.rows_per_group * slice / a.parts_per_group;
    const int64_t last = group * a.rows_per_group + a.rows_per_group * (slice + 1) / a.parts_per_group;
    const bool has_b = a.b || a.hb.q;
    float sum_x[ITERS][V], sum_y[ITERS][V];
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
#pragma unroll
        for (int i = 0; i < V; ++i) sum_x[it][i] = sum_y[it][i] = 0.f;
    for (int64_t t = first; t < last; ++t) {
        const float r = a.rstd_pre[t];
        float D[ITERS][V], x[ITERS][V];
        float dot = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * THREADS + (int)threadIdx.x) * V;
#pragma unroll
            for (int i = 0; i < V; ++i) D[it][i] = x[it][i] = 0.f;
            if (col < a.C) {
                float w[V];
                load_floats<T, V>((const T *)a.dn + t * a.lddn + col, D[it]);
                if (a.hh.q) load_held<V>(a.hh.q + t * a.ldq, a.hh.e + t * a.lde, col, x[it]);
                else load_floats<T, V>((const T *)a.h + t * a.ldh + col, x[it]);
                load_params<V>(a.w_pre + col, w);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    x[it][i] *= r;
                    sum_x[it][i] = fmaf(D[it][i], x[it][i], sum_x[it][i]);
                    D[it][i] *= w[i];
                    dot = fmaf(D[it][i], x[it][i], dot);
                }
            }
        }
        dot = cta_sum<THREADS>(dot, scratch[0]) * a.inv_C;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * THREADS + (int)threadIdx.x) * V;
            if (col < a.C) {
                float in[V], out[V];
                if (a.dh_in) load_floats<T, V>((const T *)a.dh_in + t * a.lddhi + col, in);
                else
                    for (int i = 0; i < V; ++i) in[i] = 0.f;
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    D[it][i] = fmaf(r, fmaf(-x[it][i], dot, D[it][i]), in[i]);
                    out[i] = a.res_scale * D[it][i];
                }
                store_floats<T, V>((T *)a.dh + t * a.lddh + col, out);
            }
        }
        if (has_b) {
            const float rp = a.rstd_post[t];
            dot = 0.f;
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int col = (it * THREADS + (int)threadIdx.x) * V;
                if (col < a.C) {
                    float w[V], g[V];
                    if (a.hb.q) load_held<V>(a.hb.q + t * a.ldq, a.hb.e + t * a.lde, col, x[it]);
                    else load_floats<T, V>((const T *)a.b + t * a.ldb + col, x[it]);
                    load_params<V>(a.w_post + col, w);
                    if (a.gate) {
                        load_params<V>(a.gate + group * a.C + col, g);
#pragma unroll
                        for (int i = 0; i < V; ++i) w[i] *= g[i];
                    }
#pragma unroll
                    for (int i = 0; i < V; ++i) {
                        x[it][i] *= rp;
                        sum_y[it][i] = fmaf(D[it][i], x[it][i], sum_y[it][i]);
                        D[it][i] *= w[i];
                        dot = fmaf(D[it][i], x[it][i], dot);
                    }
                }
            }
            dot = cta_sum<THREADS>(dot, scratch[1]) * a.inv_C;
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int col = (it * THREADS + (int)threadIdx.x) * V;
                if (col < a.C) {
                    float out[V];
#pragma unroll
                    for (int i = 0; i < V; ++i) out[i] = rp * fmaf(-x[it][i], dot, D[it][i]);
                    store_floats<T, V>((T *)a.db + t * a.lddb + col, out);
                }
            }
        } else if constexpr (THREADS > 32) {
            __syncthreads();                         // scratch[0] is rewritten by the next row
        }
    }
    float *px = a.partial + (int64_t)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int col = (it * THREADS + (int)threadIdx.x) * V;
        if (col < a.C)
#pragma unroll
            for (int i = 0; i < V; ++i) {
                px[col + i] = sum_x[it][i];
                if (has_b) px[a.C + col + i] = sum_y[it][i];
            }
    }
}

// The parts' sums, in the order of the parts: dw_pre; and per group S = sum D y, from which dgate = w_post S and
// dw_post = sum over groups of gate S.  CTA: 32 columns by 32 slices of the parts.
__global__ void __launch_bounds__(1024) norm_reduce_kernel(const float *__restrict__ partial, const float *__restrict__ w_post,
                                                           const float *__restrict__ gate, int64_t C, int64_t groups,
                                                           int64_t parts_per_group, int has_b, int accumulate,
                                                           float *dw_post, float *dgate, float *dw_pre) {
    __shared__ float tile[32][33];
    const int64_t col = (int64_t)blockIdx.x * 32 + threadIdx.x;
    const bool live = col < C;
    auto total = [&](int64_t first, int64_t count, int which) {      // sum over parts [first, first + count); in row 0
        float s = 0.f;
        if (live)
            for (int64_t p = threadIdx.y; p < count; p += 32) s += partial[((first + p) * 2 + which) * C + col];
        tile[threadIdx.y][threadIdx.x] = s;
        __syncthreads();
        s = 0.f;
        if (threadIdx.y == 0)
            for (int i = 0; i < 32; ++i) s += tile[i][threadIdx.x];
        __syncthreads();
        return s;
    };
    const float x = total(0, groups * parts_per_group, 0);
    const bool writer = live && threadIdx.y == 0;
    if (writer) dw_pre[col] = accumulate ? dw_pre[col] + x : x;
    if (!has_b) return;
    float w = 0.f;
    if (gate && groups >= 32) {                       // many groups: a thread sums whole groups
        for (int64_t g = threadIdx.y; live && g < groups; g += 32) {
            float s = 0.f;
            for (int64_t p = 0; p < parts_per_group; ++p) s += partial[((g * parts_per_group + p) * 2 + 1) * C + col];
            const float d = w_post[col] * s;
            dgate[g * C + col] = accumulate ? dgate[g * C + col] + d : d;
            w = fmaf(gate[g * C + col], s, w);
        }
        tile[threadIdx.y][threadIdx.x] = w;
        __syncthreads();
        w = 0.f;
        if (threadIdx.y == 0)
            for (int i = 0; i < 32; ++i) w += tile[i][threadIdx.x];
    } else {
        for (int64_t g = 0; g < groups; ++g) {
            const float s = total(g * parts_per_group, parts_per_group, 1);
            if (writer && gate) {
                const float d = w_post[col] * s;
                dgate[g * C + col] = accumulate ? dgate[g * C + col] + d : d;
                w = fmaf(gate[g * C + col], s, w);
            } else {
                w += s;
            }
        }
    }
    if (writer) dw_post[col] = accumulate ? dw_post[col] + w : w;
}

}  // namespace deft
