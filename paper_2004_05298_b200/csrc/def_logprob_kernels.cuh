// Token log probabilities with entropy and top alternatives, and their gradient (see include/def_train.h).
#pragma once

#include "def_train_common.cuh"

namespace deft {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// A logit at or below this is masked; -infinity and the lowest value of bf16 and fp32 are.
constexpr float kMasked = -1e30f;

// Running statistics of part of a row, relative to its maximum m:  s = sum 2^y,  u = sum y 2^y with
// y = (x - m) log2(e).  The difference is taken first: it is small where it counts, whatever m is.
struct Stats {
    float m, s, u;
};
__device__ __forceinline__ Stats empty_stats() { return {kMasked, 0.f, 0.f}; }
// y is held at -1e4, where 2^y is 0 and 0 times y still is.
__device__ __forceinline__ float exponent(float x, float m) { return max_nan((x - m) * kLog2e, -1e4f); }
__device__ __forceinline__ void rebase(Stats &a, float m) {              // m >= a.m
    const float d = exponent(a.m, m), f = exp2_fast(d);
    a.u = fmaf(d, a.s, a.u) * f;
    a.s *= f;
    a.m = m;
}
__device__ __forceinline__ Stats join(Stats a, Stats b) {
    const float m = fmaxf(a.m, b.m);
    rebase(a, m);
    rebase(b, m);
    return {m, a.s + b.s, a.u + b.u};
}
__device__ __forceinline__ Stats shfl_xor(const Stats &a, int lane) {
    return {__shfl_xor_sync(0xffffffffu, a.m, lane), __shfl_xor_sync(0xffffffffu, a.s, lane),
            __shfl_xor_sync(0xffffffffu, a.u, lane)};
}

// ---------------------------------------------------------------------------
// Alternatives.  Keys order (value descending, index ascending) as unsigned 64-bit integers, the largest first; keys
// of a row are all different.  0 stands for no element.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint64_t make_key(float v, int64_t index) {
    if (!(v > -INFINITY)) v = -INFINITY;              // a NaN ranks with -infinity
    v += 0.f;                                         // -0 ties with +0
    const uint32_t b = __float_as_uint(v), ordered = b & 0x80000000u ? ~b : b | 0x80000000u;
    return (uint64_t)ordered << 32 | (uint32_t)~(uint32_t)index;
}
__device__ __forceinline__ int64_t key_index(uint64_t key) { return (int64_t)(uint32_t)~(uint32_t)key; }
__device__ __forceinline__ float key_value(uint64_t key) {
    const uint32_t o = (uint32_t)(key >> 32);
    return __uint_as_float(o & 0x80000000u ? o & 0x7fffffffu : ~o);
}

// Bitonic sort of a warp's 32 keys, largest in lane 0.
__device__ __forceinline__ uint64_t exchange(uint64_t key, int distance, bool keep_max) {
    const uint64_t other = __shfl_xor_sync(0xffffffffu, key, distance);
    return (key > other) == keep_max ? key : other;
}
__device__ __forceinline__ uint64_t warp_merge_down(uint64_t key) {          // a bitonic sequence -> descending
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) key = exchange(key, d, (lane & d) == 0);
    return key;
}
__device__ __forceinline__ uint64_t warp_sort(uint64_t key) {
    const int lane = threadIdx.x & 31;
#pragma unroll
    for (int size = 2; size < 32; size <<= 1)
#pragma unroll
        for (int d = size / 2; d > 0; d >>= 1) key = exchange(key, d, ((lane & d) == 0) == ((lane & size) == 0));
    return warp_merge_down(key);
}
// The 32 largest of two descending lists.
__device__ __forceinline__ uint64_t warp_join(uint64_t a, uint64_t b) {
    const uint64_t r = __shfl_sync(0xffffffffu, b, 31 - (threadIdx.x & 31));
    return warp_merge_down(a > r ? a : r);
}
// The 32 largest of all warps' descending lists, in warp 0 (and in lists[0]).
template <int WARPS> __device__ __forceinline__ uint64_t cta_join(uint64_t list, uint64_t (*lists)[32]) {
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    __syncthreads();
    lists[warp][lane] = list;
#pragma unroll
    for (int step = 1; step < WARPS; step <<= 1) {
        __syncthreads();
        if (warp % (2 * step) == 0) {
            list = warp_join(list, lists[warp + step][lane]);
            lists[warp][lane] = list;
        }
    }
    __syncthreads();
    return list;
}

struct LogprobForward {
    const void *x;
    int64_t ldx, T, V;
    const int64_t *y;
    float *logp, *entropy, *lse;
    int64_t *top_ids;
    float *top_logp;
    int top;
};

// One CTA per row.  Thread i reads chunks i, i + THREADS, ... of V elements and keeps the running maximum, sum and
// weighted sum, and which chunk first held its maximum.
//
// Alternatives: an element among the row's `top` largest lies in the list of a thread whose own largest element is
// also among the `top` largest; at most `top` threads have one.  So the threads' maxima are ranked, and only the
// elements of the `top` best threads are looked at again (they are few, and in the L2).
template <typename T, int V, int THREADS>
__global__ void __launch_bounds__(THREADS) logprob_forward_kernel(const LogprobForward a) {
    constexpr int kWarps = THREADS / 32;
    __shared__ Stats parts[32];
    __shared__ uint64_t lists[kWarps][32];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int64_t chunks = a.V / V;                   // V divides a.V on this path
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T *row = (const T *)a.x + t * a.ldx;
        Stats st = empty_stats();
        int64_t best = threadIdx.x;
        for (int64_t c = threadIdx.x; c < chunks; c += THREADS) {
            float v[V];
            load_floats<T, V>(row + c * V, v);
            float top = v[0];
#pragma unroll
            for (int i = 1; i < V; ++i) top = fmaxf(top, v[i]);
            if (top > st.m) {
                rebase(st, top);
                best = c;
            }
            if (st.m == kMasked) {                    // nothing but masked logits, or NaN, so far
#pragma unroll
                for (int i = 0; i < V; ++i)
                    if (v[i] != v[i]) st.s = st.u = NAN;
            } else {
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    const float y = exponent(v[i], st.m), p = exp2_fast(y);
                    st.s += p;
                    st.u = fmaf(p, y, st.u);
                }
            }
        }
        const float own_max = st.m;
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) st = join(st, shfl_xor(st, d));
        if (lane == 0) parts[warp] = st;
        __syncthreads();
        st = lane < kWarps ? parts[lane] : empty_stats();
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) st = join(st, shfl_xor(st, d));
        const bool none = st.m == kMasked && st.s == 0.f;            // the row is masked throughout
        const float log_s = none ? 0.f : logf(st.s), m = none ? INFINITY : st.m;     // log p = (x - m) - log s
        if (threadIdx.x == 0) {
            a.lse[2 * t] = none ? -INFINITY : st.m;
            a.lse[2 * t + 1] = log_s;
            a.entropy[t] = none ? 0.f : log_s - st.u / st.s * kLn2;
            const int64_t y = a.y[t];
            a.logp[t] = y < 0 ? 0.f : y >= a.V ? NAN : none ? -INFINITY : (to_float<T>(row[y]) - m) - log_s;
        }
        if (a.top == 0) {
            __syncthreads();                          // parts
            continue;
        }
        // the best element of every thread
        uint64_t key = 0;
        if (own_max > kMasked) {
#pragma unroll
            for (int i = V - 1; i >= 0; --i) {
                const float v = to_float<T>(row[best * V + i]);
                if (v == own_max) key = make_key(v, best * V + i);
            }
        } else {                                      // masked logits order like others: look at all of them
            for (int64_t c = threadIdx.x; c < chunks; c += THREADS)
                for (int i = 0; i < V; ++i) {
                    const uint64_t k = make_key(to_float<T>(row[c * V + i]), c * V + i);
                    if (k > key) key = k;
                }
        }
        uint64_t list = cta_join<kWarps>(warp_sort(key), lists);
        const uint64_t threshold = lists[0][a.top - 1];              // at least `top` elements are this good
        uint64_t owner = lists[0][lane];
        __syncthreads();
        list = 0;
        for (int k = warp; k < a.top; k += kWarps) {
            const uint64_t o = __shfl_sync(0xffffffffu, owner, k);
            if (o == 0) break;
            const int64_t first = key_index(o) / V % THREADS;
            for (int64_t c0 = first; c0 < chunks; c0 += (int64_t)THREADS * 32) {
                const int64_t c = c0 + (int64_t)lane * THREADS;
                float v[V];
#pragma unroll
                for (int i = 0; i < V; ++i) v[i] = 0.f;
                if (c < chunks) load_floats<T, V>(row + c * V, v);
#pragma unroll
                for (int i = 0; i < V; ++i) {
                    uint64_t cand = c < chunks ? make_key(v[i], c * V + i) : 0;
                    if (cand < threshold) cand = 0;
                    if (__any_sync(0xffffffffu, cand > __shfl_sync(0xffffffffu, list, 31))) list = warp_join(list, warp_sort(cand));
                }
            }
        }
        list = cta_join<kWarps>(list, lists);
        if (warp == 0 && lane < a.top) {
            a.top_ids[t * a.top + lane] = key_index(list);
            a.top_logp[t * a.top + lane] = none ? -INFINITY : (key_value(list) - m) - log_s;
        }
        __syncthreads();
    }
}

struct LogprobBackward {
    const void *x;
    void *dx;
    int64_t ldx, lddx, T, V;
    const int64_t *y, *top_ids;
    const float *lse, *entropy, *dlogp, *dentropy, *dtop;
    int top;
};

// One CTA per row.  dx_j = -p_j (G + dH (log p_j + H)) everywhere; the at most 33 elements that also get a term of their
// own (the target, the alternatives) are worked out first, from the logits, and stored last, so dx may be x.
template <typename T, int V, int THREADS>
__global__ void __launch_bounds__(THREADS) logprob_backward_kernel(const LogprobBackward a) {
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        const T *row = (const T *)a.x + t * a.ldx;
        T *out = (T *)a.dx + t * a.lddx;
        const float m = a.lse[2 * t], log_s = a.lse[2 * t + 1], H = a.entropy[t], dH = a.dentropy ? a.dentropy[t] : 0.f;
        const int64_t y = a.y[t];
        const float dl = a.dlogp && y >= 0 ? (y < a.V ? a.dlogp[t] : NAN) : 0.f;
        float G = dl;
        for (int i = 0; i < a.top; ++i) G += a.dtop[t * a.top + i];
        const bool none = m == -INFINITY;
        auto spread = [&](float x) {                  // -p (G + dH (log p + H)); 0 where p is 0
            const float lp = (x - m) - log_s, p = exp2_fast(lp * kLog2e);
            const float g = -p * fmaf(dH, lp + H, G);
            return none || p == 0.f ? 0.f : g;
        };
        // Thread k < top owns alternative k, thread `top` the target; the first owner of an index sums its terms.
        int64_t at = -1;
        float special = 0.f;
        if (threadIdx.x <= a.top) {
            const int k = threadIdx.x;
            at = k < a.top ? a.top_ids[t * a.top + k] : y;
            if (at < 0 || at >= a.V) at = -1;
            for (int i = 0; i < k && at >= 0; ++i)
                if (a.top_ids[t * a.top + i] == at) at = -1;
            if (at >= 0) {
                float own = 0.f;
                for (int i = 0; i < a.top; ++i)
                    if (a.top_ids[t * a.top + i] == at) own += a.dtop[t * a.top + i];
                if (y == at) own += dl;
                special = none ? 0.f : spread(to_float<T>(row[at])) + own;
            }
        }
        __syncthreads();
        for (int64_t c = threadIdx.x; c < a.V / V; c += THREADS) {
            float v[V];
            load_floats<T, V>(row + c * V, v);
#pragma unroll
            for (int i = 0; i < V; ++i) v[i] = spread(v[i]);
            store_floats<T, V>(out + c * V, v);
        }
        __syncthreads();
        if (at >= 0) out[at] = from_float<T>(special);
    }
}

}  // namespace deft
