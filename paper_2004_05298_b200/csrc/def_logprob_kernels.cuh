// Token log probabilities with entropy and top alternatives, and their gradient (see include/def_train.h).
#pragma once

#include "def_sm100.cuh"
#include "def_train_common.cuh"

namespace deft {

constexpr float kLog2e = 1.4426950408889634f, kLn2 = 0.6931471805599453f;

__device__ __forceinline__ float exp2_fast(float x) {
    float y;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
    return y;
}
// A logit at or below this (about -1e30, and exact in bf16) is masked; -infinity and the lowest value of bf16 and fp32 are.
constexpr float kMasked = -0x1.92p+99f;

// Exponents are taken relative to the maximum m:  y = (x - base) log2(e) - r.  Where |m| < kFar, base is 0 and r is m log2(e)
// rounded to an integer: the product is not rounded before r is taken from it, so that y is as good as if m had been
// subtracted first, in one operation.  A larger product is itself too coarse to be rounded to an integer (2^-24 of it
// reaches 128 at 1.5e9), so there base is m and r is 0: x - m is exact where x is near m, and where it is not, 2^y is 0.
constexpr float kFar = 0x1p20f;
__device__ __forceinline__ bool is_far(float m) { return !(fabsf(m) < kFar); }
__device__ __forceinline__ float base_of(float m) { return is_far(m) ? m : 0.f; }
__device__ __forceinline__ float reference_of(float m) { return is_far(m) ? 0.f : rintf(m * kLog2e); }

// Running statistics of part of a row:  s = sum 2^y,  u = sum y 2^y, m the maximum so far and r = reference_of(m).
struct Stats {
    float m, r, s, u;
};
__device__ __forceinline__ Stats empty_stats() { return {kMasked, 0.f, 0.f, 0.f}; }
// y is held at -1e4, where 2^y is 0 and 0 times y still is.
__device__ __forceinline__ void rebase(Stats &a, float m, float r) {     // m >= a.m: exponents shrink, or grow by less than 1
    const float d = max_nan(fmaf(base_of(a.m) - base_of(m), kLog2e, a.r - r), -1e4f), f = exp2_fast(d);
    a.u = fmaf(d, a.s, a.u) * f;
    a.s *= f;
    a.m = m;
    a.r = r;
}
__device__ __forceinline__ Stats join(Stats a, Stats b) {
    const float m = fmaxf(a.m, b.m), r = a.m >= b.m ? a.r : b.r;
    rebase(a, m, r);
    rebase(b, m, r);
    return {m, r, a.s + b.s, a.u + b.u};
}
__device__ __forceinline__ Stats shfl_xor(const Stats &a, int lane) {
    return {__shfl_xor_sync(0xffffffffu, a.m, lane), __shfl_xor_sync(0xffffffffu, a.r, lane), __shfl_xor_sync(0xffffffffu, a.s, lane),
            __shfl_xor_sync(0xffffffffu, a.u, lane)};
}

// ---------------------------------------------------------------------------
// Alternatives.  Keys order (value descending, index ascending) as unsigned 64-bit integers, the largest first; keys
// of a row are all different.  0 stands for no element.
// ---------------------------------------------------------------------------
__device__ __forceinline__ uint32_t order_bits(float v) {
    if (!(v > -INFINITY)) v = -INFINITY;              // a NaN ranks with -infinity
    v += 0.f;                                         // -0 ties with +0
    const uint32_t b = __float_as_uint(v);
    return b & 0x80000000u ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ uint64_t make_key(float v, int64_t index) { return (uint64_t)order_bits(v) << 32 | (uint32_t)~(uint32_t)index; }
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

// A row as chunks of 8 elements that start on 16-byte boundaries, wherever the row starts: chunks [0, body), then chunk
// `body` for the elements before the first of them and chunk body + 1 for those behind the last.
template <typename T> struct RowChunks {
    const T *row;
    int head, body, tail;
    __device__ RowChunks(const T *p, int V) : row(p) {
        const int off = (int)((16u - ((uint32_t)(uintptr_t)p & 15u)) & 15u) / (int)sizeof(T);
        head = off < V ? off : V;
        body = (V - head) / 8;
        tail = V - head - body * 8;
    }
    __device__ int start(int c) const { return c < body ? head + 8 * c : c == body ? 0 : head + 8 * body; }
    __device__ int count(int c) const { return c < body ? 8 : c == body ? head : tail; }
    // Where the thread that has element `index` begins, threads taking chunks G apart; the first two also have the ends.
    __device__ int first_chunk(int index, int G) const {
        const int past = index - head;
        return past < 0 ? 0 : past >= 8 * body ? 1 : past / 8 % G;
    }
    __device__ Frag<T, 8> wide(int c) const { return load_frag<T, 8>(row + head + 8 * c); }
    __device__ void any(int c, float (&v)[8]) const {                 // -infinity where there is no element
        if (c < body) {
            to_floats<T, 8>(wide(c), v);
        } else {
            const int n = count(c), at = start(c);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = i < n ? to_float<T>(row[at + i]) : -INFINITY;
        }
    }
};

__device__ __forceinline__ float largest(const float (&v)[8]) {
    return fmaxf(fmaxf(fmaxf(v[0], v[1]), fmaxf(v[2], v[3])), fmaxf(fmaxf(v[4], v[5]), fmaxf(v[6], v[7])));
}
template <typename T> struct Two;
template <> struct Two<__nv_bfloat16> { using type = __nv_bfloat162; };
template <> struct Two<__half> { using type = __half2; };
// The largest of N chunks as loaded; NaN does not count.
template <int N> __device__ __forceinline__ float largest(const Frag<float, 8> (&f)[N]) {
    float top = -INFINITY;
#pragma unroll
    for (int k = 0; k < N; ++k) top = fmaxf(top, largest(f[k].v));
    return top;
}
template <int N, typename T> __device__ __forceinline__ float largest(const Frag<T, 8> (&f)[N]) {
    using T2 = typename Two<T>::type;
    T2 w[4 * N];
    memcpy(w, f, sizeof(w));
#pragma unroll
    for (int n = 4 * N; n > 1; n = (n + 1) / 2)
#pragma unroll
        for (int i = 0; i < n / 2; ++i) w[i] = __hmax2(w[i], w[n - 1 - i]);
    return fmaxf(to_float<T>(w[0].x), to_float<T>(w[0].y));
}

// A thread's running statistics, the sums in two halves.
struct Running {
    float m = kMasked, r = 0.f;
    Pair s = {0}, u = {0};
    __device__ __forceinline__ void reach(float top) {            // before adding elements of which `top` is the largest
        if (top > m) {
            Stats a, b;
            a.m = b.m = m;
            a.r = b.r = r;
            split_pair(s, a.s, b.s);
            split_pair(u, a.u, b.u);
            m = top;
            r = reference_of(top);
            rebase(a, m, r);
            rebase(b, m, r);
            s = make_pair(a.s, b.s);
            u = make_pair(a.u, b.u);
        }
    }
    __device__ __forceinline__ void add(const float (&v)[8]) {
        const Pair l = make_pair(kLog2e, kLog2e), minus_r = make_pair(-r, -r);
#pragma unroll
        for (int i = 0; i < 8; i += 2) {
            float y0, y1;
            split_pair(pair_fma(make_pair(v[i], v[i + 1]), l, minus_r), y0, y1);
            y0 = max_nan(y0, -1e4f);
            y1 = max_nan(y1, -1e4f);
            const Pair p = make_pair(exp2_fast(y0), exp2_fast(y1));
            s = pair_add(s, p);
            u = pair_fma(p, make_pair(y0, y1), u);
        }
    }
    // What add() takes where m is far (r is 0 there).  m == kMasked: nothing but masked logits, or NaN, so far.
    __device__ __forceinline__ void from_base(float (&v)[8]) const {
#pragma unroll
        for (int i = 0; i < 8; ++i) v[i] = m != kMasked ? v[i] - m : v[i] == v[i] ? -INFINITY : v[i];
    }
    __device__ __forceinline__ Stats total() const {
        float s0, s1, u0, u1;
        split_pair(s, s0, s1);
        split_pair(u, u0, u1);
        return {m, r, s0 + s1, u0 + u1};
    }
};

// The k-th largest of 64 numbers, k in 1..32, found by one warp: the one that fewer than k exceed and at least k reach.
__device__ __forceinline__ uint32_t kth_of_64(const uint32_t *x, int k) {
    const int lane = threadIdx.x & 31;
    const uint32_t a = x[lane], b = x[lane + 32];
    int above_a = 0, from_a = 0, above_b = 0, from_b = 0;
#pragma unroll
    for (int i = 0; i < 64; i += 4) {
        const uint4 o = *reinterpret_cast<const uint4 *>(x + i);
        above_a += (o.x > a) + (o.y > a) + (o.z > a) + (o.w > a);
        from_a += (o.x >= a) + (o.y >= a) + (o.z >= a) + (o.w >= a);
        above_b += (o.x > b) + (o.y > b) + (o.z > b) + (o.w > b);
        from_b += (o.x >= b) + (o.y >= b) + (o.z >= b) + (o.w >= b);
    }
    const bool is_a = above_a < k && k <= from_a, is_b = above_b < k && k <= from_b;
    const uint32_t lanes = __ballot_sync(0xffffffffu, is_a || is_b);
    return __shfl_sync(0xffffffffu, is_a ? a : b, __ffs(lanes) - 1);
}

// A row is read by a cluster of `split` CTAs (one CTA where there are many rows).  Thread g of all their threads takes
// chunks g, g + G, ... and keeps the running maximum, sum and weighted sum.
//
// Alternatives: each CTA finds its own, and the CTAs' lists are joined at the end.  The threads are 64 groups; the top-th
// largest of the groups' maxima bounds the top-th largest element from below, and few elements are that large.  The
// threads that saw one are listed, their elements are read again by whole warps (they are few, and in the L2), and those
// that reach the bound are ranked by counting.  Where that does not settle it -- too many ties at the bound, too few
// logits above the masked ones -- the exact way does: an element among the `top` largest lies in the list of a thread whose
// own largest is among them too, so the threads' largest elements are ranked and the `top` best threads' elements merged.
// (4096 rows of 128000 bf16, top = 8: 332 us with the exact way alone, 217 like this, 205 without alternatives; the bytes
// take 162.  2048 threads per SM with two chunks ahead each: 254 us with 1024 threads and four.)
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, 2048 / THREADS) logprob_forward_kernel(const LogprobForward a, const int split) {
    constexpr int kWarps = THREADS / 32, kAhead = 2;
    __shared__ Stats parts[32];
    __shared__ Stats whole;
    __shared__ uint64_t lists[kWarps][32];
    __shared__ __align__(16) uint32_t group_max[64];
    __shared__ uint16_t owners[THREADS];
    __shared__ uint32_t found_bound;
    __shared__ int n_owners, n_found;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = split == 1 ? 0 : (int)(blockIdx.x % split), G = split * THREADS, g = rank * THREADS + threadIdx.x;
    const int V = (int)a.V;
    const int64_t t = blockIdx.x / split;
    const RowChunks<T> row((const T *)a.x + t * a.ldx, V);
    if (threadIdx.x == 0) n_owners = n_found = 0;
    Running run;
    float v[8];
    auto add_any = [&](int chunk) {
        row.any(chunk, v);
        run.reach(largest(v));
        if (is_far(run.m)) run.from_base(v);
        run.add(v);
    };
    int c = g;
    for (; c + (kAhead - 1) * G < row.body; c += kAhead * G) {
        Frag<T, 8> f[kAhead];
#pragma unroll
        for (int k = 0; k < kAhead; ++k) f[k] = row.wide(c + k * G);
        run.reach(largest<kAhead>(f));
        if (is_far(run.m)) {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                to_floats<T, 8>(f[k], v);
                run.from_base(v);
                run.add(v);
            }
        } else {
#pragma unroll
            for (int k = 0; k < kAhead; ++k) {
                to_floats<T, 8>(f[k], v);
                run.add(v);
            }
        }
    }
    for (; c < row.body; c += G) add_any(c);
    if (g < 2 && row.count(row.body + g)) add_any(row.body + g);
    Stats st = run.total();
    const float own_max = st.m;
    const uint32_t own_rank = order_bits(own_max);
    if (a.top > 0) {
        uint32_t most = own_rank;
#pragma unroll
        for (int d = 1; d < THREADS / 64; d <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
        if (threadIdx.x % (THREADS / 64) == 0) group_max[threadIdx.x / (THREADS / 64)] = most;
    }
#pragma unroll
    for (int d = 16; d > 0; d >>= 1) st = join(st, shfl_xor(st, d));
    if (lane == 0) parts[warp] = st;
    __syncthreads();
    if (warp == 0) {                                  // the statistics are the business of the first warp from here on
        st = lane < kWarps ? parts[lane] : empty_stats();
#pragma unroll
        for (int d = 16; d > 0; d >>= 1) st = join(st, shfl_xor(st, d));
    }
    uint64_t list = 0;
    if (a.top > 0) {
        if (warp == kWarps - 1) {
            const uint32_t b = kth_of_64(group_max, a.top);
            if (lane == 0) found_bound = b;
        }
        __syncthreads();
        const uint32_t bound = found_bound;
        uint64_t *found = &lists[0][0];               // room for THREADS keys
        if (bound > order_bits(kMasked)) {
            if (own_rank >= bound) owners[atomicAdd(&n_owners, 1)] = (uint16_t)threadIdx.x;
            __syncthreads();
            for (int k = warp; k < n_owners; k += kWarps) {
                const int from = rank * THREADS + owners[k];
                auto offer = [&](float x, int index) {
                    if (order_bits(x) >= bound) {
                        const int slot = atomicAdd(&n_found, 1);
                        if (slot < THREADS) found[slot] = make_key(x, index);
                    }
                };
                for (int chunk = from + lane * G; chunk < row.body; chunk += G * 32) {
                    float w[8];
                    row.any(chunk, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) offer(w[i], row.head + 8 * chunk + i);
                }
                if (from < 2 && lane < row.count(row.body + from)) {
                    const int at = row.start(row.body + from) + lane;
                    offer(to_float<T>(row.row[at]), at);
                }
            }
            __syncthreads();
        }
        const int n = n_found;
        if (n > 0 && n <= THREADS) {                  // the same for all threads: n_found no longer changes
            uint64_t key = 0;
            int ahead = 0;
            if (threadIdx.x < n) {
                key = found[threadIdx.x];
                for (int i = 0; i < n; ++i) ahead += found[i] > key;
            }
            __syncthreads();
            if (threadIdx.x < 32) lists[0][threadIdx.x] = 0;
            __syncthreads();
            if (threadIdx.x < n && ahead < 32) lists[0][ahead] = key;
            __syncthreads();
            list = lists[0][lane];
        } else {
            uint64_t key = 0;                         // the best element of this thread
            auto look = [&](int chunk) {
                row.any(chunk, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    const uint64_t k = i < row.count(chunk) ? make_key(v[i], row.start(chunk) + i) : 0;
                    if (k > key) key = k;
                }
            };
            for (int chunk = g; chunk < row.body; chunk += G) look(chunk);
            if (g < 2) look(row.body + g);
            cta_join<kWarps>(warp_sort(key), lists);
            const uint64_t threshold = lists[0][a.top - 1];          // 0, or `top` elements of this CTA are this good
            const uint64_t best = lists[0][lane];
            __syncthreads();
            for (int k = warp; k < a.top; k += kWarps) {
                const uint64_t o = __shfl_sync(0xffffffffu, best, k);
                if (o == 0) break;
                const int from = row.first_chunk((int)key_index(o), G);
                auto offer = [&](uint64_t cand) {
                    if (cand < threshold) cand = 0;
                    if (__any_sync(0xffffffffu, cand > __shfl_sync(0xffffffffu, list, 31))) list = warp_join(list, warp_sort(cand));
                };
                for (int c0 = from; c0 < row.body; c0 += G * 32) {
                    const int chunk = c0 + lane * G;
                    const bool there = chunk < row.body;
                    float w[8];
                    row.any(there ? chunk : row.body + 1, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) offer(there ? make_key(w[i], row.start(chunk) + i) : 0);
                }
                if (from < 2) {
                    const int at = row.start(row.body + from) + lane;
                    offer(lane < row.count(row.body + from) ? make_key(to_float<T>(row.row[at]), at) : 0);
                }
            }
            list = cta_join<kWarps>(list, lists);
        }
    }
    if (split > 1) {                                  // the first CTA of the cluster joins what the others found
        if (threadIdx.x == 0) whole = st;
        cluster_sync();
        if (rank == 0 && warp == 0) {
            for (int r = 1; r < split; ++r) {
                const uint32_t at = cluster_address(smem_address(&whole), r);
                const Stats other = {cluster_load(at), cluster_load(at + 4), cluster_load(at + 8), cluster_load(at + 12)};
                st = join(st, other);
                if (a.top > 0) list = warp_join(list, cluster_load64(cluster_address(smem_address(&lists[0][lane]), r)));
            }
        }
        cluster_sync();
        if (rank != 0) return;
    }
    if (warp != 0) return;
    const bool none = st.m == kMasked && st.s == 0.f;                // the row is masked throughout
    const float m = none ? INFINITY : st.m;                          // log p = (x - m) - log_s
    const float log2_s = log2f(st.s), shift = is_far(st.m) ? 0.f : fmaf(-st.m, kLog2e, st.r);   // of the sum as kept; what m's exponent lacks to 0
    const float log_s = none ? 0.f : (log2_s + shift) * kLn2;
    if (threadIdx.x == 0) {
        a.lse[2 * t] = none ? -INFINITY : st.m;
        a.lse[2 * t + 1] = log_s;
        a.entropy[t] = none ? 0.f : (log2_s - st.u / st.s) * kLn2;
        const int64_t y = a.y[t];
        a.logp[t] = y < 0 ? 0.f : y >= a.V ? NAN : none ? -INFINITY : (to_float<T>(row.row[y]) - m) - log_s;
    }
    if (lane < a.top) {
        a.top_ids[t * a.top + lane] = key_index(list);
        a.top_logp[t * a.top + lane] = none ? -INFINITY : (key_value(list) - m) - log_s;
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

// A row is written by `split` CTAs, their chunks interleaved.  dx_j = -p_j (G + dH (log p_j + H)) everywhere; the at most 33
// elements that also get a term of their own (the target, the alternatives) are worked out first, from the logits, by the
// CTA whose chunk they lie in, and stored last, so dx may be x.
template <typename T, int THREADS>
__global__ void __launch_bounds__(THREADS, 1536 / THREADS) logprob_backward_kernel(const LogprobBackward a, const int split) {
    constexpr int kAhead = 2;
    const int rank = (int)(blockIdx.x % split), G = split * THREADS, lane = threadIdx.x & 31;
    const int64_t t = blockIdx.x / split;
    const RowChunks<T> row((const T *)a.x + t * a.ldx, (int)a.V);
    T *out = (T *)a.dx + t * a.lddx;
    const bool wide = (((uintptr_t)row.row ^ (uintptr_t)out) & 15u) == 0;
    const float m = a.lse[2 * t], log_s = a.lse[2 * t + 1], H = a.entropy[t], dH = a.dentropy ? a.dentropy[t] : 0.f;
    const int64_t y = a.y[t];
    const float dl = a.dlogp && y >= 0 ? (y < a.V ? a.dlogp[t] : NAN) : 0.f;
    const float dt = lane < a.top ? a.dtop[t * a.top + lane] : 0.f;
    const bool none = m == -INFINITY;
    // log2 p = ((x - base) log2(e) - r) - shift; G + dH (log p + H) = slope log2 p + rise
    const float base = base_of(m), r = reference_of(m), shift = fmaf(m - base, kLog2e, -r) + log_s * kLog2e;
    const float slope = dH * kLn2, rise = fmaf(dH, H, dl + warp_sum(dt));
    auto spread = [&](float x) {
        const float z = max_nan(fmaf(x - base, kLog2e, -r) - shift, -1e4f);      // p is 0 there, and 0 times the rest
        return none ? 0.f : -exp2_fast(z) * fmaf(slope, z, rise);
    };
    // Thread k < top owns alternative k, thread `top` the target; the first owner of an index sums its terms.
    int64_t at = -1;
    float special = 0.f;
    if (threadIdx.x <= a.top) {
        const int k = threadIdx.x;
        at = k < a.top ? a.top_ids[t * a.top + k] : y;
        if (at < 0 || at >= a.V) at = -1;
        if (at >= 0 && row.first_chunk((int)at, G) / THREADS != rank) at = -1;
        for (int i = 0; i < k && at >= 0; ++i)
            if (a.top_ids[t * a.top + i] == at) at = -1;
        if (at >= 0) {
            float own = 0.f;
            for (int i = 0; i < a.top; ++i)
                if (a.top_ids[t * a.top + i] == at) own += a.dtop[t * a.top + i];
            if (y == at) own += dl;
            special = none ? 0.f : spread(to_float<T>(row.row[at])) + own;
        }
    }
    __syncthreads();
    const int g = rank * THREADS + threadIdx.x;
    int c = g;
    if (wide) {
        auto put = [&](int chunk, const Frag<T, 8> &f) {
            float v[8];
            to_floats<T, 8>(f, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = spread(v[i]);
            store_floats<T, 8>(out + row.head + 8 * chunk, v);
        };
        for (; c + (kAhead - 1) * G < row.body; c += kAhead * G) {
            Frag<T, 8> f[kAhead];
#pragma unroll
            for (int k = 0; k < kAhead; ++k) f[k] = row.wide(c + k * G);
#pragma unroll
            for (int k = 0; k < kAhead; ++k) put(c + k * G, f[k]);
        }
        for (; c < row.body; c += G) put(c, row.wide(c));
    } else {
        for (; c < row.body; c += G) {
            float v[8];
            row.any(c, v);
#pragma unroll
            for (int i = 0; i < 8; ++i) out[row.start(c) + i] = from_float<T>(spread(v[i]));
        }
    }
    if (g < 2)
        for (int i = 0; i < row.count(row.body + g); ++i) {
            const int j = row.start(row.body + g) + i;
            out[j] = from_float<T>(spread(to_float<T>(row.row[j])));
        }
    __syncthreads();
    if (at >= 0) out[at] = from_float<T>(special);
}

}  // namespace deft
