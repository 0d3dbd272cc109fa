// Gated linear recurrence over tokens, and its backward pass (see include/def_train.h).
//
//     c_t = 1 / (1 + exp(g_t)),  a_t = 1 - c_t,   h_t = a_t h_{t-1} + c_t x_t
//     mu_t = a_t (dy_t + mu_{t+1}) = the gradient that reaches h_{t-1};  lambda_t = dy_t + mu_{t+1}
//
// Both are the same scan, s_i = a_i s_{i-1} + b_i, one in time's direction, one against it.  A run of steps maps the state
// before it to the one behind it as s -> P s + L; two runs join as (P2 P1, P2 L1 + L2).  A warp takes kRun steps of 32 V
// channels, which it reads once and keeps in registers: first (P, L) of its run, then, once the runs before are known, the
// states themselves.  The eight warps of a CTA hold consecutive runs, the CTAs of a cluster consecutive blocks; they hand each
// other their blocks' (P, L) through distributed shared memory, so that every input is read once however long the sequence.
// Every sum is taken in one order.
//
// Sequences lie one behind another; at a sequence's first step the state is replaced, P becomes -0 ("nothing from before":
// with a zero of that sign no infinity or NaN of another sequence gets in).
#pragma once

#include "def_sm100.cuh"
#include "def_train_common.cuh"

namespace deft {

constexpr int kRun = 16, kRecWarps = 8, kRecSteps = kRun * kRecWarps;   // steps of a warp; of a CTA's block
constexpr int kMostCluster = 8, kMostParts = 256;                       // CTAs in a cluster; parts that time is cut into
constexpr int kKeptOffsets = 1024;                                      // offsets that fit in shared memory

struct Recurrence {
    const void *x, *gate, *dy;                  // dy: backward only
    void *y, *dx, *dgate;                       // y: written forward, read backward
    int64_t ldx, ldg, ldy, lddy, lddx, lddg;
    const float *h0, *dh_last;
    float *h_last, *dh0;
    const int64_t *offsets;                     // sequences + 1 of them, or NULL: sequences of `each` tokens
    int64_t sequences;
    int T, C, each, tiles;
    int parts, part_steps;                      // time is cut into parts of so many steps, each worked on by itself
    float2 *summary;                            // [parts][C]: (P, L) of each part
};

template <typename T> __device__ __forceinline__ float fast_exp(float v) {   // two units in the last place and |v| 2^-24
    return __expf(v);
}
template <> __device__ __forceinline__ float fast_exp<float>(float v) { return expf(v); }

__device__ __forceinline__ float min_nan(float a, float b) {       // keeps a NaN
    float y;
    asm("min.NaN.f32 %0, %1, %2;" : "=f"(y) : "f"(a), "f"(b));
    return y;
}

// One lane's V consecutive elements, as they lie in memory.
template <typename T, int V> struct Few { T v[V]; };
template <typename T, int V> __device__ __forceinline__ Few<T, V> load_few(const T *p) {
    Few<T, V> f;
    if constexpr (V == 2) {
        uint32_t w;
        asm volatile("ld.global.L1::no_allocate.u32 %0, [%1];" : "=r"(w) : "l"(p));
        memcpy(&f, &w, 4);
    } else {
        f.v[0] = *p;
    }
    return f;
}
template <typename T, int V> __device__ __forceinline__ Few<T, V> no_few() {
    Few<T, V> f;
#pragma unroll
    for (int v = 0; v < V; ++v) f.v[v] = from_float<T>(0.f);
    return f;
}
template <typename T, int V> __device__ __forceinline__ void store_few(T *p, const float (&in)[V]) {
    Few<T, V> f;
#pragma unroll
    for (int v = 0; v < V; ++v) f.v[v] = from_float<T>(in[v]);
    if constexpr (V == 2) {
        uint32_t w;
        memcpy(&w, &f, 4);
        *reinterpret_cast<uint32_t *>(p) = w;
    } else {
        *p = f.v[0];
    }
}

__device__ __forceinline__ bool is_reset(float P) { return __float_as_uint(P) == 0x80000000u; }
__device__ __forceinline__ float advance(float2 m, float s) { return is_reset(m.x) ? m.y : fmaf(m.x, s, m.y); }
__device__ __forceinline__ float2 join(float2 first, float2 then) {
    return is_reset(then.x) ? then : make_float2(then.x * first.x, fmaf(then.x, first.y, then.y));
}

// Which sequence a step belongs to, and what happens there.
struct Places {
    const int64_t *offsets;
    int *kept;                                  // the offsets in shared memory, or NULL
    int sequences, each, T;
    __device__ int bound(int s) const {         // first token of sequence s (s = sequences: behind the last)
        if (kept) return kept[s];
        const int64_t o = offsets[s];
        return o < 0 ? 0 : o > T ? T : (int)o;
    }
    // The sequence of token t (or one that does not hold it, where no sequence does) and its tokens.
    __device__ int find(int t, int &first, int &behind) const {
        if (!offsets) {
            const int s = t / each;
            first = s * each;
            behind = first + each;
            return s;
        }
        int lo = 0, hi = sequences - 1;         // how many sequences end at or before t
        while (lo < hi) {
            const int mid = (lo + hi) >> 1;
            if (bound(mid + 1) <= t) lo = mid + 1;
            else hi = mid;
        }
        first = bound(lo);
        behind = bound(lo + 1);
        return lo;
    }
};

// BACK: steps count from the last token.  PART: only (P, L) of each part.
// Grid: tiles of channels x CTAs of a cluster, parts.
template <typename T, int V, bool BACK, bool PART>
__global__ void __launch_bounds__(32 * kRecWarps) recurrence_kernel(const Recurrence a, int ranks) {
    __shared__ float2 runs[2][kRecWarps][32 * V];
    __shared__ float2 blocks[2][kMostCluster][32 * V];
    __shared__ int kept[kKeptOffsets];
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = ranks > 1 ? (int)cluster_rank() : 0, tile = (int)blockIdx.x / ranks;
    const int col = tile * (32 * V) + lane * V;
    const bool mine = col < a.C;                                 // C is a multiple of V
    Places at = {a.offsets, nullptr, (int)a.sequences, a.each, a.T};
    if (a.offsets && a.sequences < kKeptOffsets) {
        for (int s = threadIdx.x; s <= at.sequences; s += blockDim.x) {
            const int64_t o = a.offsets[s];
            kept[s] = o < 0 ? 0 : o > a.T ? a.T : (int)o;
        }
        at.kept = kept;
        __syncthreads();
    }
    const float *enter_with = BACK ? a.dh_last : a.h0;
    float *leave_to = BACK ? a.dh0 : a.h_last;
    const auto entered = [&](int s, int v) { return enter_with && mine ? enter_with[(int64_t)s * a.C + col + v] : 0.f; };

    if (ranks > 1) cluster_sync();                               // all have started before one writes to another
    const int begin = (int)blockIdx.y * a.part_steps;            // of this part; parts * part_steps < 2^31
    const int end = min(a.T, begin + a.part_steps);
    float state[V], prod[V];                                     // before the block; PART: (P, L) from the part's start
#pragma unroll
    for (int v = 0; v < V; ++v) {
        state[v] = 0.f;
        prod[v] = 1.f;
    }
    if (!PART && mine) {
#pragma unroll 4
        for (int p = 0; p < (int)blockIdx.y; ++p)
#pragma unroll
            for (int v = 0; v < V; ++v) state[v] = advance(a.summary[(int64_t)p * a.C + col + v], state[v]);
    }

    const int stride = ranks * kRecSteps, rounds = (end - begin + stride - 1) / stride;
    for (int i = 0; i < rounds; ++i) {
        const int buf = i & 1, run = begin + i * stride + rank * kRecSteps + warp * kRun;
        // lanes 0 .. kRun - 1 look up the run's steps; bit j of a mask is step j
        int seq = 0;
        bool there = false, enter = false, leave = false;
        if (lane < kRun && run + lane < end) {
            const int t = BACK ? a.T - 1 - (run + lane) : run + lane;
            int first, behind;
            seq = at.find(t, first, behind);
            there = first <= t && t < behind;
            enter = there && t == (BACK ? behind - 1 : first);
            leave = there && t == (BACK ? first : behind - 1);
        }
        const uint32_t is_there = mine ? __ballot_sync(0xffffffffu, there) : (__ballot_sync(0xffffffffu, there), 0u);
        const uint32_t enters = __ballot_sync(0xffffffffu, enter), leaves = __ballot_sync(0xffffffffu, leave);

        // What comes in: forward the gate and x, backward the gate and dy (then x and the state before).
        const int64_t t0 = BACK ? a.T - 1 - run : run;
        const int dir = BACK ? -1 : 1;
        const T *pg = (const T *)a.gate + t0 * a.ldg + col, *pb = BACK ? (const T *)a.dy + t0 * a.lddy + col : (const T *)a.x + t0 * a.ldx + col;
        const int64_t sg = dir * a.ldg, sb = dir * (BACK ? a.lddy : a.ldx);
        Few<T, V> in_g[kRun], in_b[kRun];
        if (is_there == (1u << kRun) - 1u) {
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                in_g[j] = load_few<T, V>(pg + j * sg);
                in_b[j] = load_few<T, V>(pb + j * sb);
            }
        } else {
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                in_g[j] = is_there >> j & 1u ? load_few<T, V>(pg + j * sg) : no_few<T, V>();
                in_b[j] = is_there >> j & 1u ? load_few<T, V>(pb + j * sb) : no_few<T, V>();
            }
        }
        float c[kRun][V], P[V], L[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            P[v] = 1.f;
            L[v] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            if (enters >> j & 1u) {
                const int s = __shfl_sync(0xffffffffu, seq, j);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    P[v] = -0.f;
                    L[v] = entered(s, v);
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                // a step that is not there leaves the state as it is
                c[j][v] = is_there >> j & 1u ? min_nan(__fdividef(1.f, 1.f + fast_exp<T>(to_float<T>(in_g[j].v[v]))), 1.f) : 0.f;
                const float b = to_float<T>(in_b[j].v[v]), keep = 1.f - c[j][v];
                L[v] = BACK ? keep * (L[v] + b) : fmaf(keep, L[v], c[j][v] * b);
                P[v] *= keep;
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) runs[buf][warp][lane * V + v] = make_float2(P[v], L[v]);
        __syncthreads();
        if (ranks > 1) {
            if (threadIdx.x < 32 * V) {
                float2 m = runs[buf][0][threadIdx.x];
#pragma unroll
                for (int w = 1; w < kRecWarps; ++w) m = join(m, runs[buf][w][threadIdx.x]);
                const uint32_t to = smem_address(&blocks[buf][rank][threadIdx.x]);
                for (int r = 0; r < ranks; ++r) {
                    const uint32_t there_too = cluster_address(to, r);
                    asm volatile("st.shared::cluster.v2.f32 [%0], {%1, %2};" ::"r"(there_too), "f"(m.x), "f"(m.y) : "memory");
                }
            }
            cluster_sync();
        }
        float s[V];                                              // before this warp's run
        if constexpr (PART) {
#pragma unroll
            for (int w = 0; w < kRecWarps; ++w)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float2 m = join(make_float2(prod[v], state[v]), runs[buf][w][lane * V + v]);
                    prod[v] = m.x;
                    state[v] = m.y;
                }
            continue;
        }
        if (ranks > 1) {
            for (int r = 0; r < ranks; ++r) {
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (r == rank) s[v] = state[v];
                    state[v] = advance(blocks[buf][r][lane * V + v], state[v]);
                }
            }
#pragma unroll
            for (int w = 0; w < kRecWarps - 1; ++w)
                if (w < warp)
#pragma unroll
                    for (int v = 0; v < V; ++v) s[v] = advance(runs[buf][w][lane * V + v], s[v]);
        } else {
#pragma unroll
            for (int w = 0; w < kRecWarps; ++w)
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    if (w == warp) s[v] = state[v];
                    state[v] = advance(runs[buf][w][lane * V + v], state[v]);
                }
        }

        if constexpr (!BACK) {
            T *py = (T *)a.y + t0 * a.ldy + col;
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                if (enters >> j & 1u) {
                    const int q = __shfl_sync(0xffffffffu, seq, j);
#pragma unroll
                    for (int v = 0; v < V; ++v) s[v] = entered(q, v);
                }
#pragma unroll
                for (int v = 0; v < V; ++v) s[v] = fmaf(1.f - c[j][v], s[v], c[j][v] * to_float<T>(in_b[j].v[v]));
                if (is_there >> j & 1u) store_few<T, V>(py + j * a.ldy, s);
                if (leave_to && (leaves >> j & 1u)) {
                    const int q = __shfl_sync(0xffffffffu, seq, j);
                    if (mine)
#pragma unroll
                        for (int v = 0; v < V; ++v) leave_to[(int64_t)q * a.C + col + v] = s[v];
                }
            }
        } else {
            const T *px = (const T *)a.x + t0 * a.ldx + col, *py = (const T *)a.y + (t0 - 1) * a.ldy + col;
            T *pdx = (T *)a.dx + t0 * a.lddx + col, *pdg = (T *)a.dgate + t0 * a.lddg + col;
            Few<T, V> in_x[kRun], in_y[kRun];
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                in_x[j] = is_there >> j & 1u ? load_few<T, V>(px - j * a.ldx) : no_few<T, V>();
                in_y[j] = (is_there & ~leaves) >> j & 1u ? load_few<T, V>(py - j * a.ldy) : no_few<T, V>();
            }
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                if (enters >> j & 1u) {
                    const int q = __shfl_sync(0xffffffffu, seq, j);
#pragma unroll
                    for (int v = 0; v < V; ++v) s[v] = entered(q, v);
                }
                float before[V], dx[V], dg[V];
#pragma unroll
                for (int v = 0; v < V; ++v) before[v] = to_float<T>(in_y[j].v[v]);
                if (a.h0 && (leaves >> j & 1u)) {
                    const int q = __shfl_sync(0xffffffffu, seq, j);
                    if (mine)
#pragma unroll
                        for (int v = 0; v < V; ++v) before[v] = a.h0[(int64_t)q * a.C + col + v];
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float lambda = to_float<T>(in_b[j].v[v]) + s[v], keep = 1.f - c[j][v];
                    dx[v] = c[j][v] * lambda;
                    dg[v] = lambda * (before[v] - to_float<T>(in_x[j].v[v])) * (keep * c[j][v]);
                    s[v] = keep * lambda;
                }
                if (is_there >> j & 1u) {
                    store_few<T, V>(pdx - j * a.lddx, dx);
                    store_few<T, V>(pdg - j * a.lddg, dg);
                }
                if (leave_to && (leaves >> j & 1u)) {
                    const int q = __shfl_sync(0xffffffffu, seq, j);
                    if (mine)
#pragma unroll
                        for (int v = 0; v < V; ++v) leave_to[(int64_t)q * a.C + col + v] = s[v];
                }
            }
        }
    }
    if (PART) {
        if (warp == 0 && mine)
#pragma unroll
            for (int v = 0; v < V; ++v) a.summary[(int64_t)blockIdx.y * a.C + col + v] = make_float2(prod[v], state[v]);
        return;
    }
    // A sequence without tokens hands on what it was given.
    if (leave_to && blockIdx.y == 0 && rank == 0 && mine && (a.offsets || a.each == 0))
        for (int q = warp; q < at.sequences; q += kRecWarps)
            if (a.each == 0 && !a.offsets || a.offsets && at.bound(q + 1) <= at.bound(q))
#pragma unroll
                for (int v = 0; v < V; ++v) leave_to[(int64_t)q * a.C + col + v] = entered(q, v);
}

}  // namespace deft
