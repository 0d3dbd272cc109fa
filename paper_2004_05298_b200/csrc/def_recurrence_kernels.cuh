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
// It is bound by what a round of a cluster's blocks waits for, not by memory.  Measured, of the copy rate of 6562 GB/s: 16384 x 4096
// bf16 in 8 sequences forward 114 us (3.5 TB/s), backward 177 (4.5); 8192 x 4096 fp32 82 (4.9) and 166 (4.8); 16384 x 512 fp32 in
// parts 30 and 51; rows off alignment, 16384 x 4097 bf16, 234 and 436.
//
// Sequences lie one behind another; at a sequence's first step the state is replaced, P becomes -0 ("nothing from before":
// with a zero of that sign no infinity or NaN of another sequence gets in).
#pragma once

#include <cuda.h>

#include "def_sm100.cuh"
#include "def_train_common.cuh"

namespace deft {

constexpr int kRun = 8, kRecWarps = 8, kRecSteps = kRun * kRecWarps;   // steps of a warp; of a CTA's block
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
    float2 *summary;                            // (P, L) of each part and channel: [parts][C], or of pairs of channels (P, P, L, L)
};

template <bool B> struct Known { static constexpr bool value = B; };
// 1 / (1 + exp(g)) = 1 - a.
template <typename T> __device__ __forceinline__ float logistic_back(float g) { return logistic<T>(-g); }

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

// What a run keeps of the state before it: the product of its 1 - c, each of them rounded; or, where that is at least a half, 1 less
// what it lets go, Q = c + (1 - c) Q', in which nothing is lost.  Only so do memories of many tokens last as long as they should: for c =
// 2^-17 a state that is multiplied with a rounded 1 - c at every step may be off by a 256th.  (A start sets Q to 1.)  Within a run the
// rounded 1 - c serves, since what its steps are off there is not handed on; but for runs whose state leaves the call (one token of each
// sequence, say): there what the rounding takes from 1 - c (`lost`, exact) is multiplied, too.  Kernels of their own for calls that hand
// states on: 16384 x 4096 bf16 in 8 sequences 114 us forward without Q, 115 with it, 131 and 135 with states in and out; rows of even width
// off 16 bytes, 16384 x 4098 bf16, 211 and 204, 211 and 250.
__device__ __forceinline__ float kept_by(float P, float Q) { return Q < 0.5f ? 1.f - Q : P; }
__device__ __forceinline__ float lost(float keep, float c) { return (1.f - keep) - c; }
__device__ __forceinline__ float finite(float s) { return fminf(fmaxf(s, -3.402823466e38f), 3.402823466e38f); }   // 0 times infinity is no number
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

// BACK: steps count from the last token.  PART: only (P, L) of each part.  HANDED: the states behind the sequences (dh0) are wanted, which
// are then found more carefully.  Grid: tiles of channels x CTAs of a cluster, parts.
template <typename T, int V, bool BACK, bool PART, bool HANDED>
__global__ void __launch_bounds__(32 * kRecWarps, 4) recurrence_kernel(const Recurrence a, int ranks) {
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
    float *leave_to = BACK ? a.dh0 : a.h_last;                   // HANDED
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
        float c[kRun][V], P[V], Q[V], L[V];
#pragma unroll
        for (int v = 0; v < V; ++v) {
            P[v] = 1.f;
            Q[v] = L[v] = 0.f;
        }
#pragma unroll
        for (int j = 0; j < kRun; ++j) {
            if (enters >> j & 1u) {
                const int s = __shfl_sync(0xffffffffu, seq, j);
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    P[v] = -0.f;
                    Q[v] = 1.f;
                    L[v] = entered(s, v);
                }
            }
#pragma unroll
            for (int v = 0; v < V; ++v) {
                // a step that is not there leaves the state as it is
                c[j][v] = is_there >> j & 1u ? logistic_back<T>(to_float<T>(in_g[j].v[v])) : 0.f;
                const float b = to_float<T>(in_b[j].v[v]), keep = 1.f - c[j][v];
                L[v] = BACK ? keep * (L[v] + b) : fmaf(keep, L[v], c[j][v] * b);
                P[v] *= keep;
                Q[v] = fmaf(keep, Q[v], c[j][v]);
            }
        }
#pragma unroll
        for (int v = 0; v < V; ++v) runs[buf][warp][lane * V + v] = make_float2(kept_by(P[v], Q[v]), L[v]);
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

        // is_handed: the state leaves from one of these steps
        const auto in_turn = [&](const auto &step) {
            if (HANDED && leaves) {
#pragma unroll
                for (int j = 0; j < kRun; ++j) step(j, Known<true>());
            } else {
#pragma unroll
                for (int j = 0; j < kRun; ++j) step(j, Known<false>());
            }
        };
        if constexpr (!BACK) {
            T *py = (T *)a.y + t0 * a.ldy + col;
            in_turn([&](int j, auto is_handed) {
                constexpr bool kHanded = decltype(is_handed)::value;
                if (enters >> j & 1u) {
                    const int q = __shfl_sync(0xffffffffu, seq, j);
#pragma unroll
                    for (int v = 0; v < V; ++v) s[v] = entered(q, v);
                }
#pragma unroll
                for (int v = 0; v < V; ++v) {
                    const float keep = 1.f - c[j][v];
                    float in = c[j][v] * to_float<T>(in_b[j].v[v]);
                    if (kHanded) in = fmaf(lost(keep, c[j][v]), finite(s[v]), in);
                    s[v] = fmaf(keep, s[v], in);
                }
                if (is_there >> j & 1u) store_few<T, V>(py + j * a.ldy, s);
                if (kHanded && (leaves >> j & 1u)) {
                    const int q = __shfl_sync(0xffffffffu, seq, j);
                    if (mine)
#pragma unroll
                        for (int v = 0; v < V; ++v) leave_to[(int64_t)q * a.C + col + v] = s[v];
                }
            });
        } else {
            const T *px = (const T *)a.x + t0 * a.ldx + col, *py = (const T *)a.y + (t0 - 1) * a.ldy + col;
            T *pdx = (T *)a.dx + t0 * a.lddx + col, *pdg = (T *)a.dgate + t0 * a.lddg + col;
            Few<T, V> in_x[kRun], in_y[kRun];
#pragma unroll
            for (int j = 0; j < kRun; ++j) {
                in_x[j] = is_there >> j & 1u ? load_few<T, V>(px - j * a.ldx) : no_few<T, V>();
                in_y[j] = (is_there & ~leaves) >> j & 1u ? load_few<T, V>(py - j * a.ldy) : no_few<T, V>();
            }
            in_turn([&](int j, auto is_handed) {
                constexpr bool kHanded = decltype(is_handed)::value;
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
                    s[v] = kHanded ? fmaf(keep, lambda, lost(keep, c[j][v]) * finite(lambda)) : keep * lambda;
                }
                if (is_there >> j & 1u) {
                    store_few<T, V>(pdx - j * a.lddx, dx);
                    store_few<T, V>(pdg - j * a.lddg, dg);
                }
                if (kHanded && (leaves >> j & 1u)) {
                    const int q = __shfl_sync(0xffffffffu, seq, j);
                    if (mine)
#pragma unroll
                        for (int v = 0; v < V; ++v) leave_to[(int64_t)q * a.C + col + v] = s[v];
                }
            });
        }
    }
    if (PART) {
        if (warp == 0 && mine)
#pragma unroll
            for (int v = 0; v < V; ++v) a.summary[(int64_t)blockIdx.y * a.C + col + v] = make_float2(prod[v], state[v]);
        return;
    }
    // A sequence without tokens hands on what it was given.
    if (HANDED && blockIdx.y == 0 && rank == 0 && mine && (a.offsets || a.each == 0))
        for (int q = warp; q < at.sequences; q += kRecWarps)
            if (a.each == 0 && !a.offsets || a.offsets && at.bound(q + 1) <= at.bound(q))
#pragma unroll
                for (int v = 0; v < V; ++v) leave_to[(int64_t)q * a.C + col + v] = entered(q, v);
}

// ---------------------------------------------------------------------------
// The same for rows on 16-byte boundaries: blocks of steps by 64 channels come by tensor copies into a ring, so that loads run
// on under the two passes over a block and registers hold little.  Small blocks, so that two CTAs share an SM (fp32 backward:
// one): one computes while the other waits for a barrier.  Pass one leaves 1 - c and c x of a step in registers (backward: c; what else
// pass two needs it reads from the ring again).  A thread has two channels and works on both in one instruction.
// ---------------------------------------------------------------------------
constexpr int kStreamOffsets = 128;             // offsets that are kept in shared memory
template <typename T, bool BACK> struct StreamBlock {
    static constexpr int run = sizeof(T) == 2 && !BACK ? 16 : 8, steps = run * kRecWarps;
    static constexpr int tensors = BACK ? 4 : 2, row = 64 * (int)sizeof(T), bytes = steps * row;
    static constexpr int stages = 3, smem = stages * tensors * bytes + 128, part_smem = stages * 2 * bytes + 128;   // part: gate and x (dy)
    // CTAs per SM that a call is cut for, and that have room beside each other, but for fp32 backward, whose ring leaves room for one: there a
    // call runs in two waves.  Cut for one CTA (and parts rounded down), us: 16384 x 256 30 against 37, 16384 x 2048 179 against 217;
    // but 8192 x 4096 177 against 143, 16384 x 4096 359 against 297.
    static constexpr int ctas = 2;
};
struct RecurrenceMaps {
    CUtensorMap gate, first, x, y;              // first: x forward, dy backward; x and y: backward only
};

template <typename T> __device__ __forceinline__ Pair two_channels(const uint8_t *p) {
    if constexpr (sizeof(T) == 4) {
        const float2 v = *reinterpret_cast<const float2 *>(p);
        return make_pair(v.x, v.y);
    } else {
        const uint32_t w = *reinterpret_cast<const uint32_t *>(p);
        Few<T, 2> f;
        memcpy(&f, &w, 4);
        return make_pair(to_float<T>(f.v[0]), to_float<T>(f.v[1]));
    }
}
template <typename T> __device__ __forceinline__ void store_channels(T *p, Pair v) {
    float a, b;
    split_pair(v, a, b);
    if constexpr (sizeof(T) == 4) {
        *reinterpret_cast<float2 *>(p) = make_float2(a, b);
    } else {
        Few<T, 2> f;
        f.v[0] = from_float<T>(a);
        f.v[1] = from_float<T>(b);
        uint32_t w;
        memcpy(&w, &f, 4);
        *reinterpret_cast<uint32_t *>(p) = w;
    }
}
__device__ __forceinline__ Pair pair_mul(Pair a, Pair b) {
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d.bits) : "l"(a.bits), "l"(b.bits));
    return d;
}
__device__ __forceinline__ bool is_nan(Pair p) {
    float a, b;
    split_pair(p, a, b);
    return isnan(a) || isnan(b);
}
template <typename T> __device__ __forceinline__ Pair logistic_back(Pair g) {
    float a, b;
    if constexpr (sizeof(T) == 4) {
        split_pair(g, a, b);
        return make_pair(logistic_back<T>(a), logistic_back<T>(b));
    } else {
        split_pair(pair_mul(g, make_pair(1.44269504f, 1.44269504f)), a, b);
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(a));
        asm("ex2.approx.ftz.f32 %0, %0;" : "+f"(b));
        split_pair(pair_add(make_pair(a, b), make_pair(1.f, 1.f)), a, b);
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(a));
        asm("rcp.approx.ftz.f32 %0, %0;" : "+f"(b));
        return make_pair(a, b);
    }
}
__device__ __forceinline__ Pair kept_by(Pair P, Pair Q) {
    float p0, p1, q0, q1;
    split_pair(P, p0, p1);
    split_pair(Q, q0, q1);
    return make_pair(kept_by(p0, q0), kept_by(p1, q1));
}
__device__ __forceinline__ Pair lost(Pair keep, Pair c) {
    const Pair one = make_pair(1.f, 1.f), minus = make_pair(-1.f, -1.f);
    return pair_fma(c, minus, pair_fma(keep, minus, one));
}
__device__ __forceinline__ Pair finite(Pair s) {
    float a, b;
    split_pair(s, a, b);
    return make_pair(finite(a), finite(b));
}
struct alignas(16) Map2 { Pair P, L; };          // (P, L) of two channels
// `calm`: no sequence starts there.
template <bool CALM> __device__ __forceinline__ Pair advance2(const Map2 &m, Pair s) {
    if constexpr (CALM) {
        return pair_fma(m.P, s, m.L);
    } else {
        float p0, p1, l0, l1, s0, s1;
        split_pair(m.P, p0, p1);
        split_pair(m.L, l0, l1);
        split_pair(s, s0, s1);
        return make_pair(advance(make_float2(p0, l0), s0), advance(make_float2(p1, l1), s1));
    }
}
template <bool CALM> __device__ __forceinline__ Map2 join2(const Map2 &first, const Map2 &then) {
    if constexpr (CALM) {
        return {pair_mul(then.P, first.P), pair_fma(then.P, first.L, then.L)};
    } else {
        float a0, a1, b0, b1, c0, c1, d0, d1;
        split_pair(first.P, a0, a1);
        split_pair(first.L, b0, b1);
        split_pair(then.P, c0, c1);
        split_pair(then.L, d0, d1);
        const float2 x = join(make_float2(a0, b0), make_float2(c0, d0)), y = join(make_float2(a1, b1), make_float2(c1, d1));
        return {make_pair(x.x, y.x), make_pair(x.y, y.y)};
    }
}
// A CTA's block as one, from its warps' runs; the state before a warp's run and behind the cluster's blocks.
using Runs = const Map2 (&)[kRecWarps][32];
using Blocks = const Map2 (&)[kMostCluster][32];
template <bool CALM> __device__ __forceinline__ Map2 join_runs(Runs runs, int lane) {
    Map2 all = runs[0][lane];
#pragma unroll
    for (int w = 1; w < kRecWarps; ++w) all = join2<CALM>(all, runs[w][lane]);
    return all;
}
template <bool CALM> __device__ __forceinline__ Pair advance_all(Runs runs, Blocks blocks, int ranks, int rank, int warp, int lane, Pair &behind) {
    Pair s = behind;
    if (ranks > 1) {
        for (int r = 0; r < ranks; ++r) {
            if (r == rank) s = behind;
            behind = advance2<CALM>(blocks[r][lane], behind);
        }
        for (int w = 0; w < warp; ++w) s = advance2<CALM>(runs[w][lane], s);
    } else {
#pragma unroll
        for (int w = 0; w < kRecWarps; ++w) {
            if (w == warp) s = behind;
            behind = advance2<CALM>(runs[w][lane], behind);
        }
    }
    return s;
}
// 16 bytes to another CTA's shared memory, counted there on `bar`.
__device__ __forceinline__ void send(uint32_t to, uint32_t bar, const Map2 &m) {
    asm volatile("st.async.shared::cluster.mbarrier::complete_tx::bytes.v2.b64 [%0], {%1, %2}, [%3];" ::"r"(to), "l"(m.P.bits), "l"(m.L.bits), "r"(bar) : "memory");
}

template <typename T, bool BACK, bool PART, bool HANDED>
__global__ void __launch_bounds__(32 * kRecWarps, StreamBlock<T, BACK>::ctas)
    recurrence_stream_kernel(const Recurrence a, int ranks, const __grid_constant__ RecurrenceMaps maps) {
    using B = StreamBlock<T, BACK>;
    constexpr int R = B::run, kSteps = B::steps, kUsed = PART ? 2 : B::tensors;
    extern __shared__ __align__(128) uint8_t ring[];
    __shared__ Map2 runs[2][kRecWarps][32];
    __shared__ Map2 blocks[2][kMostCluster][32];
    __shared__ int kept[kStreamOffsets];
    __shared__ uint64_t bars[B::stages + 2];
    __shared__ volatile int failed;
    uint8_t *stages = (uint8_t *)(((uintptr_t)ring + 127) & ~(uintptr_t)127);
    const uint32_t full = smem_address(bars), got = full + 8 * B::stages;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int rank = ranks > 1 ? (int)cluster_rank() : 0, tile = (int)blockIdx.x / ranks;
    const int col = tile * 64 + lane * 2;
    const bool mine = col < a.C;                                 // C is even
    Places at = {a.offsets, nullptr, (int)a.sequences, a.each, a.T};
    if (a.offsets && a.sequences < kStreamOffsets) {
        for (int s = threadIdx.x; s <= at.sequences; s += blockDim.x) {
            const int64_t o = a.offsets[s];
            kept[s] = o < 0 ? 0 : o > a.T ? a.T : (int)o;
        }
        at.kept = kept;
    }
    if (threadIdx.x == 0) {
        for (int s = 0; s < B::stages + 2; ++s) barrier_init(full + 8 * s, 1);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    __syncthreads();
    if (ranks > 1) cluster_sync();                               // all have started before one writes to another
    const int begin = (int)blockIdx.y * a.part_steps;            // of this part
    const int end = min(a.T, begin + a.part_steps);
    const int stride = ranks * kSteps, rounds = (end - begin + stride - 1) / stride;
    constexpr int kStage = kUsed * B::bytes;
    const auto load = [&](int i) {                               // one thread: the block of round i
        const int s = i % B::stages, run = begin + i * stride + rank * kSteps;
        const int t0 = BACK ? a.T - run - kSteps : run;          // may lie before the first or behind the last row: zeros there
        const uint32_t bar = full + 8 * s, to = smem_address(stages + s * kStage);
        barrier_expect(bar, kStage);
        tensor_load_2d(to, &maps.gate, tile * 64, t0, bar);
        tensor_load_2d(to + B::bytes, &maps.first, tile * 64, t0, bar);
        if constexpr (BACK && !PART) {
            tensor_load_2d(to + 2 * B::bytes, &maps.x, tile * 64, t0, bar);
            tensor_load_2d(to + 3 * B::bytes, &maps.y, tile * 64, t0 - 1, bar);
        }
    };
    if (threadIdx.x == 0)
        for (int i = 0; i < B::stages && i < rounds; ++i) load(i);
    if (PART) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    else asm volatile("griddepcontrol.wait;" ::: "memory");      // the parts' maps are the kernel before's; the copies above are not

    const float *enter_with = BACK ? a.dh_last : a.h0;
    float *leave_to = BACK ? a.dh0 : a.h_last;
    const auto entered = [&](int s) {
        const float *p = enter_with + (int64_t)s * a.C + col;
        return enter_with && mine ? make_pair(p[0], p[1]) : make_pair(0.f, 0.f);
    };
    const auto left = [&](int s, Pair v) {
        if (!mine) return;
        float *p = leave_to + (int64_t)s * a.C + col;
        split_pair(v, p[0], p[1]);
    };
    const Pair zero = make_pair(0.f, 0.f), one = make_pair(1.f, 1.f), minus = make_pair(-1.f, -1.f);
    Map2 whole = {one, zero};                                    // PART: of the part so far; else L is the state before the block
    if (!PART && mine) {
#pragma unroll 4
        for (int p = 0; p < (int)blockIdx.y; ++p)
            whole.L = advance2<false>(*reinterpret_cast<const Map2 *>(a.summary + ((int64_t)p * a.tiles * 64 + col)), whole.L);
    }
    int first = 0, behind = 0;                                   // tokens of a sequence this CTA has come to
    bool ok = true;
    int stage = 0, turn = 0;                                     // of the ring: round i is stage i mod stages, in its turn-th use
    for (int i = 0; i < rounds; ++i, turn ^= stage == B::stages - 1, stage = stage == B::stages - 1 ? 0 : stage + 1) {
        const int buf = i & 1, base = begin + i * stride, run = base + rank * kSteps + warp * R;
        // Calm: all of the cluster's blocks of this round lie inside one sequence, its first and (where that matters) last token
        // elsewhere.
        const int t_lo = BACK ? a.T - base - stride : base, t_hi = t_lo + stride - 1;
        const bool calm = t_lo > first && t_hi < behind - (BACK || HANDED ? 1 : 0) && base + stride <= end;
        uint32_t is_there = (1u << R) - 1u, enters = 0, leaves = 0;
        int seq = 0;
        if (!calm) {
            bool there = false, enter = false, leave = false;
            if (base < end) at.find(BACK ? a.T - 1 - min(base + stride, end) + 1 : min(base + stride, end) - 1, first, behind);     // where the round ends
            if (lane < R && run + lane < end) {
                const int t = BACK ? a.T - 1 - (run + lane) : run + lane;
                int lo, hi;
                seq = at.find(t, lo, hi);
                there = lo <= t && t < hi;
                enter = there && t == (BACK ? hi - 1 : lo);
                leave = there && t == (BACK ? lo : hi - 1);
            }
            is_there = __ballot_sync(0xffffffffu, there);
            enters = __ballot_sync(0xffffffffu, enter);
            leaves = __ballot_sync(0xffffffffu, leave);
        }
        if (!BACK && !HANDED) leaves = 0;                      // nothing happens there
        const bool plain = is_there == (1u << R) - 1u && (enters | leaves) == 0;
        ok = ok && barrier_wait(full + 8 * stage, turn, &failed);
        // row j of the run; backward a block's rows lie in the order of time
        const uint8_t *rows = stages + stage * kStage + (BACK ? kSteps - 1 - warp * R : warp * R) * B::row + lane * (B::row / 32);
        constexpr int kStep = BACK ? -B::row : B::row;
        Pair keep[R], in[R];                                     // 1 - c (or c, see pass_one), c x (backward: c)
        Map2 m = {one, zero};
        Pair let = zero;                                         // Q
        // first_j: 1 - c; c where the state behind a run that is not plain may be handed on
        const auto pass_one = [&](int j, Pair &first_j, Pair &in_j, auto is_plain) {
            const Pair c = logistic_back<T>(two_channels<T>(rows + j * kStep)), b = two_channels<T>(rows + j * kStep + B::bytes);
            const Pair keep_j = pair_fma(c, minus, one);
            first_j = decltype(is_plain)::value || !HANDED ? keep_j : c;
            if constexpr (BACK) {
                in_j = c;
                m.L = pair_mul(keep_j, pair_add(m.L, b));
            } else {
                in_j = pair_mul(c, b);
                m.L = pair_fma(keep_j, m.L, in_j);
            }
            m.P = pair_mul(m.P, keep_j);
            let = pair_fma(keep_j, let, c);
        };
        if (plain) {
#pragma unroll
            for (int j = 0; j < R; ++j) pass_one(j, keep[j], in[j], Known<true>());
        } else {
#pragma unroll
            for (int j = 0; j < R; ++j) {
                if (enters >> j & 1u) {
                    m = {make_pair(-0.f, -0.f), entered(__shfl_sync(0xffffffffu, seq, j))};
                    let = one;
                }
                if (is_there >> j & 1u) pass_one(j, keep[j], in[j], Known<false>());
            }
        }
        m.P = kept_by(m.P, let);
        runs[buf][warp][lane] = m;
        __syncthreads();
        if (threadIdx.x == 0 && ok) {
            // forward all are done with this block, backward with the one before
            if (!BACK || PART) {
                if (i + B::stages < rounds) load(i + B::stages);
            } else if (i > 0 && i - 1 + B::stages < rounds) {
                load(i - 1 + B::stages);
            }
        }
        if (ranks > 1) {
            if (warp == 0) {
                const Map2 all = calm ? join_runs<true>(runs[buf], lane) : join_runs<false>(runs[buf], lane);
                if (lane == 0) barrier_expect(got + 8 * buf, (uint32_t)ranks * sizeof(blocks[0][0]));
                const uint32_t to = smem_address(&blocks[buf][rank][lane]);
                for (int r = 0; r < ranks; ++r) send(cluster_address(to, r), cluster_address(got + 8 * buf, r), all);
            }
            ok = ok && barrier_wait(got + 8 * buf, i >> 1 & 1, &failed);
        }
        if constexpr (PART) {
            whole = calm ? join2<true>(whole, join_runs<true>(runs[buf], lane)) : join2<false>(whole, join_runs<false>(runs[buf], lane));
            continue;
        }
        // Before this warp's run.  A start's -0 takes a finite state away in the plain product as well; others need the look.
        Pair next = whole.L, s = advance_all<true>(runs[buf], blocks[buf], ranks, rank, warp, lane, next);
        if (!calm && __any_sync(0xffffffffu, is_nan(s) || is_nan(next))) {
            next = whole.L;
            s = advance_all<false>(runs[buf], blocks[buf], ranks, rank, warp, lane, next);
        }
        whole.L = next;
        if (__any_sync(0xffffffffu, !ok || failed)) {            // a wait ran out: no numbers rather than wrong ones
            ok = false;
            s = whole.L = make_pair(NAN, NAN);
            // The others may still be sending: this CTA stays until they have given up, too.  (A barrier of the cluster at the end, or this
            // there, costs 6 us of 114.)
            if (ranks > 1 && i + 1 == rounds)
                for (const uint64_t start = nanoseconds(); nanoseconds() - start < 3 * kWaitLimit;) __nanosleep(1000);
        }
        const int64_t t0 = BACK ? a.T - 1 - run : run;
        T *out = BACK ? (T *)a.dx + t0 * a.lddx + col : (T *)a.y + t0 * a.ldy + col, *out_g = (T *)a.dgate + t0 * a.lddg + col;
        const bool handed = HANDED && leaves;
        const auto pass_two = [&](int j, Pair first_j, Pair in_j, Pair before, auto is_plain) {
            constexpr bool kPlain = decltype(is_plain)::value || !HANDED;
            const Pair keep_j = kPlain ? first_j : pair_fma(first_j, minus, one);
            const auto rest = [&](Pair v) { return pair_mul(lost(keep_j, first_j), finite(v)); };
            if constexpr (!BACK) {
                s = pair_fma(keep_j, s, !kPlain && handed ? pair_add(rest(s), in_j) : in_j);
                if (mine) store_channels<T>(out, s);
                out += a.ldy;
            } else {
                const Pair b = two_channels<T>(rows + j * kStep + B::bytes), x = two_channels<T>(rows + j * kStep + 2 * B::bytes);
                const Pair lambda = pair_add(b, s), dx = pair_mul(in_j, lambda);
                s = !kPlain && handed ? pair_fma(keep_j, lambda, rest(lambda)) : pair_mul(keep_j, lambda);
                const Pair dg = pair_mul(pair_mul(dx, keep_j), pair_fma(x, minus, before));
                if (mine) {
                    store_channels<T>(out, dx);
                    store_channels<T>(out_g, dg);
                }
                out -= a.lddx;
                out_g -= a.lddg;
            }
        };
        const auto earlier = [&](int j) { return BACK ? two_channels<T>(rows + j * kStep + 3 * B::bytes) : zero; };
        if (plain) {
#pragma unroll
            for (int j = 0; j < R; ++j) pass_two(j, keep[j], in[j], earlier(j), Known<true>());
        } else {
#pragma unroll
            for (int j = 0; j < R; ++j) {
                const int q = __shfl_sync(0xffffffffu, seq, j);
                if (enters >> j & 1u) s = ok ? entered(q) : make_pair(NAN, NAN);
                if (is_there >> j & 1u) {
                    Pair before = earlier(j);
                    if (BACK && (leaves >> j & 1u)) {
                        const float *p = a.h0 + (int64_t)q * a.C + col;
                        before = a.h0 && mine ? make_pair(p[0], p[1]) : zero;
                    }
                    pass_two(j, keep[j], in[j], before, Known<false>());
                } else {
                    out += BACK ? -a.lddx : a.ldy;
                    out_g -= a.lddg;
                }
                if (HANDED && (leaves >> j & 1u)) left(q, s);
            }
        }
    }
    if (PART) {
        if (warp == 0) *reinterpret_cast<Map2 *>(a.summary + ((int64_t)blockIdx.y * a.tiles * 64 + col)) = whole;
        return;
    }
    // A sequence without tokens hands on what it was given.
    if (HANDED && blockIdx.y == 0 && rank == 0 && mine && a.offsets)
        for (int q = warp; q < at.sequences; q += kRecWarps)
            if (at.bound(q + 1) <= at.bound(q)) left(q, entered(q));
}

}  // namespace deft
