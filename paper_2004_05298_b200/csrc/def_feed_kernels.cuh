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

// 32 values of a row rounded to T, two of 16 bits in a register.
template <typename T> struct Rounded32 {
    uint32_t w[8 * sizeof(T)];
    __device__ __forceinline__ void set(int i, float even, float odd) {       // i: even
        if constexpr (sizeof(T) == 4) {
            w[i] = __float_as_uint(even);
            w[i + 1] = __float_as_uint(odd);
        } else if constexpr (__is_same(T, __half)) {
            const __half2 two = __floats2half2_rn(even, odd);
            memcpy(&w[i / 2], &two, 4);
        } else {
            const __nv_bfloat162 two = __floats2bfloat162_rn(even, odd);
            memcpy(&w[i / 2], &two, 4);
        }
    }
    __device__ __forceinline__ float operator[](int i) const {
        if constexpr (sizeof(T) == 4) {
            return __uint_as_float(w[i]);
        } else if constexpr (!__is_same(T, __half)) {
            return __uint_as_float(i % 2 ? w[i / 2] & 0xffff0000u : w[i / 2] << 16);
        } else {
            const uint16_t bits = (uint16_t)(w[i / 2] >> i % 2 * 16);
            T v;
            memcpy(&v, &bits, 2);
            return to_float<T>(v);
        }
    }
};
// Checkpoint of a group of 32 columns that one thread holds, the first n of which exist; whole groups are turned (32 bytes a
// row).  Whole warps call it.
template <typename V>
__device__ __forceinline__ void store_group(int8_t *q, int64_t ldq, uint8_t *e, const V &x, int n, bool there, uint8_t *turn) {
    float most = 0.f;
#pragma unroll
    for (int i = 0; i < 32; ++i)
        if (i < n) most = max_nan(most, fabsf(x[i]));
    const uint32_t top = __float_as_uint(most), ex = group_exponent(top);
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
                    if (8 * (p + r) + i < n && there) q[8 * (p + r) + i] = (int8_t)v[i];
            }
        }
        if (n >= 32) turn_put_word<32>(turn, p / 2, make_uint4(w[0], w[1], w[2], w[3]));
    }
    if (n >= 32) turn_store_words<32>(turn, q, ldq, there);
    if (there) *e = (uint8_t)ex;
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
        Rounded32<T> hv;
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
                const float h_back = gs * u[i];
                d[i] = x * u[i] * (s * fmaf(g[i], 1.f - s, 1.f));
                u[i] = x * gs;
                g[i] = h_back;
            }
#pragma unroll
            for (int i = 0; i < 8; i += 2) hv.set(8 * p + i, g[i], g[i + 1]);
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

// ---------------------------------------------------------------------------
// Few tokens: every weight is read once and there is little else to do, so a warp takes one row of w_in's gate and the same of
// its other half (or one row of w_down), in runs of 8 elements per lane, several of them ahead, and multiplies them by all tokens'
// elements in fp32.  The weights of the second product are on their way before the first one is done.  2048 x 5632 fp32, 138 MB of
// weights: 1 token 33 us (4.2 TB/s), 4 tokens 53, 8 tokens 91 (fp32 multiplications).
// ---------------------------------------------------------------------------
constexpr int kFewTokens = 8, kFewWarps = 8;

template <typename T> struct FewTokens {
    const T *x, *w;
    T *out;
    int64_t ldx, ldo, rows, cols;             // of w (gated: of either half)
    int tokens;
};

template <typename T, int TOKENS, bool GATED, bool ALIGNED>
__global__ void __launch_bounds__(32 * kFewWarps) few_tokens_kernel(const FewTokens<T> a) {
    constexpr int kRows = GATED ? 2 : 1, kAhead = (sizeof(T) == 2 ? 8 : 4) / kRows;
    const int lane = threadIdx.x & 31, C = (int)a.cols;
    const int64_t row = (int64_t)blockIdx.x * kFewWarps + threadIdx.x / 32;
    const bool there = row < a.rows;
    const T *w[kRows];
#pragma unroll
    for (int r = 0; r < kRows; ++r) w[r] = a.w + ((there ? row : 0) + r * a.rows) * a.cols;
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    Frag<T, 8> f[kAhead][kRows];
    const auto fetch = [&](int c0) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int r = 0; r < kRows; ++r) {
                const int c = c0 + (i * 32 + lane) * 8;
                f[i][r] = there && c < C ? load_cols<T, ALIGNED>(w[r], c, C) : zeros<T, 8>();
            }
    };
    fetch(0);
    asm volatile("griddepcontrol.wait;" ::: "memory");             // x may come from the kernel before
    float sum[kRows][TOKENS];
#pragma unroll
    for (int r = 0; r < kRows; ++r)
#pragma unroll
        for (int t = 0; t < TOKENS; ++t) sum[r][t] = 0.f;
    for (int c0 = 0; c0 < C; c0 += kAhead * 256) {
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
            const int c = c0 + (i * 32 + lane) * 8;
            float v[kRows][8];
#pragma unroll
            for (int r = 0; r < kRows; ++r) to_floats<T, 8>(f[i][r], v[r]);
            if (c < C) {
#pragma unroll
                for (int t = 0; t < TOKENS; ++t) {
                    const T *x = a.x + (t < a.tokens ? t : a.tokens - 1) * a.ldx;
                    Frag<T, 8> g;
                    if constexpr (ALIGNED) g = *reinterpret_cast<const Frag<T, 8> *>(x + c);
                    else g = load_run<T>(x, c, C);
                    float u[8];
                    to_floats<T, 8>(g, u);
#pragma unroll
                    for (int r = 0; r < kRows; ++r)
#pragma unroll
                        for (int j = 0; j < 8; ++j) sum[r][t] = fmaf(v[r][j], u[j], sum[r][t]);
                }
            }
        }
        if (c0 + kAhead * 256 < C) fetch(c0 + kAhead * 256);
    }
#pragma unroll
    for (int t = 0; t < TOKENS; ++t) {
        float y = warp_sum(sum[0][t]);
        if constexpr (GATED) y = y * logistic<T>(y) * warp_sum(sum[1][t]);
        if (lane == 0 && there && t < a.tokens) a.out[t * a.ldo + row] = from_float<T>(y);
    }
}

// ---------------------------------------------------------------------------
// Up to 32 tokens in 16 bits on tensor cores: 128 rows of the weights (gated: of either half) are M, the tokens N, so that the
// weights stream through two rings per SM and nothing else is moved.  k is cut over the CTAs of a cluster, which leave their sums in
// shared memory and add a share of them each, in the order of k.  1 token, 2048 x 5632 bf16, 69 MB of weights: both products 20.7 us
// (3.3 TB/s; two launches), 4096 x 10240, 252 MB: 48 us (5.2 TB/s).
//
// Warps: 0 copies (one thread), 1 issues the matrix instructions (one thread), the last 4 take the sums.
// ---------------------------------------------------------------------------
constexpr int kMostTokens = 32, kMostSplit = 8;
template <bool GATED, int N> struct TokenShape {
    static constexpr int tiles = GATED ? 2 : 1, stages = GATED ? 3 : 5;
    static constexpr int bytes_w = kTileRows * kTileK * 2, bytes_x = N * kTileK * 2, bytes = tiles * bytes_w + bytes_x;
    static constexpr int columns = tiles * N < 32 ? 32 : tiles * N;                          // of tensor memory
    static constexpr int smem = 1024 + stages * bytes + 128;
    static_assert(tiles * N * kTileRows * 4 <= stages * bytes);                              // the sums take the ring's place
};
struct TokenProduct {
    int tokens, blocks, bf16;             // blocks: of k
    int chain;                            // stages after which the sums move to registers: the matrix unit's truncate
    int64_t rows, ldo;                    // rows of the weights (gated: of either half)
};

__device__ __forceinline__ void mma_single(uint32_t d, uint64_t a, uint64_t b, uint32_t idesc, bool add) {
    asm volatile(
        "{\n.reg .pred p;\n"
        "setp.ne.b32 p, %4, 0;\n"
        "tcgen05.mma.cta_group::1.kind::f16 [%0], %1, %2, %3, p;\n}" ::"r"(d),
        "l"(a), "l"(b), "r"(idesc), "r"((uint32_t)add)
        : "memory");
}
__device__ __forceinline__ void mma_commit_single(uint32_t bar) {
    asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];" ::"r"(bar) : "memory");
}

template <typename T, bool GATED, int N>
__global__ void __launch_bounds__(192, 2) token_product_kernel(const TokenProduct p, T *__restrict__ out, const __grid_constant__ CUtensorMap map_w,
                                                               const __grid_constant__ CUtensorMap map_x) {
    using S = TokenShape<GATED, N>;
    extern __shared__ uint8_t raw[];
    __shared__ uint64_t bars[2 * S::stages + 2];
    __shared__ uint32_t tmem_slot;
    __shared__ volatile int failed;
    uint8_t *base = (uint8_t *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    const uint32_t full = smem_address(bars), empty = full + 8 * S::stages, done = empty + 8 * S::stages, taken = done + 8;
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31, splits = (int)gridDim.y, rank = (int)blockIdx.y;      // a cluster lies along y
    asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    if (threadIdx.x == 0) {
        for (int s = 0; s < 2 * S::stages + 1; ++s) barrier_init(full + 8 * s, 1);
        barrier_init(taken, 4);
        failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" ::"r"(smem_address(&tmem_slot)), "n"(S::columns) : "memory");
        asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
    }
    tmem_fence_before();
    __syncthreads();
    tmem_fence_after();
    const uint32_t tmem = tmem_slot;
    const int k0 = (int)((int64_t)p.blocks * rank / splits), k1 = (int)((int64_t)p.blocks * (rank + 1) / splits);
    const int row0 = (int)blockIdx.x * kTileRows;

    if (warp == 0 && lane == 0) {
        const auto weights = [&](int i) {
            const uint32_t s = i % S::stages, bar = full + 8 * s;
            barrier_expect(bar, S::bytes);
            tensor_load_3d(smem_address(base + s * S::bytes), &map_w, (k0 + i) * kTileK, row0, 0, bar);
            if (GATED) tensor_load_3d(smem_address(base + s * S::bytes + S::bytes_w), &map_w, (k0 + i) * kTileK, (int)p.rows + row0, 0, bar);
        };
        const auto tokens = [&](int i) {
            const uint32_t s = i % S::stages;
            tensor_load_3d(smem_address(base + s * S::bytes + S::tiles * S::bytes_w), &map_x, (k0 + i) * kTileK, 0, 0, full + 8 * s);
        };
        const int n = k1 - k0, first = n < S::stages ? n : S::stages;
        for (int i = 0; i < first; ++i) weights(i);
        asm volatile("griddepcontrol.wait;" ::: "memory");         // the tokens may come from the kernel before, the weights do not
        for (int i = 0; i < first; ++i) tokens(i);
        bool ok = true;
        int loaded = first;
        for (; loaded < n; ++loaded) {
            if (!(ok = barrier_wait(empty + 8 * (loaded % S::stages), (loaded / S::stages & 1) ^ 1, &failed))) break;
            weights(loaded);
            tokens(loaded);
        }
        // the copies in flight end before the CTA does
        const uint64_t start = nanoseconds();
        for (int m = loaded > S::stages ? loaded - S::stages : 0; m < loaded; ++m)
            while (!barrier_try(full + 8 * (m % S::stages), m / S::stages & 1) && nanoseconds() - start < kWaitLimit) {}
    } else if (warp == 1 && lane == 0) {
        const uint32_t idesc = 1u << 4 | (p.bf16 ? 1u : 0u) << 7 | (p.bf16 ? 1u : 0u) << 10 | (uint32_t)(N >> 3) << 17 | (uint32_t)(kTileRows >> 4) << 24;
        uint32_t chunk = 0;
        for (int i = 0, left = p.chain; i < k1 - k0; ++i, --left) {
            if (left == 0) {
                mma_commit_single(done);
                if (!barrier_wait(taken, chunk++ & 1, &failed)) break;
                tmem_fence_after();
                left = p.chain;
            }
            const uint32_t s = i % S::stages;
            if (!barrier_wait(full + 8 * s, i / S::stages & 1, &failed)) break;
            tmem_fence_after();
            const uint8_t *at = base + s * S::bytes;
            const uint64_t db = operand_descriptor(smem_address(at + S::tiles * S::bytes_w), kTileK * 128);
#pragma unroll
            for (int t = 0; t < S::tiles; ++t) {
                const uint64_t da = operand_descriptor(smem_address(at + t * S::bytes_w), kTileK * 128);
#pragma unroll
                for (int j = 0; j < kTileK / 16; ++j) mma_single(tmem + t * N, da + j * (32 >> 4), db + j * (32 >> 4), idesc, left < p.chain || j > 0);
            }
            mma_commit_single(empty + 8 * s);
        }
        mma_commit_single(done);
        const uint64_t start = nanoseconds();
        while (!barrier_try(done, chunk & 1) && nanoseconds() - start < kWaitLimit) {}
    }
    const int row = (warp & 3) * 32 + lane;                        // of the tile, warps 2 to 5
    float sum[S::tiles][N];
    if (warp >= 2) {
#pragma unroll
        for (int t = 0; t < S::tiles; ++t)
#pragma unroll
            for (int j = 0; j < N; ++j) sum[t][j] = 0.f;
        uint32_t chunk = 0;
        const auto take = [&]() {
            const bool ok = barrier_wait(done, chunk & 1, &failed);
            tmem_fence_after();
#pragma unroll
            for (int t = 0; t < S::tiles; ++t)
#pragma unroll
                for (int q = 0; q < N / 16; ++q) {
                    uint32_t v[16];
                    __syncwarp();
                    tmem_load_16(tmem + ((uint32_t)((warp & 3) * 32) << 16) + t * N + 16 * q, v);
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[t][16 * q + j] += ok && !failed ? __uint_as_float(v[j]) : NAN;
                }
            tmem_fence_before();
        };
        for (int left = k1 - k0 - p.chain; left > 0; left -= p.chain, ++chunk) {
            take();
            __syncwarp();
            if (lane == 0) barrier_arrive_at(taken, rank);
        }
        take();
    }
    const auto store = [&](int t, float a, float b) {
        if (t < p.tokens && row0 + row < p.rows) out[t * p.ldo + row0 + row] = from_float<T>(GATED ? a * logistic<T>(a) * b : a);
    };
    if (splits == 1) {
        if (warp >= 2)
#pragma unroll
            for (int t = 0; t < N; ++t) store(t, sum[0][t], sum[S::tiles - 1][t]);
        __syncthreads();
    } else {
        __syncthreads();                                           // every copy has landed and been used
        float *mine = (float *)base;
        if (warp >= 2)
#pragma unroll
            for (int t = 0; t < S::tiles; ++t)
#pragma unroll
                for (int j = 0; j < N; ++j) mine[(t * N + j) * kTileRows + row] = sum[t][j];
        cluster_sync();
        if (warp >= 2)
            for (int t = rank; t < p.tokens; t += splits) {
                float a = 0.f, b = 0.f;
                for (int r = 0; r < splits; ++r) {
                    a += cluster_load(cluster_address(smem_address(mine + t * kTileRows + row), r));
                    if (GATED) b += cluster_load(cluster_address(smem_address(mine + (N + t) * kTileRows + row), r));
                }
                store(t, a, b);
            }
        cluster_sync();                                            // nobody reads this CTA's sums any more
    }
    if (warp == 1) {
        __syncwarp();
        tmem_fence_after();
        asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" ::"r"(tmem), "n"(S::columns));
    }
}

}  // namespace deft
