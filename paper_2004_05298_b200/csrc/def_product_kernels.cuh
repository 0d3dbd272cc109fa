// Products on tensor cores whose left operand has consecutive k, with an epilogue of the caller's choice:
//
//     D[b][m][n] = sum_p sum_k A[b][pa(p)][m][k] B[b][pb(p)][n][k]       (or B[...][k][n])
//
// p runs over pairs of 16-bit pieces ("planes") that an operand of more bits is cut into; one pair where there are no pieces.
//
// A pair of CTAs works on a 256 x 256 tile (cta_group::2): each brings half of either operand, 64 deep, in a ring of kStages,
// and holds half of D's rows in tensor memory, two tiles of them, so that the epilogue of one runs under the products of the
// next.  The matrix unit truncates when it accumulates, so where a result keeps more than 16 bits the accumulator is
// emptied into fp32 registers every CHAIN stages of 64 terms (0: at the end only, for sums that are short beside what their
// rounding takes away).
//
// Bound by the matrix unit (measured peak 1.66 PFLOP/s) where the last round of tiles is full: 8192 x 4096 x 10240 bf16 425 us (1.62
// PFLOP/s), gated with checkpoints 1000 (1.38), backward activation 570 (1.20, its epilogue); small ones by two launches,
// 12 us together.
//
// Warps: 0 copies (one thread), 1 issues the matrix instructions (one thread of the even CTA), 2 reports to it what has
// landed, the last 8 or 16 empty accumulators and store, 128 or 64 columns of a row per thread.
#pragma once

#include <cuda.h>

#include "def_sm100.cuh"
#include "def_train_common.cuh"

namespace deft {

constexpr int kTileRows = 128, kTileCols = 256, kTileK = 64;           // of one CTA's accumulator; k per stage
constexpr int kHalfBytes = kTileRows * kTileK * 2;                     // of either operand's half in a stage
constexpr int kStages = 6;
constexpr int kTurnBytes = 2048;                                       // per storing warp: rows that are turned before they are stored
// Sums in registers need them for 128 columns a thread where chains are short, of 8 warps; else 16 warps keep up with more at a
// time, also where a few of their registers are spilled (64 columns each; gated, 8192 x 1024 x 4096 bf16: 137 us against 166).
template <typename EPILOGUE, int CHAIN> struct ProductShape {
    static constexpr int store_warps = CHAIN == 0 || CHAIN >= 8 || EPILOGUE::kBoth ? 16 : 8, threads = 128 + 32 * store_warps;
    static constexpr int control_registers = 56, store_registers = store_warps == 8 ? 224 : 104;     // a thread's, of the first 4 warps and of the others
    static constexpr int smem = 1024 + kStages * 2 * kHalfBytes + store_warps * kTurnBytes + 256;
    // The storing warps take over registers that the others give up: those have to be there (launch bounds give multiples of 8).
    static_assert(65536 / threads / 8 * 8 * threads >= 128 * control_registers + 32 * store_warps * store_registers);
};
constexpr int64_t kPartFloats = (int64_t)kTileRows * kTileCols;        // of a CTA's part of a tile

struct Product {
    int tiles_m, tiles_n, batch;          // tiles of 256 rows; of 256 columns (gated: 128 of either half)
    int blocks, pairs;                    // stages along k; pairs of planes
    int planes_a, planes_b;               // of each batch's operands
    uint32_t order_a, order_b;            // plane of each pair, 4 bits each
    int triangle;                         // tiles with n <= m only (tiles_m = tiles_n)
    int step_n, second;                   // columns between tiles; where the second CTA's half of B starts, behind the first's
    int bf16;
    int64_t whole;                        // tiles [0, whole) are worked on whole, of the others each k in `cuts` parts
    int cuts;
    int early;                            // the next kernel may be set up while this one runs: where half the SMs are idle
    float *parts;                         // [(tile - whole) * cuts + cut][CTA of the pair][column][row]
};

__host__ __device__ inline int64_t product_tiles(const Product &p) {
    const int64_t n = p.triangle ? (int64_t)p.tiles_m * (p.tiles_m + 1) / 2 : (int64_t)p.tiles_m * p.tiles_n;
    return n * p.batch;
}
// Pieces of work, dealt to the pairs of CTAs in turn: first whole tiles, then the cuts of the others.
__host__ __device__ inline int64_t product_pieces(const Product &p) { return p.whole + (product_tiles(p) - p.whole) * p.cuts; }
struct Piece {
    int64_t tile;
    int k0, k1;                           // stages
    __device__ Piece(const Product &p, int i) {
        const int per_tile = p.blocks * p.pairs;
        if (i < p.whole) {
            tile = i;
            k0 = 0;
            k1 = per_tile;
        } else {
            const int64_t j = i - p.whole, cut = j % p.cuts;
            tile = p.whole + j / p.cuts;
            k0 = (int)(per_tile * cut / p.cuts);
            k1 = (int)(per_tile * (cut + 1) / p.cuts);
        }
    }
};
// Tiles in bands of 8 along m, so that the CTAs at work at one time share rows of A and of B in the L2.
__device__ __forceinline__ void product_place(const Product &p, int64_t tile, int &batch, int &m, int &n) {
    if (p.triangle) {
        const int64_t each = (int64_t)p.tiles_m * (p.tiles_m + 1) / 2, r = tile % each;
        batch = (int)(tile / each);
        m = (int)((sqrtf(8.f * (float)r + 1.f) - 1.f) * 0.5f);
        while ((int64_t)(m + 1) * (m + 2) / 2 <= r) ++m;
        while ((int64_t)m * (m + 1) / 2 > r) --m;
        n = (int)(r - (int64_t)m * (m + 1) / 2);
    } else {
        const int64_t each = (int64_t)p.tiles_m * p.tiles_n, t = tile % each, band = t / (8LL * p.tiles_n), r = t - band * 8 * p.tiles_n;
        batch = (int)(tile / each);
        const int wide = (int)(p.tiles_m - band * 8 < 8 ? p.tiles_m - band * 8 : 8);
        m = (int)(band * 8 + r % wide);
        n = (int)(r / wide);
    }
}

// D (fp32) = A B: A with k consecutive, B with k or (b_n) n consecutive.
__device__ __forceinline__ uint32_t product_descriptor(bool bf16, bool b_n) {
    return 1u << 4 | (bf16 ? 1u : 0u) << 7 | (bf16 ? 1u : 0u) << 10 | (b_n ? 1u : 0u) << 16 | (uint32_t)(kTileCols >> 3) << 17 |
           (uint32_t)(2 * kTileRows >> 4) << 24;
}

// 32 columns of the accumulator: as they are, or added to what there is, two at a time.
__device__ __forceinline__ void take_columns(uint32_t from, float (&x)[32]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        uint32_t v[16];
        tmem_load_16(from + 16 * q, v);
#pragma unroll
        for (int j = 0; j < 16; ++j) x[16 * q + j] = __uint_as_float(v[j]);
    }
}
__device__ __forceinline__ void add_columns(uint32_t from, Pair (&x)[16]) {
#pragma unroll
    for (int q = 0; q < 2; ++q) {
        uint32_t v[16];
        tmem_load_16(from + 16 * q, v);
#pragma unroll
        for (int j = 0; j < 8; ++j) x[8 * q + j] = pair_add(x[8 * q + j], make_pair(__uint_as_float(v[2 * j]), __uint_as_float(v[2 * j + 1])));
    }
}
__device__ __forceinline__ void split_columns(const Pair (&x)[16], float (&out)[32]) {
#pragma unroll
    for (int j = 0; j < 16; ++j) split_pair(x[j], out[2 * j], out[2 * j + 1]);
}

// Epilogue: store() gets 32 columns of a row per thread at a time, columns 32 u of the tile on for u < 8, or (kBoth) for u < 4
// those and 32 columns from 128 + 32 u on; whole warps call it, with rows and columns that may lie outside the result.
template <typename EPILOGUE, bool BN, int CHAIN>
__global__ void __launch_bounds__(ProductShape<EPILOGUE, CHAIN>::threads, 1)
    product_kernel(const __grid_constant__ Product p, const __grid_constant__ EPILOGUE epilogue, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b) {
    using S = ProductShape<EPILOGUE, CHAIN>;
    extern __shared__ uint8_t raw[];
    uint8_t *base = (uint8_t *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sa = base, *sb = sa + kStages * kHalfBytes;
    uint8_t *turns = sb + kStages * kHalfBytes;
    uint64_t *bars = (uint64_t *)(turns + S::store_warps * kTurnBytes);
    const uint32_t full = smem_address(bars), empty = full + 8 * kStages, ready = empty + 8 * kStages, acc_full = ready + 8 * kStages,
                   acc_empty = acc_full + 16, drained = acc_empty + 16;
    uint32_t *tmem_slot = (uint32_t *)(bars + 3 * kStages + 5);
    volatile int *failed = (volatile int *)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kStages; ++s) {
            barrier_init(full + 8 * s, 1);
            barrier_init(empty + 8 * s, 1);
            barrier_init(ready + 8 * s, 2);
        }
        for (int b = 0; b < 2; ++b) {
            barrier_init(acc_full + 8 * b, 1);
            barrier_init(acc_empty + 8 * b, 2 * S::store_warps);
        }
        barrier_init(drained, 1);
        *failed = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    }
    if (warp == 1) {
        __syncwarp();
        tmem_alloc<512>(smem_address(tmem_slot));
    }
    tmem_fence_before();
    __syncthreads();
    cluster_sync();
    tmem_fence_after();
    const uint32_t tmem = *tmem_slot;
    asm volatile("griddepcontrol.wait;" ::: "memory");             // the set-up above may overlap the kernel before
    if (p.early) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    const int pieces = (int)product_pieces(p), step = (int)gridDim.x / 2;   // the host keeps them below 2^30
    int batch, tm, tn;

    if (warp < 4) {
        registers_down<S::control_registers>();
        if (warp == 0 && lane == 0) {
            prefetch_map(&map_a);
            prefetch_map(&map_b);
            uint32_t n = 0;
            bool ok = true;
            for (int i = (int)blockIdx.x / 2; ok && i < pieces; i += step) {
                const Piece w(p, i);
                product_place(p, w.tile, batch, tm, tn);
                const int m0 = tm * 2 * kTileRows + rank * kTileRows, n0 = tn * p.step_n + (rank ? p.second : 0);
                for (int k = w.k0; k < w.k1; ++k, ++n) {
                    const uint32_t s = n % kStages, round = n / kStages, bar = full + 8 * s;
                    if (!(ok = barrier_wait(empty + 8 * s, (round & 1) ^ 1, failed))) break;
                    const int q = k / p.blocks, at = (k - q * p.blocks) * kTileK;
                    const int za = batch * p.planes_a + (int)(p.order_a >> 4 * q & 15u), zb = batch * p.planes_b + (int)(p.order_b >> 4 * q & 15u);
                    barrier_expect(bar, 2 * kHalfBytes);
                    tensor_load_3d(smem_address(sa + s * kHalfBytes), &map_a, at, m0, za, bar);
                    if constexpr (BN) {
#pragma unroll
                        for (int j = 0; j < 2; ++j)
                            tensor_load_3d(smem_address(sb + s * kHalfBytes + j * (kTileK * 128)), &map_b, n0 + 64 * j, at, zb, bar);
                    } else {
                        tensor_load_3d(smem_address(sb + s * kHalfBytes), &map_b, at, n0, zb, bar);
                    }
                }
            }
            // the copies in flight end before the CTA does
            const uint64_t start = nanoseconds();
            for (uint32_t m = n > kStages ? n - kStages : 0; m < n; ++m)
                while (!barrier_try(full + 8 * (m % kStages), (m / kStages) & 1) && nanoseconds() - start < kWaitLimit) {}
        } else if (warp == 1 && lane == 0 && rank == 0) {
            const uint32_t idesc = product_descriptor(p.bf16 != 0, BN);
            uint32_t n = 0, chunk = 0;
            bool ok = true;
            for (int i = (int)blockIdx.x / 2; ok && i < pieces; i += step) {
                const Piece w(p, i);
                for (int k = w.k0; k < w.k1 && ok; ++chunk) {
                    const uint32_t buf = chunk & 1, round = chunk >> 1;
                    if (!(ok = barrier_wait(acc_empty + 8 * buf, (round & 1) ^ 1, failed))) break;
                    tmem_fence_after();
                    const int stop = CHAIN && k + CHAIN < w.k1 ? k + CHAIN : w.k1;
                    for (int first = k; k < stop; ++k, ++n) {
                        const uint32_t s = n % kStages;
                        if (!(ok = barrier_wait(ready + 8 * s, (n / kStages) & 1, failed))) break;   // in both CTAs
                        tmem_fence_after();
                        // 16 further along k: 32 bytes within the 128-byte rows, or (BN) 16 rows
                        const uint64_t da = operand_descriptor(smem_address(sa + s * kHalfBytes), kTileK * 128);
                        const uint64_t db = operand_descriptor(smem_address(sb + s * kHalfBytes), kTileK * 128);
#pragma unroll
                        for (int j = 0; j < kTileK / 16; ++j)
                            mma(tmem + buf * kTileCols, da + j * (32 >> 4), db + j * ((BN ? 2048 : 32) >> 4), idesc, k > first || j > 0);
                        mma_commit(empty + 8 * s);
                    }
                    if (ok) mma_commit(acc_full + 8 * buf);
                }
            }
            mma_commit(drained);
        } else if (warp == 2 && lane == 0) {
            uint32_t n = 0;
            bool ok = true;
            for (int i = (int)blockIdx.x / 2; ok && i < pieces; i += step) {
                const Piece w(p, i);
                for (int k = w.k0; k < w.k1; ++k, ++n) {
                    if (!(ok = barrier_wait(full + 8 * (n % kStages), (n / kStages) & 1, failed))) break;
                    barrier_arrive_at(ready + 8 * (n % kStages), 0);
                }
            }
        }
    } else {
        registers_up<S::store_registers>();
        // a warp's columns, in units of 32: kUnits from its group's first on
        constexpr int kAll = EPILOGUE::kBoth ? 4 : 8, kUnits = kAll * 4 / S::store_warps, kSums = EPILOGUE::kBoth ? 2 * kUnits : kUnits;
        const int unit = ((warp - 4) >> 2) * kUnits, quarter = warp & 3;      // lanes quarter * 32..
        const int row = quarter * 32 + lane;
        const uint32_t source = tmem + ((uint32_t)(quarter * 32) << 16);
        uint8_t *turn = turns + (warp - 4) * kTurnBytes;
        uint32_t chunk = 0;
        bool ok = true;
        for (int i = (int)blockIdx.x / 2; i < pieces; i += step) {
            const Piece w(p, i);
            const bool cut = i >= p.whole && p.cuts > 1;
            // where this thread's columns belong
            const auto place = [&](int64_t &r0, int64_t &n0) {
                product_place(p, w.tile, batch, tm, tn);
                r0 = (int64_t)tm * 2 * kTileRows + rank * kTileRows + row;
                n0 = (int64_t)tn * p.step_n;
            };
            float a[32], b[32];
            const auto put = [&](int u) {                           // a (and b), the columns of unit u
                if (__any_sync(0xffffffffu, !ok || *failed)) {      // a wait ran out: no numbers rather than wrong ones
                    ok = false;
#pragma unroll
                    for (int j = 0; j < 32; ++j) a[j] = b[j] = NAN;
                }
                if (!cut) {
                    int64_t r0, n0;
                    place(r0, n0);
                    epilogue.store(a, b, batch, r0, n0 + 32 * u, turn);
                } else {
                    float *parts = p.parts + ((i - p.whole) * 2 + rank) * kPartFloats + 32 * u * kTileRows + row;
#pragma unroll
                    for (int j = 0; j < 32; ++j) {
                        parts[j * kTileRows] = a[j];
                        if (EPILOGUE::kBoth) parts[(128 + j) * kTileRows] = b[j];
                    }
                }
            };
            const auto release = [&](uint32_t buf) {
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive_at(acc_empty + 8 * buf, 0);
            };
            if constexpr (CHAIN > 0) {
                Pair sum[kSums][16];
#pragma unroll
                for (int u = 0; u < kSums; ++u)
#pragma unroll
                    for (int j = 0; j < 16; ++j) sum[u][j] = make_pair(0.f, 0.f);
                for (int k = w.k0; k < w.k1; k += CHAIN, ++chunk) {
                    const uint32_t buf = chunk & 1, round = chunk >> 1;
                    ok = ok && barrier_wait(acc_full + 8 * buf, round & 1, failed);
                    if (__any_sync(0xffffffffu, !ok)) break;
                    tmem_fence_after();
#pragma unroll
                    for (int u = 0; u < kUnits; ++u) {
                        add_columns(source + buf * kTileCols + 32 * (unit + u), sum[u]);
                        if constexpr (EPILOGUE::kBoth) add_columns(source + buf * kTileCols + 128 + 32 * (unit + u), sum[kUnits + u]);
                    }
                    release(buf);
                }
#pragma unroll 1
                for (int u = 0; u < kUnits; ++u) {                  // one copy of the epilogue's code: the sums move up
                    split_columns(sum[0], a);
                    if constexpr (EPILOGUE::kBoth) split_columns(sum[kUnits], b);
                    put(unit + u);
#pragma unroll
                    for (int v = 0; v + 1 < kSums; ++v)
#pragma unroll
                        for (int j = 0; j < 16; ++j) sum[v][j] = sum[v + 1][j];
                }
            } else {
                const uint32_t buf = chunk & 1, round = chunk >> 1;
                ++chunk;
                ok = ok && barrier_wait(acc_full + 8 * buf, round & 1, failed);
                ok = __all_sync(0xffffffffu, ok);
                tmem_fence_after();
#pragma unroll 1
                for (int u = 0; u < kUnits; ++u) {                  // the accumulator holds the later units' columns meanwhile
                    if (ok) {
                        take_columns(source + buf * kTileCols + 32 * (unit + u), a);
                        if (EPILOGUE::kBoth) take_columns(source + buf * kTileCols + 128 + 32 * (unit + u), b);
                        if (u == kUnits - 1) release(buf);
                    }
                    put(unit + u);
                }
            }
        }
    }
    tmem_fence_before();
    __syncthreads();
    if (threadIdx.x == 32) {                                       // the even CTA's last commit arrives in both
        const uint64_t start = nanoseconds();
        while (!barrier_try(drained, 0) && nanoseconds() - start < kWaitLimit) {}
    }
    __syncwarp();
    cluster_sync();                                                // nothing of this CTA is used by the other any more
    if (warp == 1) {
        __syncwarp();
        tmem_free<512>(tmem);
    }
}

// The tiles whose k was cut: their parts, added in order, and the same epilogue.  A thread's 32 columns (kBoth: 64) of several
// parts are on their way at once, and a CTA has 128 rows of no more, so that few tiles are spread over many SMs: joins wait for
// memory.  (256 threads, one part at a time: 256 x 256 orthogonalised 206 against 190 us, 512 x 512 x 1408 fp32 backward 42 against 32.)
constexpr int kJoinThreads = 128;
template <typename EPILOGUE>
__global__ void __launch_bounds__(kJoinThreads) product_join_kernel(const Product p, const EPILOGUE epilogue) {
    __shared__ uint4 turns[kJoinThreads / 32][kTurnBytes / 16];
    constexpr int kRuns = EPILOGUE::kBoth ? 4 : 8, kAtOnce = EPILOGUE::kBoth ? 2 : 4;
    const int64_t half_tile = blockIdx.x / kRuns, tile = half_tile / 2;
    const int rank = (int)(half_tile % 2), ca = (int)(blockIdx.x % kRuns) * 32, row = threadIdx.x;
    asm volatile("griddepcontrol.wait;" ::: "memory");             // the parts are those of the kernel before
    if (p.early) asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
    float a[32], b[32];
#pragma unroll
    for (int j = 0; j < 32; ++j) a[j] = b[j] = 0.f;
    for (int c = 0; c < p.cuts; c += kAtOnce) {
        float va[kAtOnce][32], vb[kAtOnce][32];
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u) {
            const float *in = p.parts + ((tile * p.cuts + c + u) * 2 + rank) * kPartFloats + ca * kTileRows + row;
            const bool there = c + u < p.cuts;
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                va[u][j] = there ? in[j * kTileRows] : 0.f;
                if (EPILOGUE::kBoth) vb[u][j] = there ? in[(128 + j) * kTileRows] : 0.f;
            }
        }
#pragma unroll
        for (int u = 0; u < kAtOnce; ++u)
#pragma unroll
            for (int j = 0; j < 32; ++j) {
                a[j] += va[u][j];
                if (EPILOGUE::kBoth) b[j] += vb[u][j];
            }
    }
    int batch, tm, tn;
    product_place(p, p.whole + tile, batch, tm, tn);
    epilogue.store(a, b, batch, (int64_t)tm * 2 * kTileRows + rank * kTileRows + row, (int64_t)tn * p.step_n + ca, (uint8_t *)turns[threadIdx.x / 32]);
}

// ---------------------------------------------------------------------------
// Stores of a warp's 32 rows by 32 columns, a row per thread.  They are turned in shared memory first, so that a store
// instruction writes whole sectors of few rows rather than 16 bytes of 32 rows: words of 16 bytes where the rows allow it,
// kTurn elements of a row at a time elsewhere.
// ---------------------------------------------------------------------------

// 32 rows of P bytes (64 or 32) in words of 16; no two lanes of a quarter warp in one bank, putting or taking.
template <int P> __device__ __forceinline__ uint4 *turn_word(uint8_t *turn, int row, int word) {
    return reinterpret_cast<uint4 *>(turn + row * P + (P == 64 ? word ^ (row >> 1 & 3) : word ^ (row >> 2 & 1)) * 16);
}
template <int P> __device__ __forceinline__ void turn_put_word(uint8_t *turn, int word, const uint4 &v) { *turn_word<P>(turn, threadIdx.x & 31, word) = v; }
// 8 elements from column c (a multiple of 8) of those P bytes on.
template <int P, typename T> __device__ __forceinline__ void turn_put_8(uint8_t *turn, int c, const float (&x)[8]) {
    const Frag<T, 8> f = round_run<T>(x);
    uint4 w[sizeof(T) / 2];
    memcpy(w, &f, sizeof(f));
#pragma unroll
    for (int i = 0; i < (int)sizeof(T) / 2; ++i) turn_put_word<P>(turn, c * (int)sizeof(T) / 16 + i, w[i]);
}
// What all lanes put there goes to p (this lane's row); `there`: the row exists.  Rows that exist come first.
template <int P> __device__ __forceinline__ void turn_store_words(uint8_t *turn, void *p, int64_t pitch, bool there) {
    constexpr int kWords = P / 16, kRows = 32 / kWords;             // rows that a warp stores at a time
    const int lane = threadIdx.x & 31, rows = __popc(__ballot_sync(0xffffffffu, there)), sub = lane / kWords, word = lane % kWords;
    char *out = (char *)p + (sub - lane) * pitch + word * 16;
    __syncwarp();
#pragma unroll
    for (int i = 0; i < kWords; ++i, out += kRows * pitch)
        if (sub + i * kRows < rows) *reinterpret_cast<uint4 *>(out) = *turn_word<P>(turn, sub + i * kRows, word);
    __syncwarp();
}

template <typename T> constexpr int kTurn = 64 / (int)sizeof(T);                       // columns that kTurnBytes hold
template <typename T, int W> __device__ __forceinline__ int turn_place(int row, int c) {
    // no two lanes of a warp that puts (one column, all rows) or takes in one bank, but for the narrowest
    return row * W + (c ^ (sizeof(T) == 4 ? row >> (W == 16 ? 1 : 2) & (W - 1) : W == 32 ? row & 30 : row >> 1 & 14));
}
template <typename T, int W> __device__ __forceinline__ void turn_put(uint8_t *turn, int c, float v) {
    reinterpret_cast<T *>(turn)[turn_place<T, W>(threadIdx.x & 31, c)] = from_float<T>(v);
}
// The first n <= W columns put there by all lanes go to p (this lane's row and the first column); `there`: the row exists.
template <typename T, int W> __device__ __forceinline__ void turn_store(const uint8_t *turn, T *p, int64_t ld, bool there, int n) {
    constexpr int kRows = 32 / W;                                  // rows that a warp stores at a time
    const int lane = threadIdx.x & 31, rows = __popc(__ballot_sync(0xffffffffu, there)), sub = lane / W, c = lane % W;
    T *out = p + (sub - lane) * ld + c;                            // rows that exist come first
    __syncwarp();
    if (c < n) {
#pragma unroll 8
        for (int r = sub; r < rows; r += kRows, out += kRows * ld) *out = reinterpret_cast<const T *>(turn)[turn_place<T, W>(r, c)];
    }
    __syncwarp();
}
template <typename T, typename V> __device__ __forceinline__ void store_32(T *p, int64_t ld, bool there, int n, bool wide, const V &v, uint8_t *turn) {
    if (wide && n >= 32) {
#pragma unroll
        for (int f = 0; f < 32; f += 8) {
            float part[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) part[j] = v[f + j];
            turn_put_8<64, T>(turn, f % kTurn<T>, part);
            if (f % kTurn<T> + 8 == kTurn<T>) turn_store_words<64>(turn, p + f + 8 - kTurn<T>, ld * (int64_t)sizeof(T), there);
        }
    } else {
        constexpr int W = kTurn<T>;
#pragma unroll
        for (int f = 0; f < 32; f += W) {
            if (f >= n) break;
#pragma unroll
            for (int j = 0; j < W; ++j) turn_put<T, W>(turn, j, v[f + j]);
            turn_store<T, W>(turn, p + f, ld, there, n - f);
        }
    }
}

// out [rows, cols] <- D.
template <typename T> struct StoreRows {
    static constexpr bool kBoth = false;
    T *out;
    int64_t ld, rows, cols;
    int wide;
    __device__ __forceinline__ void store(float (&a)[32], float (&)[32], int, int64_t row, int64_t col, uint8_t *turn) const {
        if (col >= cols) return;
        const int64_t left = cols - col;
        store_32<T>(out + row * ld + col, ld, row < rows, left < 32 ? (int)left : 32, wide, a, turn);
    }
};

}  // namespace deft
