// Products on tensor cores whose left operand has consecutive k, with an epilogue of the caller's choice:
//
//     D[b][m][n] = sum_p sum_k A[b][pa(p)][m][k] B[b][pb(p)][n][k]       (or B[...][k][n])
//
// p runs over pairs of 16-bit pieces ("planes") that an operand of more bits is cut into; one pair where there are no pieces.
//
// A pair of CTAs works on a 256 x 256 tile (cta_group::2): each brings half of either operand, 64 deep, in a ring of kStages,
// and holds half of D's rows in tensor memory, two tiles of them, so that the epilogue of one runs under the products of the
// next.  The accumulator is emptied into fp32 registers every `chunk` stages (the matrix unit truncates when it accumulates:
// 1024 terms in a chain keep that at 2e-7 of the magnitudes, 16384 at 7e-6).
//
// Warps: 0 copies (one thread), 1 issues the matrix instructions (one thread of the even CTA), 2 reports to it what has
// landed, the last 8 empty accumulators and store.
#pragma once

#include <cuda.h>

#include "def_sm100.cuh"
#include "def_train_common.cuh"

namespace deft {

constexpr int kTileRows = 128, kTileCols = 256, kTileK = 64;           // of one CTA's accumulator; k per stage
constexpr int kHalfBytes = kTileRows * kTileK * 2;                     // of either operand's half in a stage
constexpr int kStages = 7;
constexpr int kProductThreads = 384;
constexpr int kProductSmem = 1024 + kStages * 2 * kHalfBytes + 256;
constexpr int kShortChain = 16;                                        // stages per accumulator hand-over

struct Product {
    int tiles_m, tiles_n, batch;          // tiles of 256 rows; of 256 columns (gated: 128 of either half)
    int blocks, pairs;                    // stages along k; pairs of planes
    int chunk;
    int planes_a, planes_b;               // of each batch's operands
    uint32_t order_a, order_b;            // plane of each pair, 4 bits each
    int triangle;                         // tiles with n <= m only (tiles_m = tiles_n)
    int step_n, second;                   // columns between tiles; where the second CTA's half of B starts, behind the first's
    int bf16;
};

__device__ __forceinline__ int64_t product_tiles(const Product &p) {
    const int64_t n = p.triangle ? (int64_t)p.tiles_m * (p.tiles_m + 1) / 2 : (int64_t)p.tiles_m * p.tiles_n;
    return n * p.batch;
}
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

// Epilogue: `cols` of each thread's 128 columns start at first(half) and, for the second 64 of them, at second(half);
// store() gets them with the thread's row and its first column, of every row and column of the tile.
template <typename EPILOGUE, bool BN>
__global__ void __launch_bounds__(kProductThreads, 1)
    product_kernel(const Product p, const EPILOGUE epilogue, const __grid_constant__ CUtensorMap map_a, const __grid_constant__ CUtensorMap map_b) {
    extern __shared__ uint8_t raw[];
    uint8_t *base = (uint8_t *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sa = base, *sb = sa + kStages * kHalfBytes;
    uint64_t *bars = (uint64_t *)(sb + kStages * kHalfBytes);
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
            barrier_init(acc_empty + 8 * b, 2 * 8);
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
    const int64_t tiles = product_tiles(p), step = gridDim.x / 2;
    const int per_tile = p.blocks * p.pairs;
    int batch, tm, tn;

    if (warp < 4) {
        registers_down<56>();
        if (warp == 0 && lane == 0) {
            prefetch_map(&map_a);
            prefetch_map(&map_b);
            uint32_t n = 0;
            bool ok = true;
            for (int64_t tile = blockIdx.x / 2; ok && tile < tiles; tile += step) {
                product_place(p, tile, batch, tm, tn);
                const int m0 = tm * 2 * kTileRows + rank * kTileRows, n0 = tn * p.step_n + (rank ? p.second : 0);
                for (int q = 0; ok && q < p.pairs; ++q) {
                    const int za = batch * p.planes_a + (int)(p.order_a >> 4 * q & 15u), zb = batch * p.planes_b + (int)(p.order_b >> 4 * q & 15u);
                    for (int k = 0; k < p.blocks; ++k, ++n) {
                        const uint32_t s = n % kStages, round = n / kStages, bar = full + 8 * s;
                        if (!(ok = barrier_wait(empty + 8 * s, (round & 1) ^ 1, failed))) break;
                        barrier_expect(bar, 2 * kHalfBytes);
                        tensor_load_3d(smem_address(sa + s * kHalfBytes), &map_a, k * kTileK, m0, za, bar);
                        if constexpr (BN) {
#pragma unroll
                            for (int j = 0; j < 2; ++j)
                                tensor_load_3d(smem_address(sb + s * kHalfBytes + j * (kTileK * 128)), &map_b, n0 + 64 * j, k * kTileK, zb, bar);
                        } else {
                            tensor_load_3d(smem_address(sb + s * kHalfBytes), &map_b, k * kTileK, n0, zb, bar);
                        }
                    }
                }
            }
            // the copies in flight end before the CTA does
            const uint64_t start = nanoseconds();
            for (uint32_t m = n > kStages ? n - kStages : 0; m < n; ++m)
                while (!barrier_try(full + 8 * (m % kStages), (m / kStages) & 1) && nanoseconds() - start < kWaitLimit) {}
        } else if (warp == 1 && lane == 0 && rank != 0) {
            const uint64_t start = nanoseconds();                  // the other CTA's last commit arrives here too
            while (!barrier_try(drained, 0) && nanoseconds() - start < 2 * kWaitLimit) {}
        } else if (warp == 1 && lane == 0) {
            const uint32_t idesc = product_descriptor(p.bf16 != 0, BN);
            uint32_t n = 0, chunk = 0;
            bool ok = true;
            for (int64_t tile = blockIdx.x / 2; ok && tile < tiles; tile += step) {
                for (int k = 0; k < per_tile && ok; ++chunk) {
                    const uint32_t buf = chunk & 1, round = chunk >> 1;
                    if (!(ok = barrier_wait(acc_empty + 8 * buf, (round & 1) ^ 1, failed))) break;
                    tmem_fence_after();
                    const int stop = k + p.chunk < per_tile ? k + p.chunk : per_tile;
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
            const uint64_t start = nanoseconds();
            while (!barrier_try(drained, 0) && nanoseconds() - start < kWaitLimit) {}
        } else if (warp == 2 && lane == 0) {
            uint32_t n = 0;
            bool ok = true;
            for (int64_t tile = blockIdx.x / 2; ok && tile < tiles; tile += step)
                for (int k = 0; k < per_tile; ++k, ++n) {
                    if (!(ok = barrier_wait(full + 8 * (n % kStages), (n / kStages) & 1, failed))) break;
                    barrier_arrive_at(ready + 8 * (n % kStages), 0);
                }
        }
    } else {
        registers_up<224>();
        const int half = (warp & 7) >> 2, quarter = warp & 3;       // lanes quarter * 32..
        const int row = quarter * 32 + lane;
        const uint32_t source = tmem + ((uint32_t)(quarter * 32) << 16);
        const uint32_t c0 = EPILOGUE::first(half), c1 = EPILOGUE::second(half);
        uint32_t chunk = 0;
        bool ok = true;
        for (int64_t tile = blockIdx.x / 2; tile < tiles; tile += step) {
            product_place(p, tile, batch, tm, tn);
            float acc[128];
            for (int k = 0; k < per_tile; k += p.chunk, ++chunk) {
                const uint32_t buf = chunk & 1, round = chunk >> 1;
                ok = ok && barrier_wait(acc_full + 8 * buf, round & 1, failed);
                if (__any_sync(0xffffffffu, !ok)) break;
                tmem_fence_after();
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    uint32_t v[16];
                    tmem_load_16(source + buf * kTileCols + (q < 4 ? c0 + q * 16 : c1 + (q - 4) * 16), v);
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[q * 16 + i] = (k > 0 ? acc[q * 16 + i] : 0.f) + __uint_as_float(v[i]);
                }
                tmem_fence_before();
                __syncwarp();
                if (lane == 0) barrier_arrive_at(acc_empty + 8 * buf, 0);
            }
            if (*failed) {                                          // a wait ran out: no numbers rather than wrong ones
                ok = false;
#pragma unroll
                for (int i = 0; i < 128; ++i) acc[i] = NAN;
            }
            epilogue.store(acc, batch, (int64_t)tm * 2 * kTileRows + rank * kTileRows + row, (int64_t)tn * p.step_n, half, tm == tn);
        }
    }
    tmem_fence_before();
    __syncthreads();
    cluster_sync();                                                // nothing of this CTA is used by the other any more
    if (warp == 1) {
        __syncwarp();
        tmem_free<512>(tmem);
    }
}

// ---------------------------------------------------------------------------
// Epilogues.  A thread has 128 columns of one row: runs of 32 of them are stored in 16-byte words where the rows allow it.
// ---------------------------------------------------------------------------
template <typename T> __device__ __forceinline__ void store_32(T *p, int n, bool wide, const float (&v)[32]) {
    if (wide && n >= 32) {
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            float part[8];
#pragma unroll
            for (int j = 0; j < 8; ++j) part[j] = v[8 * i + j];
            store_floats<T, 8>(p + 8 * i, part);
        }
    } else {
#pragma unroll
        for (int i = 0; i < 32; ++i)
            if (i < n) p[i] = from_float<T>(v[i]);
    }
}

// out [rows, cols] <- D.
template <typename T> struct StoreRows {
    T *out;
    int64_t ld, rows, cols;
    int wide;
    static __device__ __forceinline__ uint32_t first(int half) { return half * 128; }
    static __device__ __forceinline__ uint32_t second(int half) { return half * 128 + 64; }
    __device__ __forceinline__ void store(const float (&acc)[128], int, int64_t row, int64_t col, int half, bool) const {
        if (row >= rows) return;
        col += half * 128;
#pragma unroll
        for (int g = 0; g < 4; ++g) {
            if (col + 32 * g >= cols) break;
            float v[32];
#pragma unroll
            for (int i = 0; i < 32; ++i) v[i] = acc[32 * g + i];
            const int64_t left = cols - col - 32 * g;
            store_32<T>(out + row * ld + col + 32 * g, left < 32 ? (int)left : 32, wide, v);
        }
    }
};

}  // namespace deft
