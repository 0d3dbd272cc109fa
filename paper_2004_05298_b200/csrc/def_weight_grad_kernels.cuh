// Weight gradient of a linear layer from the 8-bit checkpoint of its input (see include/def_train.h).
//
//     dw[o, i] = sum_t dy[t, o] x^[t, i],     x^ = q 2^k
//
// Tensor cores (tcgen05), D = A B with A = x^ (M runs over i), B = dy (N runs over o), k over tokens: both operands lie
// in memory with M resp. N consecutive, which is how they are fed; D's lanes are i, so that a store of one column of D
// is 128 consecutive floats of a row of dw, whatever dw's alignment.  q 2^k is exact in bf16, products are exact, and the
// accumulator in tensor memory is emptied into fp32 registers every kChunk blocks of tokens: the matrix unit truncates
// when it accumulates (16384 tokens in one chain are 7e-6 off), and a chain of 1024 keeps that at 2e-7.
//
// A pair of CTAs works on a 256 x 256 tile (cta_group::2): each brings half of either operand, which halves the reads of
// shared memory per product.  8192 tokens, 8192 x 4096, bf16: 390 to 413 us in a burst (1.3 to 1.4 PFLOP/s, tensor pipe 81 %
// busy), 470 in a loop of seconds under the power cap; the same with 128 x 256 tiles of single CTAs: 530 in a burst.
#pragma once

#include <cuda.h>

#include "def_sm100.cuh"
#include "def_train_common.cuh"

namespace deft {

constexpr int kTileI = 128, kTileO = 256, kTileT = 64;      // of one CTA's accumulator, and tokens per pipeline stage
constexpr int kPairI = 2 * kTileI, kHalfO = kTileO / 2;      // a pair's rows of D; the columns of dy each CTA brings
constexpr int kChunk = 16;                                   // stages per accumulator hand-over
constexpr int kBytesA = kTileI * kTileT * 2, kBytesB = kHalfO * kTileT * 2, kBytesQ = kTileI * kTileT, kBytesE = kTileT * 16;

// Two ways to the operand x^.  Widening: q is loaded and widened in shared memory by two groups of four warps, each time
// a tile needs it.  Else x^ lies in memory in 16 bits (widened once by a kernel of its own) and is loaded like dy.
// From kWidenOnce tiles along o on the second is faster: 8192 tokens, I = 4096: 4 tiles 72 us against 87, 8 tiles 125 and
// 128, 16 tiles 251 and 216, 32 tiles 470 and 400.
constexpr int kWidenOnce = 12;
template <bool WIDEN> struct GradShape {
    static constexpr int loads = 7, wides = WIDEN ? 3 : 0;   // stages of what is loaded; of widened q
    static constexpr int bytes_x = WIDEN ? kBytesQ + kBytesE : kBytesA;
    static constexpr int threads = 128 + (WIDEN ? 256 : 0) + 256;
    static constexpr int smem = 1024 + wides * kBytesA + loads * (kBytesB + bytes_x) + 256;
};

struct WeightGrad {
    const uint8_t *e;
    float *dw, *partial;                  // partial: [CTA][2][kTileO][kTileI]
    int64_t tokens, O, I, lde;
    int tiles_i, tiles_o, blocks, planes; // blocks: of kTileT tokens, per plane of dy
    int accumulate;
    int64_t whole;                        // tiles [0, whole) go to pairs one by one; the blocks of the others are cut evenly
};

// The pieces of work of one pair of CTAs: (tile, blocks [k0, k1)).  First its share of the whole tiles, then an equal run
// of the blocks of the remaining tiles in order; a tile that is cut goes to partial slot 0 of the pairs that do not hold
// its first block, slot 1 of the one that does.
struct Pieces {
    int64_t tile, pos, end, whole, per_tile;
    __device__ Pieces(const WeightGrad &a) {
        const int64_t pair = blockIdx.x / 2, pairs = gridDim.x / 2;
        per_tile = (int64_t)a.blocks * a.planes;
        whole = a.whole;
        tile = pair;
        const int64_t rest = ((int64_t)a.tiles_i * a.tiles_o - whole) * per_tile;
        pos = rest * pair / pairs;
        end = rest * (pair + 1) / pairs;
    }
    __device__ bool next(int64_t &t, int &k0, int &k1) {
        if (tile < whole) {
            t = tile;
            k0 = 0;
            k1 = (int)per_tile;
            tile += gridDim.x / 2;
            return true;
        }
        if (pos >= end) return false;
        t = pos / per_tile;
        k0 = (int)(pos - t * per_tile);
        k1 = (int)(end - t * per_tile < per_tile ? end - t * per_tile : per_tile);
        pos += k1 - k0;
        t += whole;
        return true;
    }
};

// Tiles in bands of 8 along o, so that the CTAs at work at one time share rows of dy and of q in the L2.
__device__ __forceinline__ void tile_place(const WeightGrad &a, int64_t tile, int &i0, int &o0) {
    const int64_t band = tile / (8LL * a.tiles_i), r = tile - band * 8 * a.tiles_i;
    const int wide = (int)(a.tiles_o - band * 8 < 8 ? a.tiles_o - band * 8 : 8);
    i0 = (int)(r / wide) * kPairI;
    o0 = (int)(band * 8 + r % wide) * kTileO;
}

// 16 bytes of q times 2^k as 16-bit floats.
template <typename T> __device__ __forceinline__ void widen16(uint4 q, uint32_t e, uint4 &lo, uint4 &hi) {
    const uint32_t in[4] = {q.x, q.y, q.z, q.w};
    uint32_t out[8];
    if constexpr (sizeof(T) == 2 && !__is_same(T, __half)) {
        // q = (low 7 bits + 128) - (128 or 256), both exact bf16 numbers made by bit operations
        const uint32_t s = e * 0x00800080u;
        __nv_bfloat162 scale;
        memcpy(&scale, &s, 4);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const uint32_t two = __byte_perm(in[i / 2], 0, i % 2 ? 0x4342 : 0x4140);
            const uint32_t a = (two & 0x007f007fu) | 0x43004300u, b = (two & 0x00800080u) | 0x43004300u;
            __nv_bfloat162 x, y;
            memcpy(&x, &a, 4);
            memcpy(&y, &b, 4);
            x = __hmul2(__hsub2(x, y), scale);
            memcpy(&out[i], &x, 4);
        }
    } else {
        const float scale = group_scale(e);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
            const int a = (int)(int8_t)(in[i / 2] >> (i % 2 * 16)), b = (int)(int8_t)(in[i / 2] >> (i % 2 * 16 + 8));
            const __half2 x = __floats2half2_rn((float)a * scale, (float)b * scale);
            memcpy(&out[i], &x, 4);
        }
    }
    lo = make_uint4(out[0], out[1], out[2], out[3]);
    hi = make_uint4(out[4], out[5], out[6], out[7]);
}

// WIDE_E: rows of e are multiples of 16 bytes, and 16 of them (512 columns) come per token with the other copies; else
// two warps fetch the 4 that a tile needs with one small copy per token, which costs shared memory 15 % of its cycles
// more (4-byte copies from scattered rows are stored one by one).
//
// Warps: 0 copies (one thread), 1 issues the matrix instructions (one thread of the even CTA), 2 and 3 fetch exponents
// (where x^ is loaded, 2 reports its landing instead), the next 8 widen q, the last 8 empty accumulators and store.
template <typename T, bool WIDEN, bool WIDE_E>
__global__ void __launch_bounds__(GradShape<WIDEN>::threads, 1)
    weight_grad_kernel(const WeightGrad a, const __grid_constant__ CUtensorMap map_y, const __grid_constant__ CUtensorMap map_x,
                       const __grid_constant__ CUtensorMap map_e) {
    using S = GradShape<WIDEN>;
    constexpr int kLoads = S::loads, kWides = WIDEN ? S::wides : S::loads;       // x^ is ready wide by wide, or load by load
    constexpr int kRowE = WIDE_E ? 16 : 4;
    extern __shared__ uint8_t raw[];
    uint8_t *base = (uint8_t *)(((uintptr_t)raw + 1023) & ~(uintptr_t)1023);
    uint8_t *sa = base, *sb = sa + kWides * kBytesA, *sq = sb + kLoads * kBytesB, *se = sq + (WIDEN ? kLoads * kBytesQ : 0);
    uint64_t *bars = (uint64_t *)(se + (WIDEN ? kLoads * kBytesE : 0));
    const uint32_t full = smem_address(bars), empty = full + 8 * kLoads, ready = empty + 8 * kLoads, used = ready + 8 * kWides,
                   acc_full = used + 8 * kWides, acc_empty = acc_full + 16, drained = acc_empty + 16;
    uint32_t *tmem_slot = (uint32_t *)(bars + 2 * kLoads + 2 * kWides + 5);
    volatile int *failed = (volatile int *)(tmem_slot + 1);
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const uint32_t rank = cluster_rank();
    if (threadIdx.x == 0) {
        for (int s = 0; s < kLoads; ++s) {
            barrier_init(full + 8 * s, WIDEN && !WIDE_E ? 1 + 64 : 1);
            barrier_init(empty + 8 * s, 1);
        }
        for (int s = 0; s < kWides; ++s) {
            barrier_init(ready + 8 * s, WIDEN ? 2 * 4 : 2);
            barrier_init(used + 8 * s, 1);
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
    Pieces work(a);
    int64_t tile;
    int k0, k1, i0, o0;

    if (warp < 4) {
        if (WIDEN) registers_down<48>();
        if (warp == 0 && lane == 0) {
            prefetch_map(&map_y);
            prefetch_map(&map_x);
            if (WIDEN && WIDE_E) prefetch_map(&map_e);
            uint32_t n = 0;
            bool ok = true;
            while (ok && work.next(tile, k0, k1)) {
                tile_place(a, tile, i0, o0);
                i0 += rank * kTileI;
                for (int k = k0; k < k1; ++k, ++n) {
                    const uint32_t s = n % kLoads, round = n / kLoads;
                    if (!(ok = barrier_wait(empty + 8 * s, (round & 1) ^ 1, failed))) break;
                    const int plane = k / a.blocks, t0 = (k - plane * a.blocks) * kTileT;
                    const uint32_t bar = full + 8 * s;
                    barrier_expect(bar, kBytesB + (!WIDEN ? kBytesA : kBytesQ + (WIDE_E ? kBytesE : 0)));
                    if constexpr (WIDEN) {
                        tensor_load_2d(smem_address(sq + s * kBytesQ), &map_x, i0, t0, bar);
                        if (WIDE_E) tensor_load_2d(smem_address(se + s * kBytesE), &map_e, i0 / kGroup & ~15, t0, bar);
                    } else {
#pragma unroll
                        for (int j = 0; j < kTileI / 64; ++j)
                            tensor_load_2d(smem_address(sa + s * kBytesA + j * (kTileT * 128)), &map_x, i0 + 64 * j, t0, bar);
                    }
#pragma unroll
                    for (int j = 0; j < kHalfO / 64; ++j)
                        tensor_load_3d(smem_address(sb + s * kBytesB + j * (kTileT * 128)), &map_y, o0 + rank * kHalfO + 64 * j, t0, plane, bar);
                }
            }
            // the copies in flight end before the CTA does
            const uint64_t start = nanoseconds();
            for (uint32_t m = n > kLoads ? n - kLoads : 0; m < n; ++m)
                while (!barrier_try(full + 8 * (m % kLoads), (m / kLoads) & 1) && nanoseconds() - start < kWaitLimit) {}
        } else if (warp == 1 && lane == 0 && rank != 0) {
            const uint64_t start = nanoseconds();                  // the other CTA's last commit arrives here too
            while (!barrier_try(drained, 0) && nanoseconds() - start < 2 * kWaitLimit) {}
        } else if (warp == 1 && lane == 0) {
            constexpr uint32_t idesc = instruction_descriptor(!__is_same(T, __half), kPairI, kTileO);
            uint32_t n = 0, chunk = 0;
            bool ok = true;
            while (ok && work.next(tile, k0, k1)) {
                for (int k = k0; k < k1 && ok; ++chunk) {
                    const uint32_t buf = chunk & 1, round = chunk >> 1;
                    if (!(ok = barrier_wait(acc_empty + 8 * buf, (round & 1) ^ 1, failed))) break;
                    tmem_fence_after();
                    const int stop = k + kChunk < k1 ? k + kChunk : k1;
                    for (int first = k; k < stop; ++k, ++n) {
                        const uint32_t w = n % kWides, s = n % kLoads;
                        if (!(ok = barrier_wait(ready + 8 * w, (n / kWides) & 1, failed))) break;   // both CTAs' dy has landed, too
                        tmem_fence_after();
                        const uint64_t da = operand_descriptor(smem_address(sa + w * kBytesA), kTileT * 128);
                        const uint64_t db = operand_descriptor(smem_address(sb + s * kBytesB), kTileT * 128);
#pragma unroll
                        for (int j = 0; j < kTileT / 16; ++j)     // 16 tokens each: 2048 bytes further along k
                            mma(tmem + buf * kTileO, da + j * (2048 >> 4), db + j * (2048 >> 4), idesc, k > first || j > 0);
                        if (WIDEN) mma_commit(used + 8 * w);
                        mma_commit(empty + 8 * s);
                    }
                    if (ok) mma_commit(acc_full + 8 * buf);
                }
            }
            mma_commit(drained);
            const uint64_t start = nanoseconds();
            while (!barrier_try(drained, 0) && nanoseconds() - start < kWaitLimit) {}
        } else if (!WIDEN && warp == 2 && lane == 0) {
            uint32_t n = 0;
            bool ok = true;
            while (ok && work.next(tile, k0, k1))
                for (int k = k0; k < k1; ++k, ++n) {
                    if (!(ok = barrier_wait(full + 8 * (n % kLoads), (n / kLoads) & 1, failed))) break;
                    barrier_arrive_at(ready + 8 * (n % kLoads), 0);
                }
        } else if (WIDEN && !WIDE_E && warp >= 2) {
            const int row = threadIdx.x - 64;                      // token of a stage
            uint32_t n = 0;
            bool ok = true;
            while (ok && work.next(tile, k0, k1)) {
                tile_place(a, tile, i0, o0);
                i0 += rank * kTileI;
                for (int k = k0; k < k1; ++k, ++n) {
                    const uint32_t s = n % kLoads, round = n / kLoads;
                    if (!(ok = barrier_wait(empty + 8 * s, (round & 1) ^ 1, failed))) break;
                    const int64_t t = (int64_t)(k % a.blocks) * kTileT + row;
                    const bool there = t < a.tokens && i0 < a.I;
                    const uint8_t *src = there ? a.e + t * a.lde + i0 / kGroup : a.e;
                    asm volatile("cp.async.ca.shared.global [%0], [%1], 4, %2;" ::"r"(smem_address(se + s * kBytesE + row * 4)), "l"(src),
                                 "r"(there ? 4 : 0)
                                 : "memory");                      // tokens past the end: exponent 0, q is 0 there
                    asm volatile("cp.async.mbarrier.arrive.noinc.shared::cta.b64 [%0];" ::"r"(full + 8 * s) : "memory");
                }
            }
            asm volatile("cp.async.wait_all;" ::: "memory");
        }
    } else if (WIDEN && warp < 12) {
        registers_down<56>();
        // Two groups of four warps take stages in turn.  8 threads per token, 16 columns each: a warp reads four whole
        // rows of q, and then the tokens 16, 32 and 48 further on.
        const int id = threadIdx.x & 127, part = id & 7, row = id >> 3;
        const uint32_t group = (warp - 4) >> 2;
        // The two runs of 64 columns write their even and odd 16-byte pieces alternately: no bank twice.
        const int run = part >> 2, c = (part & 3) * 2 + run;
        const int first = run * (kTileT * 128) + row * 128 + ((c ^ (row & 7)) << 4), second = first ^ 16;
        uint32_t n = 0;
        bool ok = true;
        while (ok && work.next(tile, k0, k1)) {
            tile_place(a, tile, i0, o0);
            i0 += rank * kTileI;
            const int e0 = (WIDE_E ? i0 / kGroup & 15 : 0) + (part >> 1);
            for (int k = k0; k < k1; ++k, ++n) {
                if (n % 2 != group) continue;
                const uint32_t s = n % kLoads, w = n % kWides;
                if (!(ok = barrier_wait(full + 8 * s, (n / kLoads) & 1, failed))) break;
                const uint8_t *q = sq + s * kBytesQ + row * kTileI + part * 16, *e = se + s * kBytesE + row * kRowE + e0;
                uint8_t *out = sa + w * kBytesA;
                uint4 v[4];
                uint32_t ex[4];
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    v[p] = *reinterpret_cast<const uint4 *>(q + p * 16 * kTileI);
                    ex[p] = e[p * 16 * kRowE];
                }
                if (!(ok = barrier_wait(used + 8 * w, ((n / kWides) & 1) ^ 1, failed))) break;
#pragma unroll
                for (int p = 0; p < 4; ++p) {
                    uint4 lo, hi;
                    widen16<T>(v[p], ex[p], lo, hi);
                    *reinterpret_cast<uint4 *>(out + first + p * 16 * 128) = run ? hi : lo;
                    *reinterpret_cast<uint4 *>(out + second + p * 16 * 128) = run ? lo : hi;
                }
                fence_async_shared();
                __syncwarp();
                if (lane == 0) barrier_arrive_at(ready + 8 * w, 0);
            }
        }
    } else {
        if (WIDEN) registers_up<160>();
        const int half = (warp & 7) >> 2, quarter = warp & 3;       // columns half * 128.., lanes quarter * 32..
        const int row = quarter * 32 + lane;
        const uint32_t source = tmem + ((uint32_t)(quarter * 32) << 16) + half * 128;
        uint32_t chunk = 0;
        bool ok = true;
        while (work.next(tile, k0, k1)) {
            tile_place(a, tile, i0, o0);
            i0 += rank * kTileI;
            float acc[128];
#pragma unroll
            for (int i = 0; i < 128; ++i) acc[i] = 0.f;
            for (int k = k0; k < k1; k += kChunk, ++chunk) {
                const uint32_t buf = chunk & 1, round = chunk >> 1;
                ok = ok && barrier_wait(acc_full + 8 * buf, round & 1, failed);
                if (__any_sync(0xffffffffu, !ok)) break;
                tmem_fence_after();
#pragma unroll
                for (int p = 0; p < 8; ++p) {
                    uint32_t v[16];
                    tmem_load_16(source + buf * kTileO + p * 16, v);
#pragma unroll
                    for (int i = 0; i < 16; ++i) acc[p * 16 + i] += __uint_as_float(v[i]);
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
            if (k0 > 0 || k1 < work.per_tile) {
                float *out = a.partial + ((int64_t)blockIdx.x * 2 + (k0 > 0 ? 0 : 1)) * (kTileO * kTileI) + half * 128 * kTileI + row;
#pragma unroll
                for (int i = 0; i < 128; ++i) out[i * kTileI] = acc[i];
            } else if (i0 + row < a.I) {
                float *out = a.dw + (int64_t)(o0 + half * 128) * a.I + i0 + row;
                const int64_t rows = a.O - (o0 + half * 128);
                if (a.accumulate) {
#pragma unroll
                    for (int i = 0; i < 128; ++i)
                        if (i < rows) out[i * a.I] += acc[i];
                } else {
#pragma unroll
                    for (int i = 0; i < 128; ++i)
                        if (i < rows) out[i * a.I] = acc[i];
                }
            }
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

// The tiles that pairs shared: their parts, added in the order of the tokens.  One CTA per 8 rows of dw of half a tile.
__global__ void __launch_bounds__(256) weight_grad_join_kernel(const WeightGrad a, int pairs) {
    const int64_t per_tile = (int64_t)a.blocks * a.planes, all = ((int64_t)a.tiles_i * a.tiles_o - a.whole) * per_tile;
    const int64_t half_tile = blockIdx.x / (kTileO / 8), tile = half_tile / 2;       // of the tiles that were cut
    const int rank = (int)(half_tile % 2);
    const int col = (int)(blockIdx.x % (kTileO / 8)) * 8 + threadIdx.x / 32;
    // pair c holds blocks [all c / pairs, all (c + 1) / pairs): the last pair that starts at or before a block holds it; with
    // fewer blocks than pairs some hold none
    const int64_t begin = tile * per_tile, end = begin + per_tile;
    const int first = (int)(((begin + 1) * pairs - 1) / all), last = (int)((end * pairs - 1) / all);
    asm volatile("griddepcontrol.wait;" ::: "memory");                                // the parts are those of the kernel before
    if (first == last) return;                                                        // whole in one pair: written there
    int i0, o0;
    tile_place(a, a.whole + tile, i0, o0);
    i0 += rank * kTileI;
    const int i = threadIdx.x % 32 * 4;
    if (o0 + col >= a.O || i0 + i >= a.I) return;
    float4 sum = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
    for (int c = first; c <= last; ++c) {                                             // the first holds the tile's first block
        if (all < pairs && all * c / pairs == all * (c + 1) / pairs) continue;
        const float4 v = *reinterpret_cast<const float4 *>(a.partial + (((int64_t)c * 2 + rank) * 2 + (c == first)) * (kTileO * kTileI) + col * kTileI + i);
        sum.x += v.x; sum.y += v.y; sum.z += v.z; sum.w += v.w;
    }
    float *out = a.dw + (int64_t)(o0 + col) * a.I + i0 + i;
    const float v[4] = {sum.x, sum.y, sum.z, sum.w};
#pragma unroll
    for (int j = 0; j < 4; ++j)
        if (i0 + i + j < a.I) out[j] = a.accumulate ? out[j] + v[j] : v[j];
}

// dy as the tensor cores take it, where it is not already: 16-bit pieces in rows of ld elements (a multiple of 8, the last
// ones 0).  16-bit types: a copy, of either type as bits.  fp32: three bf16 numbers of 8 bits each, by truncation, whose
// sum is dy exactly.  A thread takes 8 columns.
template <typename T>
__global__ void __launch_bounds__(256) weight_grad_planes_kernel(const T *__restrict__ dy, int64_t lddy, int64_t tokens, int O,
                                                                 uint4 *__restrict__ out, int64_t ld) {
    const int col = (int)(blockIdx.x * blockDim.x + threadIdx.x) * 8;
    if (col >= O) return;
    for (int64_t t = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; t < tokens; t += (int64_t)gridDim.y * blockDim.y) {
        const Frag<T, 8> f = load_run<T>(dy + t * lddy, col, O);
        if constexpr (sizeof(T) == 2) {
            uint4 w;
            memcpy(&w, &f, sizeof(w));
            out[(t * ld + col) / 8] = w;
        } else {
            Frag<__nv_bfloat16, 8> piece[3];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = f.v[i];
                const bool finite = fabsf(x) <= 3.402823466e38f;
                const float hi = __uint_as_float(__float_as_uint(x) & 0xffff0000u), rest = x - hi;
                const float mid = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
                piece[0].v[i] = from_float<__nv_bfloat16>(finite ? hi : x);
                piece[1].v[i] = from_float<__nv_bfloat16>(finite ? mid : 0.f);
                piece[2].v[i] = from_float<__nv_bfloat16>(finite ? rest - mid : 0.f);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                uint4 w;
                memcpy(&w, &piece[k], sizeof(w));
                out[((k * tokens + t) * ld + col) / 8] = w;
            }
        }
    }
}

}  // namespace deft
