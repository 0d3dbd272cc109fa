// Norms before and after a block, fused with its gate and residual scale (see include/def_train.h).
#pragma once

#include "def_sm100.cuh"
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
    int64_t parts_per_group;             // of the stream kernel
    float res_scale, eps, inv_C;
};

// One CTA per row; the row stays in registers between its two norms.
template <typename T, bool ALIGNED, int MOST, int ITERS>
__global__ void __launch_bounds__(MOST) norm_forward_kernel(const NormForward a) {
    __shared__ float scratch[2][32];
    const int C = (int)a.C, threads = (int)blockDim.x;
    for (int64_t t = blockIdx.x; t < a.T; t += gridDim.x) {
        float h[ITERS][8];
        const T *hr = (const T *)a.h + t * a.ldh;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * threads + (int)threadIdx.x) * 8;
            Frag<T, 8> f = zeros<T, 8>();
            if (col < C) f = load_cols<T, ALIGNED>(hr, col, C);
            to_floats<T, 8>(f, h[it]);
        }
        float sum = 0.f;
        if (a.b) {
            float b[ITERS][8];
            const T *br = (const T *)a.b + t * a.ldb;
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int col = (it * threads + (int)threadIdx.x) * 8;
                Frag<T, 8> f = zeros<T, 8>();
                if (col < C) f = load_cols<T, ALIGNED>(br, col, C);
                to_floats<T, 8>(f, b[it]);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(b[it][i], b[it][i], sum);
            }
            if (a.hb.q)
#pragma unroll
                for (int it = 0; it < ITERS; ++it) {
                    const int col = (it * threads + (int)threadIdx.x) * 8;
                    store_held<ALIGNED>(a.hb.q + t * a.ldq, a.hb.e + t * a.lde, col, C, b[it]);
                }
            sum = cta_sum(sum, scratch[0]);
            const float r = rsqrtf(fmaf(sum, a.inv_C, a.eps));
            if (threadIdx.x == 0) a.rstd_post[t] = r;
            const float *gate = a.gate ? a.gate + t / a.rows_per_group * a.C : nullptr;
            T *ho = (T *)a.h_out + t * a.ldho;
            sum = 0.f;
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int col = (it * threads + (int)threadIdx.x) * 8;
                float w[8], g[8];
                load_params(a.w_post, col, C, w);
                if (gate) {
                    load_params(gate, col, C, g);
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] *= g[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) h[it][i] = fmaf(b[it][i] * r, w[i], a.res_scale * h[it][i]);
                store_cols<T, ALIGNED>(ho, col, C, h[it]);
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(h[it][i], h[it][i], sum);
            }
            if (a.hh.q)
#pragma unroll
                for (int it = 0; it < ITERS; ++it) {
                    const int col = (it * threads + (int)threadIdx.x) * 8;
                    float x[8];
#pragma unroll
                    for (int i = 0; i < 8; ++i) x[i] = to_float<T>(from_float<T>(h[it][i]));   // h' as stored
                    store_held<ALIGNED>(a.hh.q + t * a.ldq, a.hh.e + t * a.lde, col, C, x);
                }
        } else {
#pragma unroll
            for (int it = 0; it < ITERS; ++it)
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(h[it][i], h[it][i], sum);
            if (a.hh.q)
#pragma unroll
                for (int it = 0; it < ITERS; ++it) {
                    const int col = (it * threads + (int)threadIdx.x) * 8;
                    store_held<ALIGNED>(a.hh.q + t * a.ldq, a.hh.e + t * a.lde, col, C, h[it]);
                }
        }
        sum = cta_sum(sum, scratch[1]);
        const float r = rsqrtf(fmaf(sum, a.inv_C, a.eps));
        if (threadIdx.x == 0) a.rstd_pre[t] = r;
        T *no = (T *)a.n_out + t * a.ldn;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * threads + (int)threadIdx.x) * 8;
            float n[8], w[8];
            load_params(a.w_pre, col, C, w);
#pragma unroll
            for (int i = 0; i < 8; ++i) n[i] = h[it][i] * r * w[i];
            store_cols<T, ALIGNED>(no, col, C, n);
            if (a.hn.q) {
#pragma unroll
                for (int i = 0; i < 8; ++i) n[i] = to_float<T>(from_float<T>(n[i]));           // n as stored
                store_held<ALIGNED>(a.hn.q + t * a.ldq, a.hn.e + t * a.lde, col, C, n);
            }
        }
        if (!a.b) __syncthreads();   // one sum per row: scratch[1] is rewritten by the next
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
    int ring_e;                          // the stream kernel's ring brings rows of exponents: they are whole 16-byte words
    float res_scale, inv_C;
};

// Part p = (group, slice of the group's rows): one CTA walks the slice, the column sums stay in registers.
template <typename T, bool ALIGNED, int MOST, int ITERS>
__global__ void __launch_bounds__(MOST) norm_backward_kernel(const NormBackward a) {
    __shared__ float scratch[2][32];
    const int C = (int)a.C, threads = (int)blockDim.x;
    const int64_t group = blockIdx.x / a.parts_per_group, slice = blockIdx.x % a.parts_per_group;
    const int64_t first = group * a.rows_per_group + a.rows_per_group * slice / a.parts_per_group;
    const int64_t last = group * a.rows_per_group + a.rows_per_group * (slice + 1) / a.parts_per_group;
    const bool has_b = a.b || a.hb.q;
    float sum_x[ITERS][8], sum_y[ITERS][8];
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum_x[it][i] = sum_y[it][i] = 0.f;
    for (int64_t t = first; t < last; ++t) {
        // All loads of the row first: it waits for memory once.
        Frag<T, 8> fn[ITERS], fi[ITERS], fh[ITERS], fb[ITERS];
        RawQ qh[ITERS], qb[ITERS];
        uint32_t eh[ITERS], eb[ITERS];
        const float r = a.rstd_pre[t], rp = has_b ? a.rstd_post[t] : 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * threads + (int)threadIdx.x) * 8;
            if (col < C) {
                fn[it] = load_cols<T, ALIGNED>((const T *)a.dn + t * a.lddn, col, C);
                if (a.hh.q) {
                    qh[it] = load_q(a.hh.q + t * a.ldq + col);
                    eh[it] = a.hh.e[t * a.lde + col / kGroup];
                } else {
                    fh[it] = load_cols<T, ALIGNED>((const T *)a.h + t * a.ldh, col, C);
                }
                if (a.dh_in) fi[it] = load_cols<T, ALIGNED>((const T *)a.dh_in + t * a.lddhi, col, C);
                if (a.hb.q) {
                    qb[it] = load_q(a.hb.q + t * a.ldq + col);
                    eb[it] = a.hb.e[t * a.lde + col / kGroup];
                } else if (has_b) {
                    fb[it] = load_cols<T, ALIGNED>((const T *)a.b + t * a.ldb, col, C);
                }
            }
        }
        float D[ITERS][8], x[ITERS][8];
        float dot = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * threads + (int)threadIdx.x) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) D[it][i] = x[it][i] = 0.f;
            if (col < C) {
                float w[8];
                to_floats<T, 8>(fn[it], D[it]);
                if (a.hh.q) held_cols<ALIGNED>(qh[it], eh[it], col, C, x[it]);
                else to_floats<T, 8>(fh[it], x[it]);
                load_params(a.w_pre, col, C, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[it][i] *= r;
                    sum_x[it][i] = fmaf(D[it][i], x[it][i], sum_x[it][i]);
                    D[it][i] *= w[i];
                    dot = fmaf(D[it][i], x[it][i], dot);
                }
            }
        }
        dot = cta_sum(dot, scratch[0]) * a.inv_C;
        float dot_b = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * threads + (int)threadIdx.x) * 8;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
            if (a.dh_in && col < C) to_floats<T, 8>(fi[it], v);
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                D[it][i] = fmaf(r, fmaf(-x[it][i], dot, D[it][i]), v[i]);
                v[i] = a.res_scale * D[it][i];
            }
            store_cols<T, ALIGNED>((T *)a.dh + t * a.lddh, col, C, v);
            if (has_b && col < C) {
                float w[8];
                if (a.hb.q) held_cols<ALIGNED>(qb[it], eb[it], col, C, x[it]);
                else to_floats<T, 8>(fb[it], x[it]);
                load_params(a.w_post, col, C, w);
                if (a.gate) {
                    load_params(a.gate + group * a.C, col, C, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i) w[i] *= v[i];
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    x[it][i] *= rp;
                    sum_y[it][i] = fmaf(D[it][i], x[it][i], sum_y[it][i]);
                    D[it][i] *= w[i];
                    dot_b = fmaf(D[it][i], x[it][i], dot_b);
                }
            }
        }
        if (has_b) {
            dot_b = cta_sum(dot_b, scratch[1]) * a.inv_C;
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int col = (it * threads + (int)threadIdx.x) * 8;
                float out[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) out[i] = rp * fmaf(-x[it][i], dot_b, D[it][i]);
                store_cols<T, ALIGNED>((T *)a.db + t * a.lddb, col, C, out);
            }
        } else {
            __syncthreads();                         // scratch[0] is rewritten by the next row
        }
    }
    float *px = a.partial + (int64_t)blockIdx.x * 2 * a.C;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int col = (it * threads + (int)threadIdx.x) * 8;
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i < C) {
                px[col + i] = sum_x[it][i];
                if (has_b) px[C + col + i] = sum_y[it][i];
            }
    }
}

// ---------------------------------------------------------------------------
// Stream kernels: the same rows where there are many.  A CTA walks a slice of a group's rows; the next rows are on their way
// to shared memory by bulk copies while one is worked on, and the parameters stay there in fp32.  What bounds these
// kernels otherwise is the latency of a row: its loads, then two sums over the CTA that each wait for all of it.
// 16384 x 4096 bf16 in 8 groups: forward 94 us (537 MB), backward from 8-bit saves 144 with 12 for the parts' sums (676 MB);
// one row per CTA without copies ahead: 132 and 367.
//
// Rows that are not ALIGNED are copied with the 16-byte words around them, shifted into place when they are read, and
// written as store_run does.
// ---------------------------------------------------------------------------
constexpr int kMaxStages = 4;

template <typename T> __device__ __forceinline__ Frag<T, 8> shared_frag(const uint8_t *p) {
    Frag<T, 8> f;
    constexpr int kWords = sizeof(T) * 8 / 16;
    uint4 w[kWords];
#pragma unroll
    for (int i = 0; i < kWords; ++i) w[i] = reinterpret_cast<const uint4 *>(p)[i];
    memcpy(&f, w, sizeof(f));
    return f;
}
// Parameters in shared memory: of every 8 columns the first four in one half of the array, the last four in the other, so
// that a warp's accesses lie side by side.  C: columns rounded up to 8; those that do not exist are 0.
__device__ __forceinline__ int param_place(int i, int C) { return (i % 8 < 4 ? 0 : C / 2) + i / 8 * 4 + i % 4; }
__device__ __forceinline__ void shared_params(const float *p, int col, int C, float (&x)[8]) {
    const float4 a = *reinterpret_cast<const float4 *>(p + col / 2), b = *reinterpret_cast<const float4 *>(p + C / 2 + col / 2);
    x[0] = a.x; x[1] = a.y; x[2] = a.z; x[3] = a.w; x[4] = b.x; x[5] = b.y; x[6] = b.z; x[7] = b.w;
}

// A tensor's row in the ring.  ALIGNED: its bytes.  Else: the whole 16-byte words it touches -- but never a word that is
// partly outside the tensor, which only rows at its two ends can have; patch() brings their few elements.
template <typename T, bool ALIGNED> struct RowCopy {
    const T *p;
    int C;
    uintptr_t from, to;                  // the bytes that are copied
    __device__ RowCopy(const void *base, int64_t ld, int64_t t, int64_t rows, int columns) : p((const T *)base + t * ld), C(columns) {
        from = (uintptr_t)p;
        to = (uintptr_t)(p + C);
        if constexpr (!ALIGNED) {
            const uintptr_t begin = (uintptr_t)base, end = (uintptr_t)((const T *)base + (rows - 1) * ld + C);
            from &= ~(uintptr_t)15;
            to = (to + 15) & ~(uintptr_t)15;
            if (from < begin) from = (begin + 15) & ~(uintptr_t)15;
            if (to > end) to = end & ~(uintptr_t)15;
        }
    }
    __device__ uint32_t bytes() const { return ALIGNED ? C * (uint32_t)sizeof(T) : to > from ? (uint32_t)(to - from) : 0; }
    __device__ uint32_t offset() const { return ALIGNED ? 0 : (uint32_t)((uintptr_t)p & 15); }   // of the row in its slot
    __device__ void copy(uint32_t slot, uint32_t bar) const {
        if constexpr (ALIGNED) run_load(slot, p, bytes(), bar);
        else if (bytes()) run_load(slot + (uint32_t)(from - ((uintptr_t)p & ~(uintptr_t)15)), (const void *)from, bytes(), bar);
    }
    // The elements that copy() left out, fewer than 16 bytes at either end; by the first threads of the CTA.
    __device__ void patch(uint8_t *slot) const {
        const T *a = to > from ? (const T *)from : p + C, *b = to > from ? (const T *)to : p + C;
        const int head = a > p ? (int)(a - p) : 0, tail = p + C > b ? (int)(p + C - b) : 0;
        T *row = reinterpret_cast<T *>(slot + offset());
        for (int i = threadIdx.x; i < head + tail; i += blockDim.x) {
            const int col = i < head ? i : C - tail + (i - head);
            row[col] = p[col];
        }
        fence_async_shared();            // the slot's next copy comes after these stores
    }
};
// Where a row starts in its slot.
template <typename T, bool ALIGNED> __device__ __forceinline__ uint32_t row_offset(const void *base, int64_t ld, int64_t t) {
    return ALIGNED ? 0 : ((uint32_t)(uintptr_t)base + (uint32_t)t * (uint32_t)(ld * (int64_t)sizeof(T))) & 15u;
}
// Whether row t of tensors with these bases and strides in bytes may need patch(): only rows that lie within 16 bytes of
// an end of the tensor do.
__device__ __forceinline__ bool near_end(const void *a, int64_t a_stride, const void *b, int64_t b_stride, int64_t t, int64_t rows) {
    const int64_t least = t < rows - 1 - t ? t : rows - 1 - t;
    return (a && least * a_stride < 16) || (b && least * b_stride < 16);
}
// Bytes of a row's slot.
template <typename T, bool ALIGNED> __host__ __device__ __forceinline__ int slot_bytes(int C) {
    return ALIGNED ? C * (int)sizeof(T) : (C * (int)sizeof(T) + 31) / 32 * 32 + 16;
}
// Columns [col, col + 8) of a row that starts `off` bytes into its slot; 0 for columns from C on.
template <typename T, bool ALIGNED> __device__ __forceinline__ Frag<T, 8> slot_run(const uint8_t *slot, uint32_t off, int col, int C) {
    if constexpr (ALIGNED) {
        return shared_frag<T>(slot + col * sizeof(T));
    } else {
        constexpr int kWords = 2 * (int)sizeof(T);
        uint32_t w[kWords + 4], out[kWords];
        const uint4 *q = reinterpret_cast<const uint4 *>(slot + col * sizeof(T));
#pragma unroll
        for (int i = 0; i < kWords / 4 + 1; ++i) {
            const uint4 v = q[i];
            w[4 * i] = v.x; w[4 * i + 1] = v.y; w[4 * i + 2] = v.z; w[4 * i + 3] = v.w;
        }
        shift_words<kWords>(w, off, out);
        Frag<T, 8> f;
        memcpy(&f, out, sizeof(f));
        if (col + 8 > C) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i >= C) f.v[i] = from_float<T>(0.f);
        }
        return f;
    }
}
// What rows a slice holds.
struct Slice {
    int64_t group, first, last;
    __device__ Slice(int64_t rows_per_group, int64_t parts_per_group) {
        group = blockIdx.x / parts_per_group;
        const int64_t slice = blockIdx.x % parts_per_group, base = group * rows_per_group;
        first = base + rows_per_group * slice / parts_per_group;
        last = base + rows_per_group * (slice + 1) / parts_per_group;
    }
};

// MOST: the threads of the CTA (where rows are not ALIGNED: at most; as few as cover a row).  MINB: CTAs per SM that the
// registers are meant for.
template <typename T, bool ALIGNED, int MOST, int ITERS, int MINB>
__global__ void __launch_bounds__(MOST, MINB) norm_forward_stream_kernel(const NormForward a, const int stages) {
    extern __shared__ __align__(128) uint8_t dynamic[];
    __shared__ float scratch[2][32];
    __shared__ uint4 ends[2][ALIGNED ? 1 : ITERS * 32];
    __shared__ uint64_t full[kMaxStages];
    __shared__ int failed_flag;
    volatile int *failed = &failed_flag;
    const int threads = ALIGNED ? MOST : (int)blockDim.x, C = (int)a.C, Cp = ALIGNED ? C : (C + 7) & ~7, row_bytes = slot_bytes<T, ALIGNED>(C), stage_bytes = a.b ? 2 * row_bytes : row_bytes;
    float *w_pre = (float *)dynamic, *w_post = w_pre + Cp;           // w_post times the group's gate
    uint8_t *ring = dynamic + (a.b ? 8 : 4) * Cp;
    const Slice slice(a.rows_per_group, a.parts_per_group);
    auto fetch = [&](int64_t t, int s) {
        const uint32_t bar = smem_address(&full[s]), dst = smem_address(ring + s * stage_bytes);
        const RowCopy<T, ALIGNED> h(a.h, a.ldh, t, a.T, C), b(a.b, a.ldb, t, a.T, C);
        barrier_expect(bar, h.bytes() + (a.b ? b.bytes() : 0));
        h.copy(dst, bar);
        if (a.b) b.copy(dst + row_bytes, bar);
    };
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) barrier_init(smem_address(&full[s]), 1);
        failed_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int s = 0; s < stages && slice.first + s < slice.last; ++s) fetch(slice.first + s, s);
    }
    for (int i = threadIdx.x; i < Cp; i += threads) {
        const int at = param_place(i, Cp);
        w_pre[at] = ALIGNED || i < C ? a.w_pre[i] : 0.f;
        if (a.b) w_post[at] = !ALIGNED && i >= C ? 0.f : a.gate ? a.w_post[i] * a.gate[slice.group * C + i] : a.w_post[i];
    }
    __syncthreads();
    int s = 0;
    uint32_t parity = 0;
    for (int64_t t = slice.first; t < slice.last; ++t) {
        const bool ok = barrier_wait(smem_address(&full[s]), parity, failed);
        uint8_t *row = ring + s * stage_bytes;
        const uint32_t off_h = row_offset<T, ALIGNED>(a.h, a.ldh, t), off_b = row_offset<T, ALIGNED>(a.b, a.ldb, t);
        if (!ALIGNED && near_end(a.h, a.ldh * (int)sizeof(T), a.b, a.ldb * (int)sizeof(T), t, a.T)) {
            RowCopy<T, ALIGNED>(a.h, a.ldh, t, a.T, C).patch(row);
            if (a.b) RowCopy<T, ALIGNED>(a.b, a.ldb, t, a.T, C).patch(row + row_bytes);
            __syncthreads();
        }
        float h[ITERS][8], b[ITERS][8];
        float sum = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * threads + (int)threadIdx.x) * 8;
#pragma unroll
            for (int i = 0; i < 8; ++i) h[it][i] = b[it][i] = 0.f;
            if (col < C) {
                to_floats<T, 8>(slot_run<T, ALIGNED>(row, off_h, col, C), h[it]);
                if (a.b) to_floats<T, 8>(slot_run<T, ALIGNED>(row + row_bytes, off_b, col, C), b[it]);
            }
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float x = a.b ? b[it][i] : h[it][i];
                sum = fmaf(x, x, sum);
            }
        }
        sum = cta_sum<ALIGNED ? MOST : 0>(sum, scratch[0]);
        if (threadIdx.x == 0 && ok && t + stages < slice.last) fetch(t + stages, s);       // every thread has read the stage
        float r = rsqrtf(fmaf(sum, a.inv_C, a.eps));
        if (!ok) r = NAN;                                             // the wait ran out: no numbers rather than wrong ones
        if (a.b) {
            if (threadIdx.x == 0) a.rstd_post[t] = r;
            if (a.hb.q)
#pragma unroll
                for (int it = 0; it < ITERS; ++it) {
                    const int col = (it * threads + (int)threadIdx.x) * 8;
                    store_held<ALIGNED>(a.hb.q + t * a.ldq, a.hb.e + t * a.lde, col, C, b[it]);
                }
            sum = 0.f;
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int col = (it * threads + (int)threadIdx.x) * 8;
                if (col < C) {
                    float w[8];
                    shared_params(w_post, col, Cp, w);
#pragma unroll
                    for (int i = 0; i < 8; ++i) h[it][i] = fmaf(b[it][i] * r, w[i], a.res_scale * h[it][i]);
                    if constexpr (ALIGNED) store_floats<T, 8>((T *)a.h_out + t * a.ldho + col, h[it]);
                }
#pragma unroll
                for (int i = 0; i < 8; ++i) sum = fmaf(h[it][i], h[it][i], sum);
            }
            if constexpr (!ALIGNED) store_row<T, ITERS>((T *)a.h_out + t * a.ldho, threads, C, h, ends[0]);
            sum = cta_sum<ALIGNED ? MOST : 0>(sum, scratch[1]);
            r = rsqrtf(fmaf(sum, a.inv_C, a.eps));
        } else {
            __syncthreads();                                          // one sum per row: scratch[0] is rewritten by the next
        }
        if (threadIdx.x == 0) a.rstd_pre[t] = r;
        if (a.hh.q)
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
                const int col = (it * threads + (int)threadIdx.x) * 8;
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = to_float<T>(from_float<T>(h[it][i]));       // h' as stored
                store_held<ALIGNED>(a.hh.q + t * a.ldq, a.hh.e + t * a.lde, col, C, x);
            }
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = (it * threads + (int)threadIdx.x) * 8;
            if (col < C) {
                float w[8];
                shared_params(w_pre, col, Cp, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) h[it][i] = h[it][i] * r * w[i];
                if constexpr (ALIGNED) store_floats<T, 8>((T *)a.n_out + t * a.ldn + col, h[it]);
            }
            if (a.hn.q) {
                float x[8];
#pragma unroll
                for (int i = 0; i < 8; ++i) x[i] = to_float<T>(from_float<T>(h[it][i]));       // n as stored
                store_held<ALIGNED>(a.hn.q + t * a.ldq, a.hn.e + t * a.lde, col, C, x);
            }
        }
        if constexpr (!ALIGNED) store_row<T, ITERS>((T *)a.n_out + t * a.ldn, threads, C, h, ends[1]);
        if (++s == stages) {
            s = 0;
            parity ^= 1;
        }
    }
}

// Eight columns of a saved tensor as they lie in shared memory, and what they have to be multiplied by.
template <typename T, bool HELD> struct Saved;
template <typename T> struct Saved<T, false> {
    Frag<T, 8> f;
    float factor;
    __device__ __forceinline__ void values(float (&x)[8]) const {
        to_floats<T, 8>(f, x);
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] *= factor;
    }
};
template <typename T> struct Saved<T, true> {
    uint2 q;
    float factor;
    __device__ __forceinline__ void values(float (&x)[8]) const {
        const uint32_t w[2] = {q.x ^ 0x80808080u, q.y ^ 0x80808080u};
#pragma unroll
        for (int i = 0; i < 8; ++i) x[i] = (__uint_as_float(__byte_perm(w[i / 4], 0x4b400000u, 0x7650 + i % 4)) - 12583040.f) * factor;
    }
};
// Zeros in place of what a padded row holds past its last column.
template <bool NOTHING> __device__ __forceinline__ void clear_past(float (&x)[8], int col, int C) {
    if constexpr (!NOTHING) {
#pragma unroll
        for (int i = 0; i < 8; ++i)
            if (col + i >= C) x[i] = 0.f;
    }
}
// The backward pass is bound by instructions and registers as much as by bytes: addresses advance from row to row, the step
// of a checkpoint's group and the row's statistic, both factors, are multiplied first, and what the second half of a row
// needs stays in shared memory until then (two registers too many cost 20 us in spills that miss the L1; rows wider than 8192
// columns still spill).  HELD: h' and b are checkpoints (else both are values).
template <typename T, bool ALIGNED, int MOST, int ITERS, int MINB, bool HELD>
__global__ void __launch_bounds__(MOST, MINB) norm_backward_stream_kernel(const NormBackward a, const int stages) {
    extern __shared__ __align__(128) uint8_t dynamic[];
    __shared__ float scratch[2][32];
    __shared__ uint4 ends[2][ALIGNED ? 1 : ITERS * 32];
    __shared__ uint64_t full[kMaxStages];
    __shared__ int failed_flag;
    volatile int *failed = &failed_flag;
    const bool has_b = HELD ? a.hb.q != nullptr : a.b != nullptr;
    const bool ring_e = a.ring_e;                                    // else exponents are read one by one
    const int threads = ALIGNED ? MOST : (int)blockDim.x, C = (int)a.C, Cp = ALIGNED ? C : (C + 7) & ~7, row_bytes = slot_bytes<T, ALIGNED>(C), e_bytes = ring_e ? (int)a.lde : 0, held_bytes = (int)a.ldq + e_bytes;
    const int saved_bytes = HELD ? held_bytes : row_bytes;
    const int at_in = row_bytes, at_h = at_in + (a.dh_in ? row_bytes : 0), at_b = at_h + saved_bytes, stage_bytes = at_b + (has_b ? saved_bytes : 0);
    float *w_pre = (float *)dynamic, *w_post = w_pre + Cp;           // w_post times the group's gate
    uint8_t *ring = dynamic + (has_b ? 8 : 4) * Cp;
    const Slice slice(a.rows_per_group, a.parts_per_group);
    using Copy = RowCopy<T, ALIGNED>;
    auto saved_bytes_of = [&](const Copy &values) { return HELD ? (uint32_t)held_bytes : values.bytes(); };
    auto fetch_saved = [&](uint32_t dst, const Copy &values, const HeldIn &held, int64_t t, uint32_t bar) {
        if constexpr (HELD) {
            run_load(dst, held.q + t * a.ldq, (uint32_t)a.ldq, bar);
            if (ring_e) run_load(dst + (uint32_t)a.ldq, held.e + t * a.lde, e_bytes, bar);
        } else {
            values.copy(dst, bar);
        }
    };
    auto fetch = [&](int64_t t, int s) {
        const uint32_t bar = smem_address(&full[s]), dst = smem_address(ring + s * stage_bytes);
        const Copy n(a.dn, a.lddn, t, a.T, C), in(a.dh_in, a.lddhi, t, a.T, C), h(a.h, a.ldh, t, a.T, C), b(a.b, a.ldb, t, a.T, C);
        barrier_expect(bar, n.bytes() + (a.dh_in ? in.bytes() : 0) + saved_bytes_of(h) + (has_b ? saved_bytes_of(b) : 0));
        n.copy(dst, bar);
        if (a.dh_in) in.copy(dst + at_in, bar);
        fetch_saved(dst + at_h, h, a.hh, t, bar);
        if (has_b) fetch_saved(dst + at_b, b, a.hb, t, bar);
    };
    if (threadIdx.x == 0) {
        for (int s = 0; s < stages; ++s) barrier_init(smem_address(&full[s]), 1);
        failed_flag = 0;
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        for (int s = 0; s < stages && slice.first + s < slice.last; ++s) fetch(slice.first + s, s);
    }
    for (int i = threadIdx.x; i < Cp; i += threads) {
        const int at = param_place(i, Cp);
        w_pre[at] = ALIGNED || i < C ? a.w_pre[i] : 0.f;
        if (has_b) w_post[at] = !ALIGNED && i >= C ? 0.f : a.gate ? a.w_post[i] * a.gate[slice.group * C + i] : a.w_post[i];
    }
    __syncthreads();
    float sum_x[ITERS][8], sum_y[ITERS][8];
#pragma unroll
    for (int it = 0; it < ITERS; ++it)
#pragma unroll
        for (int i = 0; i < 8; ++i) sum_x[it][i] = sum_y[it][i] = 0.f;
    // The statistics of a row are fetched while the one before it is worked on.
    const float *stat = a.rstd_pre + slice.first, *stat_b = has_b ? a.rstd_post + slice.first : stat;
    float next_r = 0.f, next_rp = 0.f;
    if (slice.first < slice.last) {
        next_r = *stat;
        next_rp = *stat_b;
    }
    const int col0 = (int)threadIdx.x * 8;
    T *out_h = (T *)a.dh + slice.first * a.lddh, *out_b = (T *)a.db + (has_b ? slice.first * a.lddb : 0);
    int s = 0;
    uint32_t parity = 0;
    for (int64_t t = slice.first; t < slice.last; ++t) {
        const bool ok = barrier_wait(smem_address(&full[s]), parity, failed);
        uint8_t *row = ring + s * stage_bytes;
        const uint32_t off_n = row_offset<T, ALIGNED>(a.dn, a.lddn, t), off_in = row_offset<T, ALIGNED>(a.dh_in, a.lddhi, t),
                       off_h = row_offset<T, ALIGNED>(a.h, a.ldh, t), off_b = row_offset<T, ALIGNED>(a.b, a.ldb, t);
        if (!ALIGNED && (near_end(a.dn, a.lddn * (int)sizeof(T), a.dh_in, a.lddhi * (int)sizeof(T), t, a.T) ||
                         near_end(a.h, a.ldh * (int)sizeof(T), a.b, a.ldb * (int)sizeof(T), t, a.T))) {
            Copy(a.dn, a.lddn, t, a.T, C).patch(row);
            if (a.dh_in) Copy(a.dh_in, a.lddhi, t, a.T, C).patch(row + at_in);
            if (!HELD) Copy(a.h, a.ldh, t, a.T, C).patch(row + at_h);
            if (!HELD && has_b) Copy(a.b, a.ldb, t, a.T, C).patch(row + at_b);
            __syncthreads();
        }
        const float r = ok ? next_r : NAN, rp = next_rp;
        auto saved = [&](int place, uint32_t off, const HeldIn &held, int col, float factor) {
            Saved<T, HELD> v;
            if constexpr (HELD) {
                v.q = *reinterpret_cast<const uint2 *>(row + place + col);
                factor *= group_scale(ring_e ? row[place + (int)a.ldq + col / kGroup] : held.e[t * a.lde + col / kGroup]);
            } else {
                v.f = slot_run<T, ALIGNED>(row + place, off, col, C);
            }
            v.factor = factor;
            return v;
        };
        float D[ITERS][8], x[ITERS][8];
        float dot = 0.f;
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = it * threads * 8 + col0;
            if (col < C) {
                float w[8];
                to_floats<T, 8>(slot_run<T, ALIGNED>(row, off_n, col, C), D[it]);
                saved(at_h, off_h, a.hh, col, r).values(x[it]);
                clear_past<ALIGNED || !HELD>(x[it], col, C);
                shared_params(w_pre, col, Cp, w);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum_x[it][i] = fmaf(D[it][i], x[it][i], sum_x[it][i]);
                    D[it][i] *= w[i];
                    dot = fmaf(D[it][i], x[it][i], dot);
                }
            }
        }
        if (t + 1 < slice.last) {
            next_r = *++stat;
            next_rp = *++stat_b;
        }
        const float minus_dot = -cta_sum<ALIGNED ? MOST : 0>(dot, scratch[0]) * a.inv_C;
        dot = 0.f;
        float first_half[ALIGNED ? 1 : ITERS][8];                     // dh, to be stored by the CTA together
#pragma unroll
        for (int it = 0; it < ITERS; ++it) {
            const int col = it * threads * 8 + col0;
            float v[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) v[i] = 0.f;
            if (col < C) {
                if (a.dh_in) to_floats<T, 8>(slot_run<T, ALIGNED>(row + at_in, off_in, col, C), v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    D[it][i] = fmaf(r, fmaf(x[it][i], minus_dot, D[it][i]), v[i]);
                    v[i] = a.res_scale * D[it][i];
                }
                if (ALIGNED) store_floats<T, 8>(out_h + col, v);
            }
            if constexpr (!ALIGNED) {
#pragma unroll
                for (int i = 0; i < 8; ++i) first_half[it][i] = v[i];
            }
            if (has_b && col < C) {
                saved(at_b, off_b, a.hb, col, rp).values(x[it]);
                clear_past<ALIGNED || !HELD>(x[it], col, C);
                shared_params(w_post, col, Cp, v);
#pragma unroll
                for (int i = 0; i < 8; ++i) {
                    sum_y[it][i] = fmaf(D[it][i], x[it][i], sum_y[it][i]);
                    D[it][i] *= v[i];
                    dot = fmaf(D[it][i], x[it][i], dot);
                }
            }
        }
        if constexpr (!ALIGNED) store_row<T, ITERS>(out_h, threads, C, first_half, ends[0]);
        out_h += a.lddh;
        if (has_b) {
            const float minus_dot_b = -cta_sum<ALIGNED ? MOST : 0>(dot, scratch[1]) * a.inv_C;
            if (threadIdx.x == 0 && ok && t + stages < slice.last) fetch(t + stages, s);   // every thread has read the stage
#pragma unroll
            for (int it = 0; it < ITERS; ++it) {
#pragma unroll
                for (int i = 0; i < 8; ++i) D[it][i] = rp * fmaf(x[it][i], minus_dot_b, D[it][i]);
                if (ALIGNED && it * threads * 8 + col0 < C) store_floats<T, 8>(out_b + it * threads * 8 + col0, D[it]);
            }
            if constexpr (!ALIGNED) store_row<T, ITERS>(out_b, threads, C, D, ends[1]);
            out_b += a.lddb;
        } else {
            __syncthreads();                                          // one sum per row: scratch[0] is rewritten by the next
            if (threadIdx.x == 0 && ok && t + stages < slice.last) fetch(t + stages, s);
        }
        if (++s == stages) {
            s = 0;
            parity ^= 1;
        }
    }
    float *px = a.partial + (int64_t)blockIdx.x * 2 * C;
#pragma unroll
    for (int it = 0; it < ITERS; ++it) {
        const int col = it * threads * 8 + col0;
        if (ALIGNED && col < C) {
#pragma unroll
            for (int i = 0; i < 8; i += 4) {
                *reinterpret_cast<float4 *>(px + col + i) = make_float4(sum_x[it][i], sum_x[it][i + 1], sum_x[it][i + 2], sum_x[it][i + 3]);
                if (has_b) *reinterpret_cast<float4 *>(px + C + col + i) = make_float4(sum_y[it][i], sum_y[it][i + 1], sum_y[it][i + 2], sum_y[it][i + 3]);
            }
        } else if (!ALIGNED) {
#pragma unroll
            for (int i = 0; i < 8; ++i)
                if (col + i < C) {
                    px[col + i] = sum_x[it][i];
                    if (has_b) px[C + col + i] = sum_y[it][i];
                }
        }
    }
}

// The parts' sums, in a fixed order: CTA (32 columns, job) adds them with 32 threads per V columns.  Job g < jobs_gate: dgate
// of group g, w_post times the sum of D y over the group's parts.  Then dw_pre, the sum of dn x over all parts, and
// dw_post, the sum of gate times D y.
template <int V>
__global__ void __launch_bounds__(1024 / V) norm_reduce_kernel(const float *__restrict__ partial, const float *__restrict__ w_post,
                                                               const float *__restrict__ gate, int C, int64_t groups,
                                                               int64_t parts_per_group, int64_t jobs_gate, int accumulate,
                                                               float *dw_post, float *dgate, float *dw_pre) {
    __shared__ float tile[32][33];
    asm volatile("griddepcontrol.wait;" ::: "memory");               // the partial sums are those of the kernel before
    const int col = (int)(blockIdx.x * 32 + threadIdx.x * V);
    const bool live = col < C;                                       // V columns at a time: C is a multiple of V
    for (int64_t job = blockIdx.y; job < jobs_gate + (dw_post ? 2 : 1); job += gridDim.y) {
        const int64_t first = job < jobs_gate ? job * parts_per_group : 0, count = (job < jobs_gate ? 1 : groups) * parts_per_group;
        const bool of_y = job != jobs_gate, gated = job == jobs_gate + 1 && gate;
        float s[V];
#pragma unroll
        for (int i = 0; i < V; ++i) s[i] = 0.f;
        if (live)
#pragma unroll 4
            for (int64_t p = threadIdx.y; p < count; p += 32) {
                struct alignas(V * 4) Run { float v[V]; };
                const Run v = *reinterpret_cast<const Run *>(partial + ((first + p) * 2 + of_y) * C + col);
                const float *g = gate + (int64_t)(gated ? (uint32_t)p / (uint32_t)parts_per_group : 0) * C + col;
#pragma unroll
                for (int i = 0; i < V; ++i) s[i] = gated ? fmaf(g[i], v.v[i], s[i]) : s[i] + v.v[i];
            }
#pragma unroll
        for (int i = 0; i < V; ++i) tile[threadIdx.y][threadIdx.x * V + i] = s[i];
        __syncthreads();
        const int c = (int)(threadIdx.y * blockDim.x + threadIdx.x), column = (int)blockIdx.x * 32 + c;
        if (c < 32 && column < C) {
            float total = 0.f;
#pragma unroll
            for (int i = 0; i < 32; ++i) total += tile[i][c];
            float *out = job < jobs_gate ? dgate + job * C + column : of_y ? dw_post + column : dw_pre + column;
            if (job < jobs_gate) total *= w_post[column];
            *out = accumulate ? *out + total : total;
        }
        __syncthreads();
    }
}

}  // namespace deft
