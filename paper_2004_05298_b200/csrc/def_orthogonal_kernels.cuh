// Orthogonalising an update by Newton-Schulz products (see include/def_train.h):
//
//     X = x / (|x|_F + eps),   then for each (a, b, c):   A = X X^T,   B = a I + b A + c A A,   X <- B X
//
// with X wide (m <= n; a tall x is taken transposed).  Everything between the steps is held as two fp16 pieces, the value
// rounded and what that leaves, which carry 22 bits; each product is the three products of pieces above 2^-22.  Singular values
// stay below 4 where the polynomial is one that converges, so no entry of X or A is larger than 16 and a power of two
// that puts 16 at the end of fp16's range serves all of them (kPieceScale).  A and A A are symmetric: tiles on and below
// the diagonal are computed, those below stored twice.  Five steps of 4096 x 10240 fp32 take 7.8 to 8.1 ms, 1.1 PFLOP/s of fp16
// products (calls back to back, one set of inputs; 8.3 ms with three in turn; chains emptied every 4 stages); of 256 x 256 187 us, 15
// products one after another.
#pragma once

#include "def_product_kernels.cuh"

namespace deft {

constexpr float kPieceScale = 4096.f;
constexpr int kNormParts64 = 512;                  // most partial sums of squares of a matrix
constexpr int kPackTile = 64;

struct Matrices {
    const void *x;
    int64_t ld, stride;                            // of rows; of matrices
    int64_t rows, cols, batch;
};

// Partial sums of squares in 64 bits: no fp32 value over- or underflows there.  Grid: parts, matrices.
template <typename T> __global__ void __launch_bounds__(256) square_sum_kernel(const Matrices a, double *__restrict__ sums) {
    __shared__ double scratch[8];
    for (int64_t b = blockIdx.y; b < a.batch; b += gridDim.y) {
        const T *x = (const T *)a.x + b * a.stride;
        double sum = 0;
        for (int64_t r = (int64_t)blockIdx.x * 8 + threadIdx.x / 32; r < a.rows; r += (int64_t)gridDim.x * 8) {
            const T *row = x + r * a.ld;
            for (int64_t c0 = 0; c0 < a.cols; c0 += 8 * 32) {
                const int64_t c = c0 + threadIdx.x % 32 * 8;
                if (c < a.cols) {
                    const Frag<T, 8> f = load_run<T>(row, (int)c, (int)a.cols);
#pragma unroll
                    for (int i = 0; i < 8; ++i) {
                        const double v = to_float<T>(f.v[i]);
                        sum = fma(v, v, sum);
                    }
                }
            }
        }
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
        if (threadIdx.x % 32 == 0) scratch[threadIdx.x / 32] = sum;
        __syncthreads();
        if (threadIdx.x == 0) {
            for (int w = 1; w < 8; ++w) sum += scratch[w];
            sums[b * gridDim.x + blockIdx.x] = sum;
        }
        __syncthreads();
    }
}

__device__ __forceinline__ void split_half(float v, __half &hi, __half &lo) {
    hi = __float2half_rn(v);
    lo = __float2half_rn(v - __half2float(hi));
}

// Pieces of X, scaled.  Grid: tiles of kPackTile columns and rows of x, matrices.  TALL: X is x transposed.
template <typename T, bool TALL>
__global__ void __launch_bounds__(256) pack_pieces_kernel(const Matrices a, const double *__restrict__ sums, int parts, float eps, __half *__restrict__ out,
                                                          int64_t ldo, int64_t plane) {
    __shared__ float tile[TALL ? kPackTile : 1][kPackTile + 1];
    const int64_t r0 = (int64_t)blockIdx.y * kPackTile, c0 = (int64_t)blockIdx.x * kPackTile;
    const int tx = threadIdx.x % 8, ty = threadIdx.x / 8;                    // 8 runs of 8 columns, 32 rows
    for (int64_t b = blockIdx.z; b < a.batch; b += gridDim.z) {
        double sum = 0;                            // every warp for itself, in one order
        for (int i = threadIdx.x % 32; i < parts; i += 32) sum += sums[b * parts + i];
#pragma unroll
        for (int s = 16; s > 0; s >>= 1) sum += __shfl_xor_sync(0xffffffffu, sum, s);
        // a NaN or an infinity anywhere: no number is right
        const double scale = !(sum <= 1e300) ? (double)NAN : sum > 0 ? kPieceScale / (sqrt(sum) + (double)eps) : 0.;
        const T *x = (const T *)a.x + b * a.stride;
        __half *o = out + b * 2 * plane;
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int64_t r = r0 + ty + 32 * h, c = c0 + tx * 8;
            float v[8] = {};
            if (r < a.rows && c < a.cols) {
                const Frag<T, 8> f = load_run<T>(x + r * a.ld, (int)c, (int)a.cols);
#pragma unroll
                for (int i = 0; i < 8; ++i) v[i] = c + i < a.cols ? (float)(to_float<T>(f.v[i]) * scale) : 0.f;
            }
            if constexpr (TALL) {
#pragma unroll
                for (int i = 0; i < 8; ++i) tile[tx * 8 + i][ty + 32 * h] = v[i];
            } else if (r < a.rows && c < ldo) {
                Frag<__half, 8> hi, lo;
#pragma unroll
                for (int i = 0; i < 8; ++i) split_half(v[i], hi.v[i], lo.v[i]);
                *reinterpret_cast<Frag<__half, 8> *>(o + r * ldo + c) = hi;
                *reinterpret_cast<Frag<__half, 8> *>(o + plane + r * ldo + c) = lo;
            }
        }
        if constexpr (TALL) {
            __syncthreads();
#pragma unroll
            for (int h = 0; h < 2; ++h) {
                const int64_t r = c0 + ty + 32 * h, c = r0 + tx * 8;         // of X
                if (r < a.cols && c < ldo) {
                    Frag<__half, 8> hi, lo;
#pragma unroll
                    for (int i = 0; i < 8; ++i) split_half(tile[ty + 32 * h][tx * 8 + i], hi.v[i], lo.v[i]);
                    *reinterpret_cast<Frag<__half, 8> *>(o + r * ldo + c) = hi;
                    *reinterpret_cast<Frag<__half, 8> *>(o + plane + r * ldo + c) = lo;
                }
            }
            __syncthreads();
        }
    }
}

// 32 columns of a row as pieces, in whole words: rows are padded to 32 elements.
__device__ __forceinline__ void store_pieces(__half *p, int64_t ld, int64_t plane, bool there, const float (&v)[32], uint8_t *turn) {
#pragma unroll 1
    for (int k = 0; k < 2; ++k) {
#pragma unroll
        for (int f = 0; f < 32; f += 8) {
            float part[8];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float hi = __half2float(__float2half_rn(v[f + i]));
                part[i] = k ? v[f + i] - hi : hi;
            }
            turn_put_8<64, __half>(turn, f, part);
        }
        turn_store_words<64>(turn, p + k * plane, ld * 2, there);
    }
}

// out <- alpha D + beta add + diagonal I in pieces, D symmetric, tiles on and below the diagonal.
struct StoreSymmetric {
    static constexpr bool kBoth = false;
    __half *out;
    const __half *add;                             // NULL: none
    int64_t ld, plane, m;                          // plane: elements of a piece
    float alpha, beta, diagonal;
    __device__ __forceinline__ void store(float (&v)[32], float (&)[32], int batch, int64_t row, int64_t col, uint8_t *turn) const {
        if (col >= m) return;
        const bool there = row < m;
        const int64_t at = (int64_t)batch * 2 * plane + row * ld + col;
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= alpha;
        if (add) {
            Frag<__half, 8> x[8];                                  // all on their way at once
#pragma unroll
            for (int k = 0; k < 8; ++k) x[k] = there ? load_frag<__half, 8>(add + at + k / 4 * plane + k % 4 * 8) : zeros<__half, 8>();
#pragma unroll
            for (int k = 0; k < 8; ++k)
#pragma unroll
                for (int i = 0; i < 8; ++i) v[k % 4 * 8 + i] = fmaf(beta, to_float<__half>(x[k].v[i]), v[k % 4 * 8 + i]);
            const int at_diagonal = row - col >= 0 && row - col < 32 ? (int)(row - col) : -1;
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i == at_diagonal) v[i] += diagonal;
        }
        store_pieces(out + at, ld, plane, there, v, turn);
        if (row / (2 * kTileRows) != col / kTileCols && there) {             // the other side of the diagonal
            __half *o = out + (int64_t)batch * 2 * plane + col * ld + row, *stop = o + (m - col < 32 ? m - col : 32) * ld;
#pragma unroll
            for (int i = 0; i < 32; ++i, o += ld) {
                __half hi, lo;
                split_half(v[i], hi, lo);
                if (o < stop) {
                    o[0] = hi;
                    o[plane] = lo;
                }
            }
        }
    }
};

// out <- alpha D in pieces.
struct StorePieces {
    static constexpr bool kBoth = false;
    __half *out;
    int64_t ld, plane, m, n;
    float alpha;
    __device__ __forceinline__ void store(float (&v)[32], float (&)[32], int batch, int64_t row, int64_t col, uint8_t *turn) const {
        if (col >= n) return;
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= alpha;
        store_pieces(out + (int64_t)batch * 2 * plane + row * ld + col, ld, plane, row < m, v, turn);
    }
};

// out <- alpha D, or its transpose.
template <typename T> struct StoreUpdate {
    static constexpr bool kBoth = false;
    T *out;
    int64_t ld, stride, m, n;
    float alpha;
    int tall, wide;
    __device__ __forceinline__ void store(float (&v)[32], float (&)[32], int batch, int64_t row, int64_t col, uint8_t *turn) const {
        if (col >= n) return;
        const int left = n - col < 32 ? (int)(n - col) : 32;
        T *o = out + batch * stride;
#pragma unroll
        for (int i = 0; i < 32; ++i) v[i] *= alpha;
        if (!tall) {
            store_32<T>(o + row * ld + col, ld, row < m, left, wide, v, turn);
        } else if (row < m) {
#pragma unroll
            for (int i = 0; i < 32; ++i)
                if (i < left) o[(col + i) * ld + row] = from_float<T>(v[i]);
        }
    }
};

}  // namespace deft
