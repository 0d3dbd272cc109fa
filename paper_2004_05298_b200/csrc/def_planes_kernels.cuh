// 16-bit pieces of rows, for products on tensor cores.
#pragma once

#include "def_train_common.cuh"

namespace deft {

// Rows as the tensor cores take them, where they do not lie like that already: 16-bit pieces in rows of ld elements (a multiple
// of 8, the last ones 0).  16-bit types: a copy, of either type as bits.  fp32: three bf16 numbers of 8 bits each, by truncation,
// whose sum is the value exactly.  A thread takes 8 columns; blockIdx.z is the matrix.
constexpr int kMostPlanes = 4;
struct Planes {
    struct Matrix {
        const void *x;
        uint4 *out;
        int64_t ldx, rows, ld;
        int cols;
    } of[kMostPlanes];
};
template <typename T> __global__ void __launch_bounds__(256) planes_kernel(const __grid_constant__ Planes p) {
    const Planes::Matrix &m = p.of[blockIdx.z];
    const T *x = (const T *)m.x;
    uint4 *out = m.out;
    const int64_t ldx = m.ldx, rows = m.rows, ld = m.ld;
    const int cols = m.cols, col = (int)(blockIdx.x * blockDim.x + threadIdx.x) * 8;
    if (col >= cols) return;
    for (int64_t t = (int64_t)blockIdx.y * blockDim.y + threadIdx.y; t < rows; t += (int64_t)gridDim.y * blockDim.y) {
        const Frag<T, 8> f = load_run<T>(x + t * ldx, col, cols);
        if constexpr (sizeof(T) == 2) {
            uint4 w;
            memcpy(&w, &f, sizeof(w));
            out[(t * ld + col) / 8] = w;
        } else {
            Frag<__nv_bfloat16, 8> piece[3];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const float v = f.v[i];
                const bool finite = fabsf(v) <= 3.402823466e38f;
                const float hi = __uint_as_float(__float_as_uint(v) & 0xffff0000u), rest = v - hi;
                const float mid = __uint_as_float(__float_as_uint(rest) & 0xffff0000u);
                piece[0].v[i] = from_float<__nv_bfloat16>(finite ? hi : v);
                piece[1].v[i] = from_float<__nv_bfloat16>(finite ? mid : 0.f);
                piece[2].v[i] = from_float<__nv_bfloat16>(finite ? rest - mid : 0.f);
            }
#pragma unroll
            for (int k = 0; k < 3; ++k) {
                uint4 w;
                memcpy(&w, &piece[k], sizeof(w));
                out[((k * rows + t) * ld + col) / 8] = w;
            }
        }
    }
}

}  // namespace deft
