// Weight gradient of a linear layer from the 8-bit checkpoint of its input (see include/def_train.h).
#pragma once

#include "def_train_common.cuh"

namespace deft {

// dw[o, i] (+)= sum_t dy[t, o] x^[t, i].  CTA: 64 x 64 of dw, 16 tokens at a time through shared memory.
template <typename T>
__global__ void __launch_bounds__(256) weight_grad_simple_kernel(const T *__restrict__ dy, int64_t lddy, const int8_t *__restrict__ q,
                                                                 const uint8_t *__restrict__ e, int64_t ldq, int64_t lde, int64_t tokens,
                                                                 int64_t O, int64_t I, float *dw, int accumulate) {
    __shared__ float sy[16][64], sx[16][64];
    const int64_t o0 = (int64_t)blockIdx.y * 64, i0 = (int64_t)blockIdx.x * 64;
    const int tx = threadIdx.x % 16, ty = threadIdx.x / 16;
    float acc[4][4] = {};
    for (int64_t t0 = 0; t0 < tokens; t0 += 16) {
        for (int k = threadIdx.x; k < 1024; k += 256) {
            const int64_t t = t0 + k / 64, o = o0 + k % 64, i = i0 + k % 64;
            sy[k / 64][k % 64] = t < tokens && o < O ? to_float<T>(dy[t * lddy + o]) : 0.f;
            float x = 0.f;
            if (t < tokens && i < I) x = to_float<T>(from_float<T>((float)q[t * ldq + i] * group_scale(e[t * lde + i / kGroup])));
            sx[k / 64][k % 64] = x;
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < 16; ++k)
#pragma unroll
            for (int a = 0; a < 4; ++a)
#pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(sy[k][ty * 4 + a], sx[k][tx + 16 * b], acc[a][b]);
        __syncthreads();
    }
    for (int a = 0; a < 4; ++a)
        for (int b = 0; b < 4; ++b) {
            const int64_t o = o0 + ty * 4 + a, i = i0 + tx + 16 * b;
            if (o < O && i < I) dw[o * I + i] = accumulate ? dw[o * I + i] + acc[a][b] : acc[a][b];
        }
}

}  // namespace deft
