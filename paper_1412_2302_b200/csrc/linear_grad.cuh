// Weight gradient of a linear layer whose input was kept as an 8-bit checkpoint: dw[o][i] = sum_r dy[r][o] x[r][i].
#pragma once
#include "checkpoint.cuh"

namespace op {

// 64 x 64 outputs per block, 16 rows at a time
template <int FMT>
__global__ void __launch_bounds__(256) linear_grad_simple_kernel(const __nv_bfloat16* __restrict__ dy, long long ld_dy, const uint8_t* __restrict__ codes, const uint8_t* __restrict__ scales,
                                                                 long long rows, int n_in, int n_out, float* __restrict__ dw) {
    kn::pdl_sync();
    __shared__ float sd[16][64], sx[16][64];
    const int tx = threadIdx.x & 15, ty = threadIdx.x >> 4;
    const int i0 = blockIdx.x * 64, o0 = blockIdx.y * 64, blocks = (n_in + 31) / 32;
    float acc[4][4] = {};
    for (long long r0 = 0; r0 < rows; r0 += 16) {
        for (int t = threadIdx.x; t < 16 * 64; t += 256) {
            const int k = t >> 6, c = t & 63;
            const long long r = r0 + k;
            sd[k][c] = r < rows && o0 + c < n_out ? __bfloat162float(dy[r * ld_dy + o0 + c]) : 0.f;
            float f = 0.f;
            if (r < rows && i0 + c < n_in) {
                code_values<FMT, 1>(codes[r * n_in + i0 + c], &f);
                f *= scale_of(scales[r * blocks + (i0 + c) / 32]);
            }
            sx[k][c] = f;
        }
        __syncthreads();
        #pragma unroll
        for (int k = 0; k < 16; ++k)
            #pragma unroll
            for (int a = 0; a < 4; ++a)
                #pragma unroll
                for (int b = 0; b < 4; ++b) acc[a][b] = fmaf(sd[k][ty + 16 * a], sx[k][tx + 16 * b], acc[a][b]);
        __syncthreads();
    }
    #pragma unroll
    for (int a = 0; a < 4; ++a)
        #pragma unroll
        for (int b = 0; b < 4; ++b) {
            const int o = o0 + ty + 16 * a, i = i0 + tx + 16 * b;
            if (o < n_out && i < n_in) dw[(long long)o * n_in + i] = acc[a][b];
        }
}

}  // namespace op
