// The sum of partial rows that many blocks left, in a fixed order: weight gradients of the norms.
#pragma once
#include "common.h"

namespace relibra {

// dw (+)= the sum of P partial rows: 32 columns a block, 128 strips of rows, joined in ascending order.
constexpr int kReduceStrips = 128;
static __global__ void __launch_bounds__(kReduceStrips * 8)
row_reduce_kernel(const float *__restrict__ part0, const float *__restrict__ part1, float *__restrict__ dw0, float *__restrict__ dw1, int P, int h, int add)
{
    __shared__ float4 join[kReduceStrips][8];
    const float *part = blockIdx.y ? part1 : part0;
    float *dw = blockIdx.y ? dw1 : dw0;
    if (!dw) return;
    const int col = threadIdx.x & 7, strip = threadIdx.x >> 3, at = blockIdx.x * 32 + col * 4;
    float4 s = make_float4(0.f, 0.f, 0.f, 0.f);
    if (at < h)
#pragma unroll 4
        for (int p = strip; p < P; p += kReduceStrips) {
            const float4 v = *reinterpret_cast<const float4 *>(part + (size_t)p * h + at);
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
    join[strip][col] = s;
    __syncthreads();
    // 128 strips to 8, then one thread a column the rest
    if (strip < 8) {
        for (int i = strip + 8; i < kReduceStrips; i += 8) {
            const float4 v = join[i][col];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        join[strip][col] = s;
    }
    __syncthreads();
    if (strip == 0 && at < h) {
        for (int i = 1; i < 8; ++i) {
            const float4 v = join[i][col];
            s.x += v.x; s.y += v.y; s.z += v.z; s.w += v.w;
        }
        float4 *to = reinterpret_cast<float4 *>(dw + at);
        if (add) {
            const float4 o = *to;
            s.x += o.x; s.y += o.y; s.z += o.z; s.w += o.w;
        }
        *to = s;
    }
}

}  // namespace relibra
