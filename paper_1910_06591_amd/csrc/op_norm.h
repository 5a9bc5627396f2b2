// Group normalisation with an activation, channels last:
//   y = act((x - mean) / sqrt(var + eps) * weight + bias),
// mean and variance over all points of a row and the channels of a group.
#pragma once
#include "op_common.h"

namespace seedinf {

struct NormArgs {
    const void* x; void* y;
    const float* weight; const float* bias;      // [channels] or nullptr
    int N, P, C, G;
    float eps;
};

__device__ __forceinline__ float norm_block_sum(float v, float* scratch)
{
#pragma unroll
    for (int off = 32; off > 0; off >>= 1) v += __shfl_xor(v, off, 64);
    __syncthreads();                             // the previous sum's readers are done
    if ((threadIdx.x & 63) == 0) scratch[threadIdx.x >> 6] = v;
    __syncthreads();
    return (scratch[0] + scratch[1]) + (scratch[2] + scratch[3]);
}

// One workgroup per row and group, three passes: mean, sum of squared differences, result.
template <class T, int ACT>
__global__ __launch_bounds__(256) void group_norm_kernel(NormArgs p)
{
    __shared__ float scratch[4];
    const int cg = p.C / p.G, g = blockIdx.x % p.G;
    const size_t n = blockIdx.x / p.G, base = n * (size_t)p.P * p.C + (size_t)g * cg;
    const size_t count = (size_t)p.P * cg;
    const T* x = (const T*)p.x + base;
    T* y = (T*)p.y + base;
    float s = 0.0f;
    for (size_t i = threadIdx.x; i < count; i += 256) s += (float)x[i / cg * p.C + i % cg];
    const float mean = norm_block_sum(s, scratch) / (float)count;
    float m2 = 0.0f;
    for (size_t i = threadIdx.x; i < count; i += 256) {
        const float d = (float)x[i / cg * p.C + i % cg] - mean;
        m2 = fmaf(d, d, m2);
    }
    const float rstd = 1.0f / sqrtf(norm_block_sum(m2, scratch) / (float)count + p.eps);
    for (size_t i = threadIdx.x; i < count; i += 256) {
        const int c = (int)(i % cg);
        float v = ((float)x[i / cg * p.C + c] - mean) * rstd;
        if (p.weight) v *= p.weight[g * cg + c];
        if (p.bias) v += p.bias[g * cg + c];
        y[i / cg * p.C + c] = (T)op_activate<ACT>(v);
    }
}

template <class T>
static void norm_launch(const NormArgs& p, int act, hipStream_t s)
{
    const dim3 grid((unsigned)((size_t)p.N * p.G));
    if (act == SEED_ACT_NONE) hipLaunchKernelGGL((group_norm_kernel<T, SEED_ACT_NONE>), grid, dim3(256), 0, s, p);
    else if (act == SEED_ACT_RELU) hipLaunchKernelGGL((group_norm_kernel<T, SEED_ACT_RELU>), grid, dim3(256), 0, s, p);
    else hipLaunchKernelGGL((group_norm_kernel<T, SEED_ACT_SILU>), grid, dim3(256), 0, s, p);
}

}  // namespace seedinf
