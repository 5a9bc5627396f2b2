// What the stand-alone operators share: their element types and loads of 16 bytes or single elements.
#pragma once
#include <hip/hip_runtime.h>

#include <atomic>
#include <cstddef>
#include <cstdint>

#include "../../include/seedinf.h"
#include "bf16_common.h"

namespace seedinf {

// 16 bytes as they travel.  (HIP's uint4 is a class: choosing between two of them chooses between their addresses, which
// takes them out of registers.)
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// x / (1 + exp(-x)).  The exponential is 2 to the power t = -x / ln 2; what rounding t loses (2^-24 of t, of which the
// result would lose as much) is put back by the derivative.  The instructions for 2^t and the reciprocal are good to one unit
// in the last place: 9 roundings in all.  Results below 2^-118 (x < -87) are zero.  Of a result that is rounded to bf16 T is
// that type: it does without the correction (2^-16 of the result at the far end, beside 2^-9; 65536 groups of 128 bf16:
// 10.2 us, with it 10.9).
template <class T>
__device__ __forceinline__ float op_silu(float x)
{
    if constexpr (sizeof(T) == 2) return x * __builtin_amdgcn_rcpf(1.0f + __expf(-x));
    const float c = __builtin_amdgcn_fmed3f(x, -88.0f, 128.0f), t = c * -1.44269504088896341f;
    const float lost = fmaf(t, -1.90465429995776804525e-9f, fmaf(t, 0.693147182464599609375f, c));     // c + t ln 2
    const float e = __builtin_amdgcn_exp2f(t);
    return x * __builtin_amdgcn_rcpf(1.0f + fmaf(e, -lost, e));
}

template <int ACT, class T>
__device__ __forceinline__ float op_activate(float x)
{
    if constexpr (ACT == SEED_ACT_RELU) return x < 0.0f ? 0.0f : x;    // (a comparison: NaN stays NaN)
    else if constexpr (ACT == SEED_ACT_SILU) return op_silu<T>(x);
    else return x;
}

// More than 64 KiB of LDS has to be asked for, once a kernel and device; `asked` remembers the devices.
static inline hipError_t op_allow_lds(const void* kernel, size_t bytes, std::atomic<uint64_t>& asked)
{
    if (bytes <= 65536) return hipSuccess;
    int dev = 0;
    hipError_t e = hipGetDevice(&dev);
    if (e != hipSuccess) return e;
    const uint64_t bit = 1ull << (dev & 63);
    if (dev < 64 && (asked.load(std::memory_order_relaxed) & bit)) return hipSuccess;
    e = hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, (int)bytes);
    if (e == hipSuccess && dev < 64) asked.fetch_or(bit, std::memory_order_relaxed);
    return e;
}

// What seed_op_sample checks of its arguments (ops.hip), for a step that samples behind its heads.
seed_status_t op_sample_check(int32_t dtype, int32_t rows, int32_t choices, int64_t row_stride, const void* logits, const float* uniforms,
                              const float* temperature, const int32_t* top_k, const float* top_p, const float* min_p, int32_t* token_out, float* logprob_out);

static inline size_t op_dtype_size(int32_t dtype) { return dtype == SEED_DTYPE_FP32 ? 4 : 2; }

}  // namespace seedinf
