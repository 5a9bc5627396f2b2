// What the stand-alone operators share: their element types and loads of 16 bytes or single elements.
#pragma once
#include <hip/hip_runtime.h>

#include <cstddef>
#include <cstdint>

#include "../../include/seedinf.h"
#include "bf16_common.h"

namespace seedinf {

template <class T> struct ElemVec;
template <> struct ElemVec<float> { static constexpr int N = 4; typedef floatx4 V; };
template <> struct ElemVec<__bf16> { static constexpr int N = 8; typedef bf16x8 V; };

// x / (1 + exp(-x)); the reciprocal instruction is good to one unit in the last place
__device__ __forceinline__ float op_silu(float x) { return x * __builtin_amdgcn_rcpf(1.0f + __expf(-x)); }

template <int ACT>
__device__ __forceinline__ float op_activate(float x)
{
    if constexpr (ACT == SEED_ACT_RELU) return x < 0.0f ? 0.0f : x;    // (a comparison: NaN stays NaN)
    else if constexpr (ACT == SEED_ACT_SILU) return op_silu(x);
    else return x;
}

static inline size_t op_dtype_size(int32_t dtype) { return dtype == SEED_DTYPE_FP32 ? 4 : 2; }

}  // namespace seedinf
