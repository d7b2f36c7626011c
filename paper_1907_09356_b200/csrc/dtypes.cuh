// Element types of the embedding and AdamW kernels: values are float32 inside the kernels and
// rounded once, to nearest even, when they are stored.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "../../include/choco.h"

namespace choco {

inline bool dtype_ok(int32_t t) { return t == CHOCO_F32 || t == CHOCO_BF16 || t == CHOCO_F16; }
inline int64_t dtype_size(int32_t t) { return t == CHOCO_F32 ? 4 : 2; }
inline bool aligned_to(const void* p, int64_t bytes) { return ((uintptr_t)p & (uintptr_t)(bytes - 1)) == 0; }

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }

template <typename T>
__device__ __forceinline__ T from_float(float v);
template <>
__device__ __forceinline__ float from_float<float>(float v) { return v; }
template <>
__device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }
template <>
__device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }

// one element of an array whose type is known at run time
__device__ __forceinline__ float load_as_float(const void* p, int64_t i, int32_t dtype)
{
    if (dtype == CHOCO_F32) return static_cast<const float*>(p)[i];
    if (dtype == CHOCO_BF16) return to_float(static_cast<const __nv_bfloat16*>(p)[i]);
    return to_float(static_cast<const __half*>(p)[i]);
}
__device__ __forceinline__ void store_from_float(void* p, int64_t i, int32_t dtype, float v)
{
    if (dtype == CHOCO_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == CHOCO_BF16) static_cast<__nv_bfloat16*>(p)[i] = from_float<__nv_bfloat16>(v);
    else static_cast<__half*>(p)[i] = from_float<__half>(v);
}

} // namespace choco
