// Element types of the embedding and AdamW kernels: values are float32 inside the kernels and
// rounded once, to nearest even, when they are stored.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <type_traits>

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

// one element of an array whose type is known at run time, in two halves, so that several loads can be under way before the
// first is converted
__device__ __forceinline__ uint32_t load_bits(const void* p, int64_t i, int32_t dtype)
{
    return dtype == CHOCO_F32 ? static_cast<const uint32_t*>(p)[i] : (uint32_t)static_cast<const unsigned short*>(p)[i];
}
__device__ __forceinline__ float bits_to_float(uint32_t b, int32_t dtype)
{
    if (dtype == CHOCO_F32) return __uint_as_float(b);
    if (dtype == CHOCO_BF16) return __uint_as_float(b << 16);
    return __half2float(__ushort_as_half((unsigned short)b));
}
__device__ __forceinline__ void store_from_float(void* p, int64_t i, int32_t dtype, float v)
{
    if (dtype == CHOCO_F32) static_cast<float*>(p)[i] = v;
    else if (dtype == CHOCO_BF16) static_cast<__nv_bfloat16*>(p)[i] = from_float<__nv_bfloat16>(v);
    else static_cast<__half*>(p)[i] = from_float<__half>(v);
}

// V consecutive elements as raw words, so that a batch of loads can be in flight before the first
// is unpacked; V * sizeof(T) is 2, 4, 8, 16 or 32 bytes and the address a multiple of it (of 16 for 32).
// Plain loads, not those of read-only memory: AdamW writes what it reads, and a kernel that was launched
// early is there while the one before it still writes.
template <typename T, int V>
struct Raw {
    static constexpr int kBytes = V * (int)sizeof(T);
    uint32_t w[(kBytes + 3) / 4];
};
template <typename T, int V>
__device__ __forceinline__ void load_raw(Raw<T, V>& r, const T* p)
{
    constexpr int b = Raw<T, V>::kBytes;
    if constexpr (b >= 16) {
#pragma unroll
        for (int k = 0; k < b / 16; ++k) {
            const uint4 u = reinterpret_cast<const uint4*>(p)[k];
            r.w[4 * k] = u.x; r.w[4 * k + 1] = u.y; r.w[4 * k + 2] = u.z; r.w[4 * k + 3] = u.w;
        }
    } else if constexpr (b == 8) {
        const uint2 u = *reinterpret_cast<const uint2*>(p);
        r.w[0] = u.x; r.w[1] = u.y;
    } else if constexpr (b == 4) {
        r.w[0] = *reinterpret_cast<const uint32_t*>(p);
    } else {
        r.w[0] = *reinterpret_cast<const unsigned short*>(p);
    }
}
template <typename T, int V>
__device__ __forceinline__ float raw_get(const Raw<T, V>& r, int e)
{
    if constexpr (sizeof(T) == 4) {
        return __uint_as_float(r.w[e]);
    } else {
        const unsigned short h = (unsigned short)(r.w[e / 2] >> (16 * (e & 1)));
        if constexpr (std::is_same_v<T, __nv_bfloat16>) return __uint_as_float((uint32_t)h << 16);
        else return __half2float(__ushort_as_half(h));
    }
}
// the reverse: V floats rounded to T
template <typename T, int V>
__device__ __forceinline__ void store_vec(T* p, const float* f)
{
    constexpr int b = V * (int)sizeof(T);
    uint32_t w[(b + 3) / 4];
    if constexpr (sizeof(T) == 4) {
#pragma unroll
        for (int e = 0; e < V; ++e) w[e] = __float_as_uint(f[e]);
    } else if constexpr (V == 1) {
        *p = from_float<T>(f[0]);
    } else {
#pragma unroll
        for (int e = 0; e < V; e += 2) {
            if constexpr (std::is_same_v<T, __nv_bfloat16>) {
                const __nv_bfloat162 h = __floats2bfloat162_rn(f[e], f[e + 1]);
                w[e / 2] = *reinterpret_cast<const uint32_t*>(&h);
            } else {
                const __half2 h = __floats2half2_rn(f[e], f[e + 1]);
                w[e / 2] = *reinterpret_cast<const uint32_t*>(&h);
            }
        }
    }
    if constexpr (b >= 16) {
#pragma unroll
        for (int k = 0; k < b / 16; ++k)
            reinterpret_cast<uint4*>(p)[k] = make_uint4(w[4 * k], w[4 * k + 1], w[4 * k + 2], w[4 * k + 3]);
    } else if constexpr (b == 8) {
        *reinterpret_cast<uint2*>(p) = make_uint2(w[0], w[1]);
    } else if constexpr (b == 4) {
        *reinterpret_cast<uint32_t*>(p) = w[0];
    }
}

} // namespace choco
