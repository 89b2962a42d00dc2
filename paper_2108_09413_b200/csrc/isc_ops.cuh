// What the kernels of the operators on device tensors share: 16-byte loads and stores of the element types, conversions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

namespace isc {
namespace ops {

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(int8_t v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// Eight elements as they lie in memory.
template <typename T> struct alignas(sizeof(T) == 1 ? 8 : 16) Eight { T v[8]; };

// once-read data: past the first-level cache
template <typename T> __device__ __forceinline__ Eight<T> load_eight(const T *p)
{
    Eight<T> e;
    uint4 *w = reinterpret_cast<uint4 *>(&e);
#pragma unroll
    for (unsigned i = 0; i < sizeof(e) / 16; ++i) w[i] = __ldcs(reinterpret_cast<const uint4 *>(p) + i);
    return e;
}
template <typename T> __device__ __forceinline__ void store_eight(T *p, const Eight<T> &e)
{
    const uint4 *w = reinterpret_cast<const uint4 *>(&e);
#pragma unroll
    for (unsigned i = 0; i < sizeof(e) / 16; ++i) reinterpret_cast<uint4 *>(p)[i] = w[i];
}

// maximum that keeps a NaN
__device__ __forceinline__ float max_nan(float a, float b)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2;" : "=f"(d) : "f"(a), "f"(b));
    return d;
}

}  // namespace ops
}  // namespace isc
