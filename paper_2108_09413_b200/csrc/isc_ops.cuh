// What the kernels of the operators on device tensors share: 16-byte loads and stores of the element types, conversions.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "isc_tc.cuh"

namespace isc {
namespace ops {

// Wait of one thread for a phase of an mbarrier, two seconds at most: false after that, or at once when another wait of the
// block has run out before (`failed`, shared).
__device__ __forceinline__ bool wait_limited(uint32_t bar, uint32_t parity, volatile int *failed)
{
    if (tc::mbar_test(bar, parity)) return true;
    const unsigned long long t0 = tc::globaltimer();
    for (int spin = 0; !tc::mbar_try(bar, parity); ++spin)
        if ((spin & 7) == 7 && (*failed || tc::globaltimer() - t0 > 2000000000ull)) {
            *failed = 1;
            return false;
        }
    return true;
}

__device__ __forceinline__ float to_float(float v) { return v; }
__device__ __forceinline__ float to_float(__half v) { return __half2float(v); }
__device__ __forceinline__ float to_float(__nv_bfloat16 v) { return __bfloat162float(v); }
__device__ __forceinline__ float to_float(int8_t v) { return (float)v; }
template <typename T> __device__ __forceinline__ T from_float(float v);
template <> __device__ __forceinline__ float from_float<float>(float v) { return v; }
template <> __device__ __forceinline__ __half from_float<__half>(float v) { return __float2half_rn(v); }
template <> __device__ __forceinline__ __nv_bfloat16 from_float<__nv_bfloat16>(float v) { return __float2bfloat16_rn(v); }

// A kernel file's number of bounded waits that have run out.  It only grows, so that no reader takes it away from another.
__device__ __forceinline__ void count_timeout(uint32_t *timeouts) { atomicAdd(timeouts, 1u); }
// The number after `st`'s work.
inline cudaError_t read_timeouts(const uint32_t &timeouts, cudaStream_t st, uint32_t *count)
{
    const cudaError_t e = cudaMemcpyFromSymbolAsync(count, timeouts, sizeof(*count), 0, cudaMemcpyDeviceToHost, st);
    return e == cudaSuccess ? cudaStreamSynchronize(st) : e;
}

// Eight elements as they lie in memory.
template <typename T> struct alignas(16) Eight { T v[8]; };

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

// Two single-precision numbers that one instruction works on.
typedef unsigned long long Pair;
__device__ __forceinline__ Pair make_pair(float a, float b)
{
    Pair d;
    asm("mov.b64 %0, {%1, %2};" : "=l"(d) : "f"(a), "f"(b));
    return d;
}
__device__ __forceinline__ void split(Pair p, float &a, float &b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(p)); }
__device__ __forceinline__ Pair add2(Pair a, Pair b)
{
    Pair d;
    asm("add.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair mul2(Pair a, Pair b)
{
    Pair d;
    asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(d) : "l"(a), "l"(b));
    return d;
}
__device__ __forceinline__ Pair fma2(Pair a, Pair b, Pair c)
{
    Pair d;
    asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(d) : "l"(a), "l"(b), "l"(c));
    return d;
}
// elements 2 i, 2 i + 1 as numbers, and back
__device__ __forceinline__ Pair pair_of(const Eight<float> &e, int i) { return make_pair(e.v[2 * i], e.v[2 * i + 1]); }
__device__ __forceinline__ Pair pair_of(const Eight<__half> &e, int i)
{
    const float2 f = __half22float2(__halves2half2(e.v[2 * i], e.v[2 * i + 1]));
    return make_pair(f.x, f.y);
}
__device__ __forceinline__ Pair pair_of(const Eight<__nv_bfloat16> &e, int i)
{
    const uint32_t w = reinterpret_cast<const uint32_t *>(&e)[i];
    return make_pair(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ void put_pair(Eight<float> &e, int i, Pair p) { split(p, e.v[2 * i], e.v[2 * i + 1]); }
__device__ __forceinline__ void put_pair(Eight<__half> &e, int i, Pair p)
{
    float a, b;
    split(p, a, b);
    reinterpret_cast<__half2 *>(&e)[i] = __floats2half2_rn(a, b);
}
__device__ __forceinline__ void put_pair(Eight<__nv_bfloat16> &e, int i, Pair p)
{
    float a, b;
    split(p, a, b);
    reinterpret_cast<__nv_bfloat162 *>(&e)[i] = __floats2bfloat162_rn(a, b);
}

// the largest of a and the two magnitudes, a NaN among them kept
__device__ __forceinline__ float max3_abs_nan(float a, float b, float c)
{
    float d;
    asm("max.NaN.abs.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max3_nan(float a, float b, float c)
{
    float d;
    asm("max.NaN.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
}
__device__ __forceinline__ float max3(float a, float b, float c)
{
    float d;
    asm("max.f32 %0, %1, %2, %3;" : "=f"(d) : "f"(a), "f"(b), "f"(c));
    return d;
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
