// Root-mean-square norm of x + r with int8 output and one scale per row (isc_rms_norm_quant).
//
//   h = x + r,  p_i = h_i w_i,  n_i = p_i / sqrt(mean(h^2) + eps),  scale = max |n| / 127,  q_i = rint(p_i 127 / max |p|)
//
// The root is the same for a whole row, so it cancels in q: one pass over the row gives both sums (h^2 and max |p|), and the
// codes need no second reduction.  A row is read once and stays in registers: as it lies in memory, because the codes near a
// border between two are computed again from it.
//
// The codes are those of the exact quotient.  In single precision v = p * (127 / max |p|) is off by at most six roundings,
// |v| 2^-21.4; where v is nearer than |v| 2^-21 to the middle between two codes, p and max |p| are computed in double
// precision and divided there.  One row in ten of 4,096 elements has such a code.  Rows whose sums leave the range of single
// precision (values above 1e19 or all below 1e-15, zeros, infinities, NaN) are computed in double precision altogether.
//
// Memory bound: bf16 with a residual 7 bytes an element (reads x and r, writes h and q).
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "isc_ops.cuh"
#include "isc_ops.h"

namespace isc {
namespace {

using namespace ops;

constexpr int kChunks = 4;              // chunks of eight elements a thread holds
constexpr int kBlock = 512;             // most threads for a row
constexpr int kHeld = kBlock * kChunks * 8;
constexpr float kBorder = 4.76837158203125e-7f;      // 2^-21

struct NormParams {
    const void *x, *r, *w;
    void *h;
    int8_t *q;
    float *scale;
    int64_t rows, ldx, ldr, ldh, ldq;
    int width;
    float eps;
    bool wide_w;                        // weights in single precision beside narrower rows
    bool vec, vec_w, vec_h, vec_q;      // 16-byte accesses (8-byte for q) are aligned
};

struct Sums { float ss, most; };

__device__ __forceinline__ Sums combine(Sums a, Sums b) { return Sums{a.ss + b.ss, max_nan(a.most, b.most)}; }

template <typename T> __device__ __forceinline__ float weight_at(const NormParams &p, int i)
{
    return p.wide_w ? __ldg(static_cast<const float *>(p.w) + i) : to_float(static_cast<const T *>(p.w)[i]);
}

// Eight elements of a row from `base` on: `step` apart (1 where accesses are wide).
template <typename T> __device__ __forceinline__ Eight<T> fetch(const T *row, int base, int step, int width, bool vec)
{
    if (vec && base + 8 <= width) return load_eight(row + base);
    Eight<T> e;
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int i = base + j * step;
        e.v[j] = i < width ? row[i] : from_float<T>(0.0f);
    }
    return e;
}

template <typename T> __device__ __forceinline__ void fetch_weights(const NormParams &p, int base, int step, float (&w)[8])
{
    if (p.vec_w && step == 1 && base + 8 <= p.width) {
        if (p.wide_w) {
            const float4 *f = reinterpret_cast<const float4 *>(static_cast<const float *>(p.w) + base);
            const float4 a = __ldg(f), b = __ldg(f + 1);
            w[0] = a.x; w[1] = a.y; w[2] = a.z; w[3] = a.w; w[4] = b.x; w[5] = b.y; w[6] = b.z; w[7] = b.w;
        } else {
            Eight<T> e;
            const uint4 *f = reinterpret_cast<const uint4 *>(static_cast<const T *>(p.w) + base);
#pragma unroll
            for (unsigned i = 0; i < sizeof(e) / 16; ++i) reinterpret_cast<uint4 *>(&e)[i] = __ldg(f + i);
#pragma unroll
            for (int j = 0; j < 8; ++j) w[j] = to_float(e.v[j]);
        }
        return;
    }
#pragma unroll
    for (int j = 0; j < 8; ++j) {
        const int i = base + j * step;
        w[j] = i < p.width ? weight_at<T>(p, i) : 0.0f;
    }
}

// the exact product, or its nearest double-precision number
template <typename T> __device__ __forceinline__ double exact_sum(T x, T r, bool has_r) { return has_r ? (double)to_float(x) + (double)to_float(r) : (double)to_float(x); }

// What a row's threads share.
struct Exchange {
    float ss[kBlock / 32], most[kBlock / 32];
    double ss_d[kBlock / 32];
    unsigned long long most_d;
    int bad;
};

// One row, held by `threads` threads of which this is number `t`; a warp (kWarp) or the block.
template <typename T, bool kWarp>
__device__ void norm_row(const NormParams &p, int64_t row, int t, int threads, Exchange *sh)
{
    const T *x = static_cast<const T *>(p.x) + row * p.ldx, *r = p.r ? static_cast<const T *>(p.r) + row * p.ldr : nullptr;
    const int step = p.vec ? 1 : threads;
    Eight<T> xe[kChunks], re[kChunks];
    int base[kChunks];
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        base[c] = p.vec ? (c * threads + t) * 8 : c * 8 * threads + t;
        if (base[c] < p.width) xe[c] = fetch(x, base[c], step, p.width, p.vec);
    }
    if (r) {
#pragma unroll
        for (int c = 0; c < kChunks; ++c)
            if (base[c] < p.width) re[c] = fetch(r, base[c], step, p.width, p.vec);
    }
    Sums s{0.0f, 0.0f};
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        if (base[c] >= p.width) continue;
        float w[8];
        fetch_weights<T>(p, base[c], step, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float h = r ? to_float(xe[c].v[j]) + to_float(re[c].v[j]) : to_float(xe[c].v[j]);
            s.ss = fmaf(h, h, s.ss);
            s.most = max_nan(s.most, fabsf(h * w[j]));
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) s = combine(s, Sums{__shfl_xor_sync(0xffffffffu, s.ss, d), __shfl_xor_sync(0xffffffffu, s.most, d)});
    if (!kWarp) {
        const int warps = threads >> 5;
        if ((t & 31) == 0) { sh->ss[t >> 5] = s.ss; sh->most[t >> 5] = s.most; }
        if (t == 0) { sh->most_d = 0; sh->bad = 0; }
        __syncthreads();
        s = Sums{0.0f, 0.0f};
        for (int k = 0; k < warps; ++k) s = combine(s, Sums{sh->ss[k], sh->most[k]});
    }
    if (p.h) {
        T *h = static_cast<T *>(p.h) + row * p.ldh;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            if (base[c] >= p.width) continue;
            Eight<T> e;
#pragma unroll
            for (int j = 0; j < 8; ++j) e.v[j] = r ? from_float<T>(to_float(xe[c].v[j]) + to_float(re[c].v[j])) : xe[c].v[j];
            if (p.vec_h && step == 1 && base[c] + 8 <= p.width) store_eight(h + base[c], e);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (base[c] + j * step < p.width) h[base[c] + j * step] = e.v[j];
            }
        }
    }
    // the range in which single precision keeps the sums' relative error
    const bool plain = s.ss >= 1e-30f && s.ss <= 1e37f && s.most >= 1e-30f && s.most <= 1e37f;
    const float inv = 127.0f / s.most;
    uint2 code[kChunks];
    unsigned redo[kChunks];             // one bit for each code that double precision decides
    bool any = !plain;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        code[c] = make_uint2(0, 0);
        redo[c] = 0;
        if (base[c] >= p.width) continue;
        if (!plain) { redo[c] = 0xFFu; continue; }
        float w[8];
        fetch_weights<T>(p, base[c], step, w);
        int k[8];
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const float h = r ? to_float(xe[c].v[j]) + to_float(re[c].v[j]) : to_float(xe[c].v[j]);
            const float v = h * w[j] * inv, near = rintf(v);
            k[j] = (int)near;
            if (0.5f - fabsf(v - near) < fabsf(v) * kBorder) redo[c] |= 1u << j;
        }
        any |= redo[c] != 0;
        code[c].x = (k[0] & 255) | (k[1] & 255) << 8 | (k[2] & 255) << 16 | (unsigned)k[3] << 24;
        code[c].y = (k[4] & 255) | (k[5] & 255) << 8 | (k[6] & 255) << 16 | (unsigned)k[7] << 24;
    }
    any = kWarp ? __any_sync(0xffffffffu, any) : __syncthreads_or(any) != 0;
    float scale = s.most / sqrtf(s.ss / (float)p.width + p.eps) / 127.0f;
    if (any) {
        // the largest product in double precision, among those that single precision puts near it
        const float from = plain ? s.most * (1.0f - 4.0f * kBorder) : 0.0f;
        double most = 0.0, ss = 0.0;
        bool bad = false;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            if (base[c] >= p.width) continue;
            float w[8];
            fetch_weights<T>(p, base[c], step, w);
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const float h = r ? to_float(xe[c].v[j]) + to_float(re[c].v[j]) : to_float(xe[c].v[j]);
                if (plain && !(fabsf(h * w[j]) >= from)) continue;
                const double hd = exact_sum(xe[c].v[j], r ? re[c].v[j] : xe[c].v[j], r != nullptr), pd = fabs(hd * (double)w[j]);
                if (base[c] + j * step < p.width) {
                    ss += hd * hd;
                    bad |= !(pd <= DBL_MAX) || !(fabs(hd) <= DBL_MAX);
                    most = fmax(most, pd);
                }
            }
        }
        if (kWarp) {
#pragma unroll
            for (int d = 16; d; d >>= 1) {
                most = fmax(most, __shfl_xor_sync(0xffffffffu, most, d));
                ss += __shfl_xor_sync(0xffffffffu, ss, d);
            }
            bad = __any_sync(0xffffffffu, bad);
        } else {
#pragma unroll
            for (int d = 16; d; d >>= 1) {
                most = fmax(most, __shfl_xor_sync(0xffffffffu, most, d));
                ss += __shfl_xor_sync(0xffffffffu, ss, d);
            }
            if ((t & 31) == 0) {
                sh->ss_d[t >> 5] = ss;
                atomicMax(&sh->most_d, (unsigned long long)__double_as_longlong(most));      // not negative: ordered as an integer
            }
            bad = __syncthreads_or(bad) != 0;
            most = __longlong_as_double((long long)sh->most_d);
            ss = 0.0;
            for (int k = 0; k < threads >> 5; ++k) ss += sh->ss_d[k];
        }
        if (!plain) scale = bad ? NAN : most > 0.0 ? (float)(most / sqrt(ss / (double)p.width + (double)p.eps) / 127.0) : 0.0f;
        if (bad || !(most > 0.0)) {
#pragma unroll
            for (int c = 0; c < kChunks; ++c) { code[c] = make_uint2(0, 0); redo[c] = 0; }
        }
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            if (!redo[c]) continue;
#pragma unroll
            for (int j = 0; j < 8; ++j) {
                const int i = base[c] + j * step;
                if (!(redo[c] >> j & 1) || i >= p.width) continue;
                const double pd = exact_sum(xe[c].v[j], r ? re[c].v[j] : xe[c].v[j], r != nullptr) * (double)weight_at<T>(p, i);
                const unsigned k = (unsigned)(int)rint(pd * 127.0 / most) & 255u, at = 8 * (j & 3);
                unsigned &word = j < 4 ? code[c].x : code[c].y;
                word = (word & ~(255u << at)) | k << at;
            }
        }
    }
    if (t == 0) p.scale[row] = scale;
    int8_t *q = p.q + row * p.ldq;
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        if (base[c] >= p.width) continue;
        if (p.vec_q && step == 1 && base[c] + 8 <= p.width) *reinterpret_cast<uint2 *>(q + base[c]) = code[c];
        else {
#pragma unroll
            for (int j = 0; j < 8; ++j)
                if (base[c] + j * step < p.width) q[base[c] + j * step] = (int8_t)((j < 4 ? code[c].x : code[c].y) >> 8 * (j & 3));
        }
    }
}

// a block for a row
template <typename T> __global__ void __launch_bounds__(kBlock) k_norm_block(const __grid_constant__ NormParams p)
{
    __shared__ Exchange sh;
    norm_row<T, false>(p, blockIdx.x, threadIdx.x, blockDim.x, &sh);
}

// a warp for a row
constexpr int kWarpRows = 4;
template <typename T> __global__ void __launch_bounds__(32 * kWarpRows) k_norm_warp(const __grid_constant__ NormParams p)
{
    const int64_t row = (int64_t)blockIdx.x * kWarpRows + (threadIdx.x >> 5);
    if (row < p.rows) norm_row<T, true>(p, row, threadIdx.x & 31, 32, nullptr);
}

// Rows too long for registers: read twice, in double precision throughout (each thread reads again, from the second-level
// cache, the elements that it read before, and writes h only then, so h may be x or r).
template <typename T> __global__ void __launch_bounds__(kBlock) k_norm_long(const __grid_constant__ NormParams p)
{
    __shared__ double ss_w[kBlock / 32], most_w[kBlock / 32];
    const int64_t row = blockIdx.x;
    const T *x = static_cast<const T *>(p.x) + row * p.ldx, *r = p.r ? static_cast<const T *>(p.r) + row * p.ldr : nullptr;
    T *h = p.h ? static_cast<T *>(p.h) + row * p.ldh : nullptr;
    const int step = p.vec ? 1 : kBlock;
    double ss = 0.0, most = 0.0;
    bool bad = false;
    for (int first = 0; first < p.width; first += 8 * kBlock) {
        const int base = first + (p.vec ? 8 * threadIdx.x : threadIdx.x);
        if (base >= p.width) continue;
        const Eight<T> xe = fetch(x, base, step, p.width, p.vec), re = r ? fetch(r, base, step, p.width, p.vec) : xe;
        float w[8];
        fetch_weights<T>(p, base, step, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            if (base + j * step >= p.width) continue;
            const double hd = exact_sum(xe.v[j], re.v[j], r != nullptr), pd = fabs(hd * (double)w[j]);
            ss += hd * hd;
            bad |= !(pd <= DBL_MAX) || !(fabs(hd) <= DBL_MAX);
            most = fmax(most, pd);
        }
    }
#pragma unroll
    for (int d = 16; d; d >>= 1) {
        ss += __shfl_xor_sync(0xffffffffu, ss, d);
        most = fmax(most, __shfl_xor_sync(0xffffffffu, most, d));
    }
    if ((threadIdx.x & 31) == 0) { ss_w[threadIdx.x >> 5] = ss; most_w[threadIdx.x >> 5] = most; }
    bad = __syncthreads_or(bad) != 0;
    ss = most = 0.0;
    for (int k = 0; k < kBlock / 32; ++k) { ss += ss_w[k]; most = fmax(most, most_w[k]); }
    if (threadIdx.x == 0)
        p.scale[row] = bad ? NAN : most > 0.0 ? (float)(most / sqrt(ss / (double)p.width + (double)p.eps) / 127.0) : 0.0f;
    int8_t *q = p.q + row * p.ldq;
    for (int first = 0; first < p.width; first += 8 * kBlock) {
        const int base = first + (p.vec ? 8 * threadIdx.x : threadIdx.x);
        if (base >= p.width) continue;
        const Eight<T> xe = fetch(x, base, step, p.width, p.vec), re = r ? fetch(r, base, step, p.width, p.vec) : xe;
        float w[8];
        fetch_weights<T>(p, base, step, w);
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int i = base + j * step;
            if (i >= p.width) continue;
            const double pd = exact_sum(xe.v[j], re.v[j], r != nullptr) * (double)w[j];
            q[i] = bad || !(most > 0.0) ? 0 : (int8_t)(int)rint(pd * 127.0 / most);
            if (h) h[i] = r ? from_float<T>(to_float(xe.v[j]) + to_float(re.v[j])) : xe.v[j];
        }
    }
}

template <typename T> cudaError_t launch_norm(const NormParams &p, cudaStream_t st)
{
    const int chunks = (p.width + 7) / 8;
    if (p.width > kHeld) k_norm_long<T><<<(unsigned)p.rows, kBlock, 0, st>>>(p);
    else if (chunks <= 32 * kChunks) k_norm_warp<T><<<(unsigned)((p.rows + kWarpRows - 1) / kWarpRows), 32 * kWarpRows, 0, st>>>(p);
    else k_norm_block<T><<<(unsigned)p.rows, std::max(64, (chunks + kChunks - 1) / kChunks + 31 & ~31), 0, st>>>(p);
    return cudaGetLastError();
}

}  // namespace
}  // namespace isc

extern "C" int isc_rms_norm_quant(const void *x, int64_t ldx, const void *residual, int64_t ldr, const void *weight, int weight_type, int type, int64_t rows, int64_t width, float eps,
                                  void *sum, int64_t lds, int8_t *q, int64_t ldq, float *scale, void *cuda_stream)
{
    using namespace isc;
    using namespace isc::ops;
    if (rows < 0 || width < 1 || !is_float_type(type) || (weight_type != type && weight_type != ISC_F32) || !(eps >= 0.0f) || eps > FLT_MAX) return ISC_ERR_ARG;
    if (rows == 0) return ISC_OK;
    if (!x || !weight || !q || !scale) return ISC_ERR_ARG;
    if (width > INT32_MAX - 8 * kBlock || rows > INT32_MAX) return ISC_ERR_UNSUPPORTED;
    if (ldx < width || ldq < width || (residual && ldr < width) || (sum && lds < width)) return ISC_ERR_ARG;
    const int bytes = type_bytes(type);
    if (!aligned(x, bytes) || !aligned(residual, bytes) || !aligned(sum, bytes) || !aligned(weight, type_bytes(weight_type)) || !aligned(scale, 4)) return ISC_ERR_ARG;
    NormParams p = {};
    p.x = x; p.r = residual; p.w = weight; p.h = sum; p.q = q; p.scale = scale;
    p.rows = rows; p.ldx = ldx; p.ldr = ldr; p.ldh = lds; p.ldq = ldq;
    p.width = (int)width;
    p.eps = eps;
    p.wide_w = weight_type == ISC_F32 && type != ISC_F32;
    const auto wide = [&](const void *a, int64_t ld) { return aligned(a, 16) && (rows == 1 || ld * bytes % 16 == 0); };
    p.vec = wide(x, ldx) && (!residual || wide(residual, ldr));
    p.vec_w = aligned(weight, 16);
    p.vec_h = wide(sum, lds);
    p.vec_q = aligned(q, 8) && (rows == 1 || ldq % 8 == 0);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const cudaError_t e = type == ISC_BF16 ? launch_norm<__nv_bfloat16>(p, st) : type == ISC_F16 ? launch_norm<__half>(p, st) : launch_norm<float>(p, st);
    return status_of(e, "rms_norm_quant");
}
