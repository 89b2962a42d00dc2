// Root-mean-square norm of x + r with int8 output and one scale per row (isc_rms_norm_quant).
//
//   h = x + r,  p_i = h_i w_i,  n_i = p_i / sqrt(mean(h^2) + eps),  scale = max |n| / 127,  q_i = rint(p_i 127 / max |p|)
//
// The root is the same for a whole row, so it cancels in q: one pass over the row gives both sums (h^2 and max |p|), and the
// codes need no second reduction.  The products stay in registers from the sums to the codes.
//
// The codes are those of the exact quotient.  In single precision v = p * (127 / max |p|) is off by at most seven roundings,
// 7 2^-24 |v|; where v is nearer than 10 2^-24 |v| to the middle between two codes (the three units between them cover the test's own
// roundings), p and max |p| are computed in double precision, from the row as it lies in memory, and divided there.  Of 8,192 plain Gaussian
// bf16 elements one row in five has such a code, of a residual stream with a few large channels one in fifty.  Rows whose sums
// leave the range of single precision (values above 1e18, products above 1e20, all of either tiny, zeros, infinities, NaN) are computed in double
// precision altogether.
//
// Forms.  Many rows of more than 1,024 16-bit (512 32-bit) elements: persistent blocks whose teams bring rows ahead by bulk copies (k_norm_ring).
// Else a block for a row, a warp for a short one.  Rows too long for registers are read twice.
//
// Memory bound: bf16 with a residual 7 bytes an element (reads x and r, writes h and q).  Measured: 16,384 x 8,192 bf16 with residual
// 155 to 163 us, 5.8 to 6.0 TB/s (249 us for plain Gaussian rows, one in five of them with a doubtful code); 8,192 x 4,096 fp32 with residual 80 us, 5.4 TB/s;
// one row of 4,096 3.6 us.  Rows at odd addresses (20,000 x 5,001 bf16: 341 us of 107) and beyond registers (4,096 x 20,000: 592 of 88) are far from it.  Two-number instructions, one
// reciprocal and a hardware maximum over the warp brought the persistent form from 210 us there: what it does between
// two barriers is what a row costs.
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

__device__ uint32_t timeouts;            // bounded waits that have run out

constexpr int kChunks = 2;              // chunks of eight elements a thread holds
constexpr int kBlock = 1024;            // most threads for a row
constexpr int kHeld = kBlock * kChunks * 8;
constexpr float kBorder = 5.9604645e-7f;     // 10 2^-24

struct NormParams {
    const void *x, *r, *w;
    void *h;
    int8_t *q;
    float *scale;
    int64_t rows, ldx, ldr, ldh, ldq;
    int width;
    float eps, most_ss;                 // most_ss: largest sum of squares that single precision settles
    bool wide_w;                        // weights in single precision beside narrower rows
    bool vec, vec_w, vec_h, vec_q;      // 16-byte accesses (8-byte for q) are aligned
};

struct Sums { float ss, most; };

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

// x + r in double precision: exact unless their exponents lie far apart
template <typename T> __device__ __forceinline__ double exact_sum(T x, T r, bool has_r) { return has_r ? (double)to_float(x) + (double)to_float(r) : (double)to_float(x); }

// Where single precision leaves no doubt about anything but codes next to the middle between two: the range in which the sums
// keep their relative error, and in which nothing on the way to the scale leaves it: a largest product of 1e20 over a root of 1e-15 / 128 is
// a number still, and a mean square added to eps is one (most_ss).
__device__ __forceinline__ bool in_range(Sums s, float most_ss) { return s.ss >= 1e-30f && s.ss <= most_ss && s.most >= 1e-30f && s.most <= 1e20f; }
// 127 / most; the reciprocal is within one unit in the last place
__device__ __forceinline__ float step_inverse(float most)
{
    float d;
    asm("rcp.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(most));
    return 127.0f * d;
}
__device__ __forceinline__ float row_scale(Sums s, int width, float eps) { return s.most / sqrtf(s.ss / (float)width + eps) / 127.0f; }

constexpr float kRound = 12582912.0f;   // 1.5 2^23: adding it leaves the nearest integer in the low bits, ties to even

// Eight codes from the products, and how far the doubtful one of them is into its neighbourhood: above one half, double
// precision has to decide.
__device__ __forceinline__ uint2 codes_of(const Pair (&p)[4], float inv, float &doubt)
{
    uint32_t t[8];
    const float near = inv * kBorder;
    const Pair inv2 = make_pair(inv, inv), round2 = make_pair(kRound, kRound), minus2 = make_pair(-1.0f, -1.0f);
#pragma unroll
    for (int j = 0; j < 4; ++j) {
        const Pair v = fma2(p[j], inv2, round2), off = fma2(p[j], inv2, fma2(v, minus2, round2));
        float p0, p1, d0, d1, v0, v1;
        split(p[j], p0, p1);
        split(off, d0, d1);
        split(v, v0, v1);
        t[2 * j] = __float_as_uint(v0);
        t[2 * j + 1] = __float_as_uint(v1);
        doubt = max3(doubt, fmaf(fabsf(p0), near, fabsf(d0)), fmaf(fabsf(p1), near, fabsf(d1)));
    }
    return make_uint2(__byte_perm(__byte_perm(t[0], t[1], 0x0040), __byte_perm(t[2], t[3], 0x0040), 0x5410),
                      __byte_perm(__byte_perm(t[4], t[5], 0x0040), __byte_perm(t[6], t[7], 0x0040), 0x5410));
}

// What a thread adds to its row's sums: pairs of squares are summed apart.
struct Partial {
    Pair ss;
    float most;
    __device__ __forceinline__ Partial() : ss(0), most(0.0f) {}
    __device__ __forceinline__ void add(Pair h, Pair p)
    {
        float a, b;
        split(p, a, b);
        ss = fma2(h, h, ss);
        most = max3_abs_nan(most, a, b);
    }
    __device__ __forceinline__ Sums sums() const
    {
        float a, b;
        split(ss, a, b);
        return Sums{a + b, most};
    }
};

// A row's sums in double precision.
struct Exact { double ss, most; };
__device__ __forceinline__ void add_exact(Exact &e, bool &bad, double h, double p)
{
    p = fabs(p);
    h = fabs(h);
    e.ss += h * h;
    e.most = fmax(e.most, p);
    bad |= !(p <= DBL_MAX) || !(h <= DBL_MAX);
}
__device__ __forceinline__ float exact_scale(const Exact &e, bool bad, int width, float eps)
{
    return bad ? NAN : e.most > 0.0 ? (float)(e.most / sqrt(e.ss / (double)width + (double)eps) / 127.0) : 0.0f;
}
__device__ __forceinline__ uint32_t exact_code(double p, double most) { return (uint32_t)(int)rint(p * 127.0 / most) & 255u; }

// What a row's threads share.
template <int kThreads> struct ExchangeFor {
    alignas(16) float ss[kThreads / 32], most[kThreads / 32];
    double ss_exact[kThreads / 32], most_exact[kThreads / 32];
    // by every thread of the block, before its first barrier
    __device__ __forceinline__ void clear(int t, int threads)
    {
        for (int k = t; k < kThreads / 32; k += threads) ss[k] = most[k] = 0.0f;
    }
};
typedef ExchangeFor<kBlock> Exchange;

// The threads that hold one row together: a warp, or a block or part of it with a hardware barrier of its own.
template <bool kWarp> struct Team {
    int t, threads, barrier;
    Exchange *sh;
    __device__ __forceinline__ void sync() const
    {
        __syncwarp();
        if (!kWarp) asm volatile("barrier.cta.sync.aligned %0, %1;" ::"r"(barrier), "r"(threads) : "memory");
    }
    __device__ __forceinline__ bool any(bool v) const
    {
        if (kWarp) return __any_sync(0xffffffffu, v) != 0;
        uint32_t r;
        __syncwarp();
        asm volatile("{\n\t.reg .pred p, q;\n\tsetp.ne.u32 p, %3, 0;\n\tbarrier.cta.red.or.pred.aligned q, %1, %2, p;\n\tselp.u32 %0, 1, 0, q;\n\t}"
                     : "=r"(r) : "r"(barrier), "r"(threads), "r"((uint32_t)v) : "memory");
        return r != 0;
    }
    // every thread gets the row's sums; a barrier has to come before the next call
    __device__ __forceinline__ Sums total(Sums s) const
    {
#pragma unroll
        for (int d = 16; d; d >>= 1) s.ss += __shfl_xor_sync(0xffffffffu, s.ss, d);
        asm("redux.sync.max.NaN.f32 %0, %1, 0xffffffff;" : "=f"(s.most) : "f"(s.most));
        if (kWarp || threads == 32) return s;
        if ((t & 31) == 0) { sh->ss[t >> 5] = s.ss; sh->most[t >> 5] = s.most; }
        sync();
        // four warps at a time; the entries of warps that there are not stay zero
        const float4 *ss = reinterpret_cast<const float4 *>(sh->ss), *most = reinterpret_cast<const float4 *>(sh->most);
        s = Sums{0.0f, 0.0f};
        for (int k = 0; k < threads; k += 128) {
            const float4 a = ss[k >> 7], m = most[k >> 7];
            s.ss += (a.x + a.y) + (a.z + a.w);
            s.most = max3_abs_nan(max3_abs_nan(s.most, m.x, m.y), m.z, m.w);
        }
        return s;
    }
    __device__ __forceinline__ Exact total(Exact e) const
    {
#pragma unroll
        for (int d = 16; d; d >>= 1) {
            e.ss += __shfl_xor_sync(0xffffffffu, e.ss, d);
            e.most = fmax(e.most, __shfl_xor_sync(0xffffffffu, e.most, d));
        }
        if (kWarp) return e;
        if ((t & 31) == 0) { sh->ss_exact[t >> 5] = e.ss; sh->most_exact[t >> 5] = e.most; }
        sync();
        e = Exact{0.0, 0.0};
        for (int k = 0; k < threads >> 5; ++k) { e.ss += sh->ss_exact[k]; e.most = fmax(e.most, sh->most_exact[k]); }
        return e;
    }
};

// The part of a row that single precision leaves in doubt: `plain` rows' codes next to the middle between two, any other row
// altogether (its scale too).  `prod`: the products in single precision; element(i, x, r, w) gives element i mod 8 of this
// thread's chunk i / 8, `held` has a bit for each that exists.  Few elements of a plain row need it, found by their
// products, so that the row's other threads do not wait long.
template <int kN, bool kWarp, typename Element>
__device__ __forceinline__ void settle(const Team<kWarp> &team, Element element, uint32_t held, const Pair (&prod)[kN][4], bool has_r, bool plain, float single_most, int width, float eps,
                                       uint2 (&code)[kN], float &scale)
{
    const float from = single_most * (1.0f - 4.0f * kBorder), inv = step_inverse(single_most);
    uint32_t large = held, doubtful = held;
    if (plain) {
        large = doubtful = 0;
#pragma unroll
        for (int c = 0; c < kN; ++c)
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                float p[2];
                split(prod[c][j], p[0], p[1]);
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const uint32_t bit = 1u << (8 * c + 2 * j + h);
                    // the largest product is among those that single precision puts near it
                    if (fabsf(p[h]) >= from) large |= bit;
                    const float v = fmaf(p[h], inv, kRound) - kRound;
                    if (fmaf(fabsf(p[h]), inv * kBorder, fabsf(fmaf(p[h], inv, -v))) > 0.5f) doubtful |= bit;
                }
            }
        large &= held;
        doubtful &= held;
    }
    Exact e{0.0, 0.0};
    bool bad = false;
    while (large) {
        const int i = __ffs((int)large) - 1;
        large &= large - 1;
        float x, r, w;
        element(i, x, r, w);
        const double h = has_r ? (double)x + (double)r : (double)x;
        add_exact(e, bad, h, h * (double)w);
    }
    bad = team.any(bad);
    e = team.total(e);
    if (!plain) scale = exact_scale(e, bad, width, eps);
    while (doubtful) {
        const int i = __ffs((int)doubtful) - 1;
        doubtful &= doubtful - 1;
        float x, r, w;
        element(i, x, r, w);
        const uint32_t k = !bad && e.most > 0.0 ? exact_code((has_r ? (double)x + (double)r : (double)x) * (double)w, e.most) : 0u, at = 8 * (i & 3);
#pragma unroll
        for (int c = 0; c < kN; ++c) {
            if (i >> 2 == 2 * c) code[c].x = (code[c].x & ~(255u << at)) | k << at;
            if (i >> 2 == 2 * c + 1) code[c].y = (code[c].y & ~(255u << at)) | k << at;
        }
    }
    team.sync();
}

// One row, read straight into registers.
template <typename T, bool kWarp>
__device__ __forceinline__ void norm_row(const NormParams &p, int64_t row, const Team<kWarp> &team)
{
    const T *x = static_cast<const T *>(p.x) + row * p.ldx, *r = p.r ? static_cast<const T *>(p.r) + row * p.ldr : nullptr;
    const int t = team.t, threads = team.threads, step = p.vec ? 1 : threads;
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
    Partial part;
    Pair prod[kChunks][4];
    uint32_t held = 0;                  // a bit for each element that exists
#pragma unroll
    for (int c = 0; c < kChunks; ++c) {
        if (base[c] >= p.width) continue;
#pragma unroll
        for (int j = 0; j < 8; ++j) held |= base[c] + j * step < p.width ? 1u << (8 * c + j) : 0u;
        float w[8];
        fetch_weights<T>(p, base[c], step, w);
#pragma unroll
        for (int j = 0; j < 4; ++j) {
            const Pair h = r ? add2(pair_of(xe[c], j), pair_of(re[c], j)) : pair_of(xe[c], j);
            prod[c][j] = mul2(h, make_pair(w[2 * j], w[2 * j + 1]));
            part.add(h, prod[c][j]);
        }
    }
    const Sums s = team.total(part.sums());
    const bool plain = in_range(s, p.most_ss);
    const float inv = step_inverse(s.most);
    uint2 code[kChunks];
    float doubt = plain ? 0.0f : 1.0f, scale = t == 0 ? row_scale(s, p.width, p.eps) : 0.0f;
#pragma unroll
    for (int c = 0; c < kChunks; ++c)
        if (base[c] < p.width) code[c] = codes_of(prod[c], inv, doubt);
    if (team.any(doubt > 0.5f))
        settle(team, [&](int i, float &xv, float &rv, float &wv) {
            const int c = i >> 3, at = (p.vec ? (c * threads + t) * 8 : c * 8 * threads + t) + (i & 7) * step;
            xv = to_float(x[at]);
            rv = r ? to_float(r[at]) : 0.0f;
            wv = weight_at<T>(p, at);
        }, held, prod, r != nullptr, plain, s.most, p.width, p.eps, code, scale);
    if (p.h) {                          // last: it may be x or r, from which doubtful codes were computed again
        T *h = static_cast<T *>(p.h) + row * p.ldh;
#pragma unroll
        for (int c = 0; c < kChunks; ++c) {
            if (base[c] >= p.width) continue;
            Eight<T> e = xe[c];
            if (r) {
#pragma unroll
                for (int j = 0; j < 4; ++j) put_pair(e, j, add2(pair_of(xe[c], j), pair_of(re[c], j)));
            }
            if (p.vec_h && step == 1 && base[c] + 8 <= p.width) store_eight(h + base[c], e);
            else {
#pragma unroll
                for (int j = 0; j < 8; ++j)
                    if (base[c] + j * step < p.width) h[base[c] + j * step] = e.v[j];
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
    sh.clear(threadIdx.x, blockDim.x);
    __syncthreads();
    norm_row<T, false>(p, blockIdx.x, Team<false>{(int)threadIdx.x, (int)blockDim.x, 0, &sh});
}

// a warp for a row
constexpr int kWarpRows = 4;
template <typename T> __global__ void __launch_bounds__(32 * kWarpRows) k_norm_warp(const __grid_constant__ NormParams p)
{
    const int64_t row = (int64_t)blockIdx.x * kWarpRows + (threadIdx.x >> 5);
    if (row < p.rows) norm_row<T, true>(p, row, Team<true>{(int)threadIdx.x & 31, 32, 0, nullptr});
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

// Many rows: persistent blocks whose teams (a row each, one thread for kHeldChunks chunks) bring their next rows into shared memory by
// bulk copies, kDepth rows ahead, while they work on the present one.  A team keeps its weights in registers from row to row.
// With a block for a row and loads straight into registers the loads of a row waited for the row before on the same SM.
constexpr int kRingThreads = 512, kDepth = 3, kMostTeams = 16, kRingSmem = kRingThreads * 128 * kDepth;      // a thread holds 64 bytes of x and of r
template <typename T> struct RingShape {
    static constexpr int kHeldChunks = sizeof(T) == 2 ? 4 : 2;
    static constexpr int kMostWidth = kRingThreads * kHeldChunks * 8;
};
template <typename T, typename W> __global__ void __launch_bounds__(kRingThreads, 1) k_norm_ring(const __grid_constant__ NormParams p, int team_threads, int row_bytes)
{
    constexpr int kN = RingShape<T>::kHeldChunks;
    extern __shared__ __align__(128) uint8_t slots[];
    __shared__ Exchange sh[kMostTeams];
    __shared__ __align__(8) uint64_t full[kMostTeams][kDepth];
    __shared__ int failed;
    const int teams = blockDim.x / team_threads, which = threadIdx.x / team_threads;
    const Team<false> team{(int)(threadIdx.x % team_threads), team_threads, which, &sh[which]};
    const int t = team.t;
    if (threadIdx.x == 0) failed = 0;
    sh[which].clear(t, team_threads);
    if (t == 0)
        for (int d = 0; d < kDepth; ++d) tc::mbar_init(tc::smem_u32(&full[which][d]), 1);
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    __syncthreads();
    const T *x = static_cast<const T *>(p.x), *r = static_cast<const T *>(p.r);
    const int slot_bytes = r ? 2 * row_bytes : row_bytes;
    uint8_t *mine = slots + (size_t)which * kDepth * slot_bytes;
    const int64_t first = (int64_t)blockIdx.x * teams + which, stride = (int64_t)gridDim.x * teams;
    const auto fetch_row = [&](int64_t row, int slot) {
        const uint32_t bar = tc::smem_u32(&full[which][slot]), dst = tc::smem_u32(mine + slot * slot_bytes);
        tc::mbar_expect_tx(bar, (uint32_t)slot_bytes);
        tc::bulk_g2s(dst, x + row * p.ldx, (uint32_t)row_bytes, bar);
        if (r) tc::bulk_g2s(dst + row_bytes, r + row * p.ldr, (uint32_t)row_bytes, bar);
    };
    int64_t issued = 0;                 // the team's k-th copy goes to slot k mod kDepth
    if (t == 0)
        for (int d = 0; d < kDepth; ++d)
            if (first + d * stride < p.rows) {
                fetch_row(first + d * stride, d);
                ++issued;
            }
    Eight<W> w[kN];
    int base[kN];
    uint32_t held = 0;
#pragma unroll
    for (int c = 0; c < kN; ++c) {
        base[c] = (c * team_threads + t) * 8;
        if (base[c] < p.width) held |= 255u << 8 * c;
        if (base[c] < p.width) w[c] = fetch(static_cast<const W *>(p.w), base[c], 1, p.width, p.vec_w);
    }
    int slot = 0, use = 0;
    for (int64_t row = first; row < p.rows; row += stride) {
        if (!wait_limited(tc::smem_u32(&full[which][slot]), (uint32_t)use & 1u, &failed)) count_timeout(&timeouts);
        const T *xs = reinterpret_cast<const T *>(mine + slot * slot_bytes), *rs = reinterpret_cast<const T *>(mine + slot * slot_bytes + row_bytes);
        Partial part;
        Pair prod[kN][4];
#pragma unroll
        for (int c = 0; c < kN; ++c) {
            if (base[c] >= p.width) continue;
            Eight<T> e = *reinterpret_cast<const Eight<T> *>(xs + base[c]), re;
            if (r) re = *reinterpret_cast<const Eight<T> *>(rs + base[c]);
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const Pair h = r ? add2(pair_of(e, j), pair_of(re, j)) : pair_of(e, j);
                prod[c][j] = mul2(h, pair_of(w[c], j));
                part.add(h, prod[c][j]);
                if (r) put_pair(e, j, h);
            }
            if (p.h) store_eight(static_cast<T *>(p.h) + row * p.ldh + base[c], e);
        }
        const Sums s = team.total(part.sums());
        const bool plain = in_range(s, p.most_ss);
        const float inv = step_inverse(s.most);
        uint2 code[kN];
        float doubt = plain ? 0.0f : 1.0f, scale = t == 0 ? row_scale(s, p.width, p.eps) : 0.0f;
#pragma unroll
        for (int c = 0; c < kN; ++c)
            if (base[c] < p.width) code[c] = codes_of(prod[c], inv, doubt);
        if (team.any(doubt > 0.5f))
            settle(team, [&](int i, float &xv, float &rv, float &wv) {
                const int at = ((i >> 3) * team_threads + t) * 8 + (i & 7);
                xv = to_float(xs[at]);
                rv = r ? to_float(rs[at]) : 0.0f;
                wv = weight_at<T>(p, at);
            }, held, prod, r != nullptr, plain, s.most, p.width, p.eps, code, scale);
        // all of the team have read the slot
        if (t == 0) {
            if (row + kDepth * stride < p.rows && !failed) {
                fetch_row(row + kDepth * stride, slot);
                ++issued;
            }
            p.scale[row] = failed ? NAN : scale;
        }
        int8_t *q = p.q + row * p.ldq;
#pragma unroll
        for (int c = 0; c < kN; ++c)
            if (base[c] < p.width) *reinterpret_cast<uint2 *>(q + base[c]) = code[c];
        if (++slot == kDepth) { slot = 0; ++use; }
    }
    // after a failure copies may still be under way: the block's shared memory stays until they have come, or another limit ends
    if (t == 0 && failed) {
        for (int64_t k = issued > kDepth ? issued - kDepth : 0; k < issued; ++k) {
            int again = 0;
            wait_limited(tc::smem_u32(&full[which][k % kDepth]), (uint32_t)(k / kDepth) & 1u, &again);
        }
    }
}

// Blocks hold as many teams as fit their threads; the fewer rows, the fewer blocks.  Below two rows for each team of the
// device nothing would be brought ahead, and a block for a row is as fast.
template <typename T> cudaError_t launch_ring(const Device &dev, const NormParams &p, cudaStream_t st, bool *taken)
{
    constexpr int kPerThread = RingShape<T>::kHeldChunks * 8;
    *taken = false;
    const int64_t bytes = (int64_t)p.width * (int64_t)sizeof(T);
    if (p.width % 8 || !p.vec || !p.vec_h || !p.vec_q || p.width > RingShape<T>::kMostWidth || p.width <= 32 * kPerThread) return cudaSuccess;
    const int team_threads = ((p.width + kPerThread - 1) / kPerThread + 31) & ~31, teams = std::min(kRingThreads / team_threads, kMostTeams);
    if (p.rows < 2 * (int64_t)teams * dev.n_sms) return cudaSuccess;
    const size_t smem = (size_t)teams * kDepth * (size_t)bytes * (p.r ? 2 : 1);
    void (*const kernel)(NormParams, int, int) = p.wide_w ? k_norm_ring<T, float> : k_norm_ring<T, T>;
    cudaError_t e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, kRingSmem);     // one value: another thread may launch meanwhile
    if (e != cudaSuccess) return e;
    *taken = true;
    kernel<<<(unsigned)dev.n_sms, (unsigned)(teams * team_threads), smem, st>>>(p, team_threads, (int)bytes);
    return cudaGetLastError();
}

template <typename T> cudaError_t launch_norm(const Device &dev, const NormParams &p, cudaStream_t st)
{
    bool taken;
    const cudaError_t e = launch_ring<T>(dev, p, st, &taken);
    if (taken || e != cudaSuccess) return e;
    const int chunks = (p.width + 7) / 8;
    if (p.width > kHeld) k_norm_long<T><<<(unsigned)p.rows, kBlock, 0, st>>>(p);
    else if (chunks <= 32 * kChunks) k_norm_warp<T><<<(unsigned)((p.rows + kWarpRows - 1) / kWarpRows), 32 * kWarpRows, 0, st>>>(p);
    else k_norm_block<T><<<(unsigned)p.rows, std::max(64, ((chunks + kChunks - 1) / kChunks + 31) & ~31), 0, st>>>(p);
    return cudaGetLastError();
}

}  // namespace

namespace ops {
cudaError_t norm_timeouts(cudaStream_t st, uint32_t *count) { return read_timeouts(timeouts, st, count); }
}  // namespace ops
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
    p.most_ss = eps <= 1e38f ? 1e37f : 0.0f;      // (beyond, no row: a sum with eps may not be a number)
    p.wide_w = weight_type == ISC_F32 && type != ISC_F32;
    const auto wide = [&](const void *a, int64_t ld) { return aligned(a, 16) && (rows == 1 || ld * bytes % 16 == 0); };
    p.vec = wide(x, ldx) && (!residual || wide(residual, ldr));
    p.vec_w = aligned(weight, 16);
    p.vec_h = !sum || wide(sum, lds);
    p.vec_q = aligned(q, 8) && (rows == 1 || ldq % 8 == 0);
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    Device dev;
    cudaError_t e = current_device(&dev);
    if (e == cudaSuccess) e = type == ISC_BF16 ? launch_norm<__nv_bfloat16>(dev, p, st) : type == ISC_F16 ? launch_norm<__half>(dev, p, st) : launch_norm<float>(dev, p, st);
    return status_of(e, "rms_norm_quant");
}
