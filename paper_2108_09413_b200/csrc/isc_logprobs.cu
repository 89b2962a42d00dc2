// Log probabilities of given tokens, entropies, alternatives and votes from logits (isc_log_probs).
//
//   z_i = scale (l_i - m),  S = sum exp(z),  log p_i = z_i - log S,  H = log S - sum(exp(z) z) / S
//
// One pass over a row: a thread takes every n-th chunk of eight logits and keeps its largest logit m, and S and
// U = sum exp(z) z relative to it, scaled again when a larger one comes; the threads' (m, S, U) are joined at the end.
//
// Alternatives without a second pass.  A thread's chunks are a subset of the row, and each of the row's k largest logits lies
// in one of the k subsets with the largest maxima (a logit whose subset comes after those has k larger ones before it).  So
// a thread keeps its first chunk with its maximum, k subsets are chosen by (maximum, chunk), and only these are read again,
// out of the second-level cache: every logit not below the k-th maximum is a candidate, usually little more than k of them.
// Order is by logit, then by lowest index, held as one 64-bit key, so ties are decided exactly.
//
// Memory bound: 2 bytes a logit in bf16, one exponential each (11.6 logits a clock and SM at the copy bandwidth, of 16
// exponentials).
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

constexpr int kMostTop = 32;
constexpr int kThreads = 512;           // most threads of a block
constexpr int kCandidates = 1024;
constexpr int kMostCluster = 8;
constexpr float kFloorZ = -150.0f;      // exp2 of it is zero in single precision
typedef unsigned long long Key;

struct LogProbParams {
    const void *logits;
    const int64_t *targets;
    float *log_probs, *entropy, *top_log_probs;
    int32_t *top_ids, *votes;
    int64_t rows, ld;
    int vocab, top, cluster;
    float scale, scale2;                // scale2 = scale log2(e)
};

__device__ __forceinline__ float exp2_fast(float v)
{
    float d;
    asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(d) : "f"(v));
    return d;
}

// A logit as an integer that orders as it does (the two zeros are one); and back.
__device__ __forceinline__ uint32_t ordered(float v)
{
    const uint32_t b = __float_as_uint(v + 0.0f);
    return b ^ ((uint32_t)((int)b >> 31) | 0x80000000u);
}
__device__ __forceinline__ float from_ordered(uint32_t o) { return __uint_as_float(o ^ ((uint32_t)((int)~o >> 31) | 0x80000000u)); }
__device__ __forceinline__ Key make_key(float v, uint32_t index) { return (Key)ordered(v) << 32 | (uint32_t)~index; }
__device__ __forceinline__ uint32_t key_index(Key k) { return ~(uint32_t)k; }

// Largest logit, and both sums relative to it in powers of two.
struct Sums {
    float m, s, u;
    __device__ __forceinline__ void scale_to(float to, float c)
    {
        const float d = fmaxf((m - to) * c, kFloorZ), f = exp2_fast(d);      // (NaN, both infinite: nothing summed yet)
        u = f * fmaf(d, s, u);
        s *= f;
        m = to;
    }
};
__device__ __forceinline__ Sums join(Sums a, Sums b, float c)
{
    const float m = fmaxf(a.m, b.m);
    a.scale_to(m, c);
    b.scale_to(m, c);
    return Sums{m, a.s + b.s, a.u + b.u};
}

// What a row's results are made of.
struct RowResult {
    float m, log_s, entropy;
    bool bad, empty;
};
__device__ __forceinline__ RowResult row_result(Sums t, bool bad)
{
    RowResult r;
    r.bad = bad;
    r.empty = !bad && t.m == -INFINITY;
    r.m = t.m;
    r.log_s = bad ? NAN : r.empty ? 0.0f : logf(t.s);
    r.entropy = bad ? NAN : r.empty ? 0.0f : fmaxf(r.log_s - 0.693147180559945f * (t.u / t.s), 0.0f);
    return r;
}
__device__ __forceinline__ float log_prob(const LogProbParams &p, const RowResult &r, float logit)
{
    return r.bad ? NAN : r.empty ? -INFINITY : (logit - r.m) * p.scale - r.log_s;
}
template <typename T> __device__ __forceinline__ void write_row(const LogProbParams &p, const RowResult &r, const T *row_logits, int64_t row)
{
    if (p.entropy) p.entropy[row] = r.entropy;
    if (p.log_probs) {
        const int64_t target = p.targets[row];
        p.log_probs[row] = target < 0 ? 0.0f : target >= p.vocab ? NAN : log_prob(p, r, to_float(row_logits[target]));
    }
}
__device__ __forceinline__ void write_alternative(const LogProbParams &p, const RowResult &r, int64_t row, int place, bool some, uint32_t index, float logit)
{
    p.top_ids[row * p.top + place] = some && !r.bad ? (int32_t)index : -1;
    p.top_log_probs[row * p.top + place] = r.bad ? NAN : some ? log_prob(p, r, logit) : -INFINITY;
}

// ---- a block, or a cluster of blocks, for a row

// A row in chunks of eight: chunk i holds elements 8 i - skew .. 8 i - skew + 7, so that whole chunks are aligned.
template <typename T> struct Row {
    const T *at;
    int vocab, skew, chunks;
    __device__ Row(const T *row, int v) : at(row), vocab(v)
    {
        skew = (int)(((uintptr_t)row & (8 * sizeof(T) < 16 ? 7 : 15)) / sizeof(T));
        chunks = (int)(((int64_t)vocab + skew + 7) >> 3);
    }
    __device__ __forceinline__ Eight<T> load(int chunk) const;
    __device__ __forceinline__ bool whole(int chunk) const { return 8 * chunk >= skew && 8 * (int64_t)chunk - skew + 8 <= vocab; }
    // element j of a chunk as a number, minus infinity outside the row
    __device__ __forceinline__ float value(const Eight<T> &e, int chunk, int j) const
    {
        const int64_t i = 8 * (int64_t)chunk - skew + j;
        return i < 0 || i >= vocab ? -INFINITY : to_float(e.v[j]);
    }
};
template <typename T> __device__ __forceinline__ Eight<T> Row<T>::load(int chunk) const
{
    const int64_t first = 8 * (int64_t)chunk - skew;
    Eight<T> e;
    if (whole(chunk)) {
        if (sizeof(T) == 1) *reinterpret_cast<uint2 *>(&e) = __ldg(reinterpret_cast<const uint2 *>(at + first));
        else {
#pragma unroll
            for (unsigned w = 0; w < (sizeof(e) >= 16 ? sizeof(e) / 16 : 1); ++w) reinterpret_cast<uint4 *>(&e)[w] = __ldg(reinterpret_cast<const uint4 *>(at + first) + w);
        }
    } else {
#pragma unroll
        for (int j = 0; j < 8; ++j) {
            const int64_t i = first + j;
            e.v[j] = at[i < 0 ? 0 : i >= vocab ? vocab - 1 : i];
        }
    }
    return e;
}

struct Shared {
    Sums warp[kThreads / 32];
    Sums block;                         // read by the cluster's other blocks
    int bad, n_candidates;
    Key sorted[kThreads / 32][32];
    Key chosen[kMostTop];
    Key top[kMostTop];                  // read by the cluster's first block
    Key candidate[kCandidates];
};

__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
// the address of another block's copy of a shared variable
__device__ __forceinline__ uint32_t in_block(const void *p, int rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"((uint32_t)__cvta_generic_to_shared(p)), "r"(rank));
    return a;
}
__device__ __forceinline__ uint32_t read_remote(uint32_t addr)
{
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// Places of the `n` keys in `list` by counting the larger ones; the first `k` go to `top` (zero: none).
__device__ void rank_candidates(Shared &sh, int n, int k, int t, int threads)
{
    if (t < kMostTop) sh.top[t] = 0;
    __syncthreads();
    for (int i = t; i < n; i += threads) {
        const Key mine = sh.candidate[i];
        int place = 0;
        for (int j = 0; j < n; ++j) place += sh.candidate[j] > mine;
        if (place < k && mine) sh.top[place] = mine;
    }
    __syncthreads();
}

// The k largest logits of this block's chunks into sh.top.
template <typename T> __device__ void block_top(Shared &sh, const Row<T> &row, float m, int best, int first, int stride, int k, int t, int threads)
{
    const int lane = t & 31, warp = t >> 5, warps = threads >> 5;
    Key key = m > -INFINITY ? make_key(m, (uint32_t)best) : 0;
    // every warp sorts its threads' maxima, the largest first
#pragma unroll
    for (int size = 2; size <= 32; size <<= 1) {
#pragma unroll
        for (int d = size >> 1; d; d >>= 1) {
            const Key other = __shfl_xor_sync(0xffffffffu, key, d);
            const bool keep_larger = ((lane & d) == 0) == ((lane & size) == 0 || size == 32);
            key = (key > other) == keep_larger ? key : other;
        }
    }
    sh.sorted[warp][lane] = key;
    if (t < kMostTop) sh.chosen[t] = 0;
    if (t == 0) sh.n_candidates = 0;
    __syncthreads();
    // its place among all: the larger ones of every other warp, by bisection (keys differ: their chunks do)
    if (lane < k && key) {
        int place = lane;
        for (int w = 0; w < warps; ++w) {
            if (w == warp) continue;
            int lo = 0, hi = min(k, 32);
            while (lo < hi) {
                const int mid = (lo + hi) >> 1;
                if (sh.sorted[w][mid] > key) lo = mid + 1; else hi = mid;
            }
            place += lo;
        }
        if (place < k) sh.chosen[place] = key;
    }
    __syncthreads();
    const Key least = sh.chosen[k - 1];
    for (int j = warp; j < k; j += warps) {
        const Key subset = sh.chosen[j];
        if (!subset) break;
        const int from = (int)(key_index(subset) % (uint32_t)stride);        // the subset's first chunk
        for (int i = from + lane * stride; i < row.chunks; i += 32 * stride) {
            const Eight<T> e = row.load(i);
#pragma unroll
            for (int q = 0; q < 8; ++q) {
                const float v = row.value(e, i, q);
                if (v > -INFINITY && make_key(v, (uint32_t)i) >= least) {
                    const int at = atomicAdd(&sh.n_candidates, 1);
                    if (at < kCandidates) sh.candidate[at] = make_key(v, (uint32_t)(8 * i - row.skew + q));
                }
            }
        }
    }
    __syncthreads();
    const int n = sh.n_candidates;
    if (n <= kCandidates) {
        rank_candidates(sh, n, k, t, threads);
        return;
    }
    // a row whose large logits all lie in a few subsets: one alternative after the other
    Key last = ~(Key)0;
    for (int r = 0; r < kMostTop; ++r) {
        Key found = 0;
        if (r < k)
            for (int i = first; i < row.chunks; i += stride) {
                const Eight<T> e = row.load(i);
#pragma unroll
                for (int q = 0; q < 8; ++q) {
                    const float v = row.value(e, i, q);
                    const Key mine = v > -INFINITY ? make_key(v, (uint32_t)(8 * i - row.skew + q)) : 0;
                    if (mine < last && mine > found) found = mine;
                }
            }
#pragma unroll
        for (int d = 16; d; d >>= 1) found = max(found, __shfl_xor_sync(0xffffffffu, found, d));
        __syncthreads();
        if (lane == 0) sh.sorted[warp][0] = found;
        __syncthreads();
        found = 0;
        for (int w = 0; w < warps; ++w) found = max(found, sh.sorted[w][0]);
        if (t == 0) sh.top[r] = found;
        last = found;
    }
    __syncthreads();
}

template <typename T> __global__ void __launch_bounds__(kThreads) k_log_probs(const __grid_constant__ LogProbParams p)
{
    __shared__ Shared sh;
    const int t = threadIdx.x, threads = blockDim.x, rank = p.cluster > 1 ? (int)(blockIdx.x % (unsigned)p.cluster) : 0;
    const int64_t row_index = blockIdx.x / (unsigned)p.cluster;
    const Row<T> row(static_cast<const T *>(p.logits) + row_index * p.ld, p.vocab);
    const int stride = threads * p.cluster, first = rank * threads + t;
    const float c = p.scale2;
    Sums own{-INFINITY, 0.0f, 0.0f};
    int best = 0;
    bool bad = false;
    constexpr int kAhead = 4;
    for (int i0 = first; i0 < row.chunks; i0 += kAhead * stride) {
        Eight<T> e[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (i0 + a * stride < row.chunks) e[a] = row.load(i0 + a * stride);
#pragma unroll
        for (int a = 0; a < kAhead; ++a) {
            const int i = i0 + a * stride;
            if (i >= row.chunks) continue;
            float x[8];
            if (row.whole(i)) {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = to_float(e[a].v[j]);
            } else {
#pragma unroll
                for (int j = 0; j < 8; ++j) x[j] = row.value(e[a], i, j);
            }
            float m = x[0];
#pragma unroll
            for (int j = 1; j < 8; ++j) m = sizeof(T) == 1 ? fmaxf(m, x[j]) : max_nan(m, x[j]);
            if (sizeof(T) != 1) bad |= !(m < INFINITY);
            if (m > own.m) {
                own.scale_to(m, c);
                best = i;
            }
            if (own.m > -INFINITY) {
#pragma unroll
                for (int j = 0; j < 8; ++j) {
                    const float z = fmaxf((x[j] - own.m) * c, kFloorZ), ez = exp2_fast(z);
                    own.s += ez;
                    own.u = fmaf(ez, z, own.u);
                }
            }
        }
    }
    Sums all = own;
#pragma unroll
    for (int d = 16; d; d >>= 1)
        all = join(all, Sums{__shfl_xor_sync(0xffffffffu, all.m, d), __shfl_xor_sync(0xffffffffu, all.s, d), __shfl_xor_sync(0xffffffffu, all.u, d)}, c);
    if ((t & 31) == 0) sh.warp[t >> 5] = all;
    bad = __syncthreads_or(bad) != 0;
    all = sh.warp[0];
    for (int w = 1; w < threads >> 5; ++w) all = join(all, sh.warp[w], c);
    const int k = max(p.top, p.votes ? 1 : 0);
    if (k) block_top<T>(sh, row, own.m, best, first, stride, k, t, threads);
    if (p.cluster > 1) {
        if (t == 0) { sh.block = all; sh.bad = bad; }
        cluster_sync();
        if (rank == 0) {
            for (int b = 1; t < 32 && b < p.cluster; ++b) {      // the first warp writes the results
                const uint32_t from = in_block(&sh.block, b);
                all = join(all, Sums{__uint_as_float(read_remote(from)), __uint_as_float(read_remote(from + 4)), __uint_as_float(read_remote(from + 8))}, c);
                bad |= read_remote(in_block(&sh.bad, b)) != 0;
            }
            if (k) {
                for (int i = t; i < p.cluster * kMostTop; i += threads) {
                    const uint32_t from = in_block(&sh.top[i % kMostTop], i / kMostTop);
                    sh.candidate[i] = (Key)read_remote(from + 4) << 32 | read_remote(from);
                }
                __syncthreads();
                rank_candidates(sh, p.cluster * kMostTop, k, t, threads);
            }
        }
        cluster_sync();
        if (rank) return;
    }
    const RowResult r = row_result(all, bad);
    if (t == 0) write_row<T>(p, r, row.at, row_index);
    if (t < p.top) {
        const Key key = sh.top[t];
        write_alternative(p, r, row_index, t, key != 0, key_index(key), from_ordered((uint32_t)(key >> 32)));
    }
    if (p.votes && t == 0 && !bad && sh.top[0]) atomicAdd(p.votes + key_index(sh.top[0]), 1);
}

// ---- kLanes lanes of a warp for a row of at most kLanes x kHeld logits, which stay in registers

constexpr int kGroupThreads = 256;
template <typename T, int kLanes, int kHeld> __global__ void __launch_bounds__(kGroupThreads) k_log_probs_group(const __grid_constant__ LogProbParams p)
{
    // votes are counted per block: rows are many and classes few
    __shared__ int32_t votes[kLanes * kHeld];
    if (p.votes) {
        for (int i = threadIdx.x; i < p.vocab; i += kGroupThreads) votes[i] = 0;
        __syncthreads();
    }
    constexpr int kRows = kGroupThreads / kLanes;
    const int lane = threadIdx.x % kLanes;
    const float c = p.scale2;
    // whole groups leave together, but the warp's shuffles need all lanes: rows past the end are computed and not written
    for (int64_t row0 = (int64_t)blockIdx.x * kRows; row0 < p.rows; row0 += (int64_t)gridDim.x * kRows) {
        const int64_t row_index = row0 + threadIdx.x / kLanes;
        const bool mine = row_index < p.rows;
        const T *row = static_cast<const T *>(p.logits) + (mine ? row_index : p.rows - 1) * p.ld;
        float x[kHeld];
        float m = -INFINITY;
#pragma unroll
        for (int e = 0; e < kHeld; ++e) {
            x[e] = e * kLanes + lane < p.vocab ? to_float(row[e * kLanes + lane]) : -INFINITY;
            m = max_nan(m, x[e]);
        }
#pragma unroll
        for (int d = kLanes / 2; d; d >>= 1) m = max_nan(m, __shfl_xor_sync(0xffffffffu, m, d));
        const bool bad = !(m < INFINITY);
        Sums all{m, 0.0f, 0.0f};
        if (m > -INFINITY && !bad) {
#pragma unroll
            for (int e = 0; e < kHeld; ++e) {
                const float z = fmaxf((x[e] - m) * c, kFloorZ), ez = exp2_fast(z);
                all.s += ez;
                all.u = fmaf(ez, z, all.u);
            }
        }
#pragma unroll
        for (int d = kLanes / 2; d; d >>= 1) {
            all.s += __shfl_xor_sync(0xffffffffu, all.s, d);
            all.u += __shfl_xor_sync(0xffffffffu, all.u, d);
        }
        const RowResult r = row_result(all, bad);
        if (mine && lane == 0) write_row<T>(p, r, row, row_index);
        const int k = max(p.top, p.votes ? 1 : 0);
        uint32_t used = 0;
        for (int place = 0; place < k; ++place) {
            float v = -INFINITY;
            int at = 0;
#pragma unroll
            for (int e = 0; e < kHeld; ++e)
                if (!(used >> e & 1) && x[e] > v) { v = x[e]; at = e; }
            uint32_t index = (uint32_t)(at * kLanes + lane);
            const uint32_t own = index;
#pragma unroll
            for (int d = kLanes / 2; d; d >>= 1) {
                const float ov = __shfl_xor_sync(0xffffffffu, v, d);
                const uint32_t oi = __shfl_xor_sync(0xffffffffu, index, d);
                if (ov > v || (ov == v && oi < index)) { v = ov; index = oi; }
            }
            const bool some = v > -INFINITY;
            if (some && own == index) used |= 1u << at;
            if (mine && lane == 0) {
                if (place < p.top) write_alternative(p, r, row_index, place, some, index, v);
                if (place == 0 && p.votes && some && !bad) atomicAdd(votes + index, 1);
            }
        }
    }
    if (p.votes) {
        __syncthreads();
        for (int i = threadIdx.x; i < p.vocab; i += kGroupThreads)
            if (votes[i]) atomicAdd(p.votes + i, votes[i]);
    }
}

template <typename T> cudaError_t launch_log_probs(const Device &dev, LogProbParams p, cudaStream_t st)
{
    if (p.vocab <= 1024) {
        const bool narrow = p.vocab <= 64;
        const int64_t per_block = kGroupThreads / (narrow ? 8 : 32);
        const unsigned grid = (unsigned)std::min<int64_t>((p.rows + per_block - 1) / per_block, 8 * dev.n_sms);
        if (narrow) k_log_probs_group<T, 8, 8><<<grid, kGroupThreads, 0, st>>>(p);
        else k_log_probs_group<T, 32, 32><<<grid, kGroupThreads, 0, st>>>(p);
        return cudaGetLastError();
    }
    const int chunks = p.vocab / 8;
    const int threads = chunks >= 4 * kThreads ? kThreads : chunks >= 2 * kThreads ? kThreads / 2 : kThreads / 4;
    p.cluster = 1;
    while (p.cluster < kMostCluster && p.rows * p.cluster * 2 <= 2 * dev.n_sms && chunks >= 4 * threads * p.cluster) p.cluster *= 2;
    cudaLaunchAttribute attr;
    attr.id = cudaLaunchAttributeClusterDimension;
    attr.val.clusterDim.x = (unsigned)p.cluster;
    attr.val.clusterDim.y = attr.val.clusterDim.z = 1;
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = dim3((unsigned)(p.rows * p.cluster));
    cfg.blockDim = dim3((unsigned)threads);
    cfg.stream = st;
    cfg.attrs = &attr;
    cfg.numAttrs = p.cluster > 1 ? 1 : 0;
    return cudaLaunchKernelEx(&cfg, k_log_probs<T>, p);
}

}  // namespace
}  // namespace isc

extern "C" int isc_log_probs(const void *logits, int64_t ld, int type, int64_t rows, int64_t vocab, float scale, const int64_t *targets, int top,
                             float *out_log_probs, float *out_entropy, int32_t *out_top_ids, float *out_top_log_probs, int32_t *votes, void *cuda_stream)
{
    using namespace isc;
    using namespace isc::ops;
    if (rows < 0 || vocab < 1 || (!is_float_type(type) && type != ISC_I8) || !(scale > 0.0f) || scale > FLT_MAX || top < 0 || top > kMostTop) return ISC_ERR_ARG;
    if (rows == 0) return ISC_OK;
    if (!logits || ld < vocab || (targets != nullptr) != (out_log_probs != nullptr) || (top > 0 && (!out_top_ids || !out_top_log_probs))) return ISC_ERR_ARG;
    if (!aligned(logits, type_bytes(type)) || !aligned(targets, 8) || !aligned(out_log_probs, 4) || !aligned(out_entropy, 4) || !aligned(out_top_ids, 4) || !aligned(out_top_log_probs, 4) ||
        !aligned(votes, 4)) return ISC_ERR_ARG;
    if (rows > INT32_MAX / kMostCluster || vocab > INT32_MAX / 2) return ISC_ERR_UNSUPPORTED;
    Device dev;
    cudaError_t e = current_device(&dev);
    if (e != cudaSuccess) return status_of(e, "device");
    LogProbParams p = {};
    p.logits = logits; p.targets = targets;
    p.log_probs = out_log_probs; p.entropy = out_entropy; p.top_ids = out_top_ids; p.top_log_probs = out_top_log_probs; p.votes = votes;
    p.rows = rows; p.ld = ld; p.vocab = (int)vocab; p.top = top; p.cluster = 1;
    p.scale = scale;
    p.scale2 = scale * 1.44269504088896f;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    e = type == ISC_BF16 ? launch_log_probs<__nv_bfloat16>(dev, p, st) : type == ISC_F16 ? launch_log_probs<__half>(dev, p, st) :
        type == ISC_F32 ? launch_log_probs<float>(dev, p, st) : launch_log_probs<int8_t>(dev, p, st);
    return status_of(e, "log_probs");
}
