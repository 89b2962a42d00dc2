// Log probabilities of given tokens, entropies, alternatives and votes from logits (isc_log_probs).
//
//   z_i = scale (l_i - m),  S = sum exp(z),  log p_i = z_i - log S,  H = log S - sum(exp(z) z) / S
//
// One pass over a row: a thread takes every n-th chunk of 16 bytes and keeps its largest logit m, and S and
// U = sum exp(z) z relative to it, scaled again when a larger one comes; the threads' (m, S, U) are joined at the end.
//
// Alternatives without a second pass.  A thread's chunks are a subset of the row, and each of the row's k largest logits lies
// in one of the k subsets with the largest maxima (a logit whose subset comes after those has k larger ones before it).  So
// a thread keeps its first chunk with its maximum, k subsets are chosen by (maximum, chunk), and only these are read again,
// out of the second-level cache: every logit not below the k-th maximum is a candidate, usually little more than k of them.
// Order is by logit, then by lowest index, held as one 64-bit key, so ties are decided exactly.
//
// Four forms.  Many long rows: persistent blocks, three to an SM, each with a ring of bulk copies that runs on into the next row while the
// present one's threads join their sums and choose alternatives (k_log_probs_stream).  Few long rows: a block or a cluster of them for a row, joined through
// its shared memory (k_log_probs; tiny factors take it too).  Rows of up to 4,096 logits, or 16,384 where there are many: a warp for a row (k_log_probs_warp).  Up to 64: a few lanes of a
// warp, the row in registers (k_log_probs_group).
//
// What bounds it.  fp32: memory (4,096 x 131,072 with five alternatives 335 us, 98 % of the copy bandwidth).  bf16 has twice the logits a byte and
// is not: 257 us, 64 %; 219 without alternatives.  Eleven instructions a logit, two numbers in one where that goes, fill 63 % of the issue slots, the
// exponentials half of their pipe, and with 24 warps an SM what a warp waits for is its own chain of them.
#include <cuda_runtime.h>
#include <float.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>
#include <type_traits>

#include "isc_ops.cuh"
#include "isc_ops.h"

namespace isc {
namespace {

using namespace ops;

constexpr int kMostTop = 32;
constexpr int kThreads = 512;           // most threads of a block
constexpr int kCandidates = 512;
constexpr int kMostCluster = 8;
constexpr float kFloorZ = -150.0f;      // exp2 of it is zero in single precision
typedef unsigned long long Key;

__device__ uint32_t timeouts;            // bounded waits that have run out

struct LogProbParams {
    const void *logits;
    const int64_t *targets;
    float *log_probs, *entropy, *top_log_probs;
    int32_t *top_ids, *votes;
    int64_t rows, ld;
    int vocab, top, cluster;
    float scale, scale2;                // scale2 = scale log2(e)
    float least, limit;                 // rows whose largest logit lies between them take the short way (set_range)
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

// (x - m) c.  kFar: also where the difference is beyond single precision's range and a tiny factor brings the two near each other; that of their
// halves is not, and halving is exact.
template <bool kFar> __device__ __forceinline__ float times_difference(float x, float m, float c) { return kFar ? fmaf(0.5f, x, -0.5f * m) * (2.0f * c) : (x - m) * c; }
constexpr float kTinyFactor = 1e-36f;   // from here on such a difference's exponential is zero

// Largest logit, and both sums relative to it in powers of two.
struct Sums {
    float m, s, u;
    template <bool kFar> __device__ __forceinline__ void scale_to(float to, float c)
    {
        const float d = fmaxf(times_difference<kFar>(m, to, c), kFloorZ), f = exp2_fast(d);      // (NaN, both infinite: nothing summed yet)
        u = f * fmaf(d, s, u);
        s *= f;
        m = to;
    }
};
template <bool kFar> __device__ __forceinline__ Sums join(Sums a, Sums b, float c)
{
    const float m = fmaxf(a.m, b.m);
    a.scale_to<kFar>(m, c);
    b.scale_to<kFar>(m, c);
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
    return r.bad ? NAN : r.empty ? -INFINITY : times_difference<true>(logit, r.m, p.scale) - r.log_s;
}
// A row's given token, loaded ahead of the row: two dependent loads that its end would wait for.
struct Given { int64_t target; float logit; };
template <typename T> __device__ __forceinline__ Given given_of(const LogProbParams &p, const T *row_logits, int64_t row, bool mine)
{
    Given g{-1, 0.0f};
    if (mine && p.log_probs) {
        g.target = p.targets[row];
        if (g.target >= 0 && g.target < p.vocab) g.logit = to_float(row_logits[g.target]);
    }
    return g;
}
__device__ __forceinline__ void write_row(const LogProbParams &p, const RowResult &r, const Given &g, int64_t row)
{
    if (p.entropy) p.entropy[row] = r.entropy;
    if (p.log_probs) p.log_probs[row] = g.target < 0 ? 0.0f : g.target >= p.vocab ? NAN : log_prob(p, r, g.logit);
}
__device__ __forceinline__ void write_alternative(const LogProbParams &p, const RowResult &r, int64_t row, int place, bool some, uint32_t index, float logit)
{
    p.top_ids[row * p.top + place] = some && !r.bad ? (int32_t)index : -1;
    p.top_log_probs[row * p.top + place] = r.bad ? NAN : some ? log_prob(p, r, logit) : -INFINITY;
}

// ---- long rows

// Sixteen bytes of a row.
template <typename T> struct alignas(16) Chunk {
    static constexpr int kSize = 16 / (int)sizeof(T);
    T v[kSize];
};
__device__ __forceinline__ Pair pair_in(const Chunk<float> &c, int i) { return make_pair(c.v[2 * i], c.v[2 * i + 1]); }
__device__ __forceinline__ Pair pair_in(const Chunk<__half> &c, int i)
{
    const float2 f = __half22float2(reinterpret_cast<const __half2 *>(&c)[i]);
    return make_pair(f.x, f.y);
}
__device__ __forceinline__ Pair pair_in(const Chunk<__nv_bfloat16> &c, int i)
{
    const uint32_t w = reinterpret_cast<const uint32_t *>(&c)[i];
    return make_pair(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}
__device__ __forceinline__ Pair pair_in(const Chunk<int8_t> &c, int i) { return make_pair((float)c.v[2 * i], (float)c.v[2 * i + 1]); }

// A row: whole aligned chunks, and up to 15 logits before the first and behind the last of them.
template <typename T> struct Row {
    const T *at;
    int vocab, head, chunks;
    __device__ Row(const T *row, int v) : at(row), vocab(v)
    {
        head = (int)((0u - (uint32_t)(uintptr_t)row & 15u) / (uint32_t)sizeof(T));
        chunks = (vocab - head) / Chunk<T>::kSize;
    }
    __device__ __forceinline__ const T *body() const { return at + head; }
    __device__ __forceinline__ Chunk<T> load(int chunk) const
    {
        Chunk<T> c;
        *reinterpret_cast<uint4 *>(&c) = __ldg(reinterpret_cast<const uint4 *>(body()) + chunk);
        return c;
    }
    __device__ __forceinline__ int index(int chunk, int j) const { return head + chunk * Chunk<T>::kSize + j; }
    // the logit outside the chunks that lane `lane` (0 .. 31) of one warp takes: its index, or -1
    __device__ __forceinline__ int edge(int lane) const
    {
        const int i = lane < 16 ? lane : index(chunks, 0) + lane - 16;
        return lane < 16 ? (i < head ? i : -1) : i < vocab ? i : -1;
    }
};

// Masked logits as numbers that a product with zero leaves zero: minus infinity as the lowest finite number that the type's arithmetic
// below can do without (kMasked), and whatever lies under it.  It stands for a mask only where its exponential is zero as well: below a largest
// logit that set_range gives.
template <typename T> struct Finite {
    static constexpr float kMasked = -1e30f;
    static __device__ __forceinline__ Chunk<T> of(Chunk<T> c) { return c; }
};
template <> struct Finite<__half> {
    static constexpr float kMasked = -65504.0f;
    static __device__ __forceinline__ Chunk<__half> of(Chunk<__half> c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) asm("max.f16x2 %0, %0, %1;" : "+r"(reinterpret_cast<uint32_t *>(&c)[j]) : "r"(0xFBFFFBFFu));
        return c;
    }
};
template <> struct Finite<__nv_bfloat16> {
    static constexpr float kMasked = -1.2676506e30f;     // -2^100
    static __device__ __forceinline__ Chunk<__nv_bfloat16> of(Chunk<__nv_bfloat16> c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) asm("max.bf16x2 %0, %0, %1;" : "+r"(reinterpret_cast<uint32_t *>(&c)[j]) : "r"(0xF180F180u));
        return c;
    }
};
template <> struct Finite<float> {
    static constexpr float kMasked = -1e30f;
    static __device__ __forceinline__ Chunk<float> of(Chunk<float> c)
    {
#pragma unroll
        for (int j = 0; j < 4; ++j) c.v[j] = fmaxf(c.v[j], kMasked);
        return c;
    }
};

// Whether there is a mask among fp16 logits, where it has to be known (set_range).
__device__ __forceinline__ bool any_masked(const Chunk<__half> &e)
{
    uint32_t least = 0x7BFF7BFFu;
#pragma unroll
    for (int j = 0; j < 4; ++j) asm("min.f16x2 %0, %0, %1;" : "+r"(least) : "r"(reinterpret_cast<const uint32_t *>(&e)[j]));
    return (least & 0xFFFFu) == 0xFC00u || least >> 16 == 0xFC00u;
}
template <typename T> __device__ __forceinline__ bool any_masked(const Chunk<T> &) { return true; }

template <typename T> __device__ __forceinline__ float largest(const Chunk<T> &e)
{
    float most = -INFINITY;
#pragma unroll
    for (int j = 0; j < Chunk<T>::kSize / 2; ++j) {
        float a, b;
        split(pair_in(e, j), a, b);
        most = sizeof(T) == 1 ? max3(most, a, b) : max3_nan(most, a, b);
    }
    return most;
}

// A thread's part of a row.  Sums are kept as pairs, relative to m.
template <bool kFar> struct Own {
    float m = -INFINITY, seen = -INFINITY;      // seen: m, or NaN if there is one
    Pair s = 0, u = 0;
    float top = -INFINITY;              // of the present subset of its chunks: the largest logit,
    int best = 0;                       // the first chunk that has it
    __device__ __forceinline__ Key subset()
    {
        const Key k = top > -INFINITY ? make_key(top, (uint32_t)best) : 0;
        top = -INFINITY;
        return k;
    }
    __device__ __forceinline__ Sums sums() const
    {
        float a, b, x, y;
        split(s, a, b);
        split(u, x, y);
        return Sums{m, a + b, x + y};
    }
    // a larger logit
    __device__ __forceinline__ void rise(float to, float c)
    {
        Sums all = sums();
        all.scale_to<kFar>(to, c);
        m = to;
        s = make_pair(all.s, 0.0f);
        u = make_pair(all.u, 0.0f);
    }
    // Logits between -1e30 and 1e29, but for masks, and factors below 1e8: no difference leaves single precision's range.  No masks, or
    // m far enough above kMasked that nothing at or below it weighs anything.
    template <typename T> __device__ __forceinline__ void add_plain(const Chunk<T> &masked, Pair minus_m, Pair c2)
    {
        const Chunk<T> e = Finite<T>::of(masked);
#pragma unroll
        for (int j = 0; j < Chunk<T>::kSize / 2; ++j) {
            float a, b;
            const Pair z = mul2(add2(pair_in(e, j), minus_m), c2);
            split(z, a, b);
            const Pair e2 = make_pair(exp2_fast(a), exp2_fast(b));
            s = add2(s, e2);
            u = fma2(e2, z, u);
        }
    }
    // any logits
    template <typename T> __device__ __noinline__ static void add_any(const Chunk<T> &e, float m, float c, Pair &s, Pair &u)
    {
        float sum = 0.0f, weighted = 0.0f;
        for (int j = 0; j < Chunk<T>::kSize; ++j) {
            const float z = fmaxf(times_difference<kFar>(to_float(e.v[j]), m, c), kFloorZ), ez = exp2_fast(z);
            sum += ez;
            weighted = fmaf(ez, z, weighted);
        }
        s = add2(s, make_pair(sum, 0.0f));
        u = add2(u, make_pair(weighted, 0.0f));
    }
    // chunks first, first + stride, ...: `n` of them
    template <typename T, int kN> __device__ __forceinline__ void add(const Chunk<T> (&e)[kN], int n, int first, int stride, float c, float least, float limit)
    {
        float most[kN], all = -INFINITY;
#pragma unroll
        for (int i = 0; i < kN; ++i) {
            most[i] = i < n ? largest(e[i]) : -INFINITY;
            all = sizeof(T) == 1 ? fmaxf(all, most[i]) : max_nan(all, most[i]);
        }
        if (sizeof(T) != 1) seen = max_nan(seen, all);
        if (all > top) {
            top = all;
#pragma unroll
            for (int i = kN - 1; i >= 0; --i)
                if (most[i] == all) best = first + i * stride;
            if (all > m) rise(all, c);
        }
        bool plain = m > least;
        if (sizeof(T) == 2 && !plain) {
            plain = true;
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (i < n && any_masked(e[i])) plain = false;
        }
        if (plain && fabsf(m) < limit) {
            const Pair minus_m = make_pair(-m, -m), c2 = make_pair(c, c);
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (i < n) add_plain(e[i], minus_m, c2);
        } else if (m > -INFINITY) {
#pragma unroll
            for (int i = 0; i < kN; ++i)
                if (i < n) {
                    Chunk<T> copy = e[i];
                    Pair s_now = s, u_now = u;
                    add_any(copy, m, c, s_now, u_now);
                    s = s_now;
                    u = u_now;
                }
        }
    }
};

template <int kWarps, int kSubsets = 1> struct Shared {
    Sums warp[kWarps];
    Sums block;                         // read by the cluster's other blocks
    int bad[kWarps], block_bad, n_candidates, n_chosen;
    int chosen[32 * kWarps * kSubsets]; // first chunks of the subsets that hold the alternatives
    Key group[32], found[kWarps];
    Key top[kMostTop];                  // read by the cluster's first block
    alignas(16) Key candidate[kCandidates];
};

// The threads that share a row, with a hardware barrier of their own.
struct Team {
    int t, threads, barrier;            // barrier < 0: one warp
    __device__ __forceinline__ void sync() const
    {
        __syncwarp();
        if (barrier >= 0) asm volatile("barrier.cta.sync.aligned %0, %1;" ::"r"(barrier), "r"(threads) : "memory");
    }
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

// Every thread gets its team's sums.  `edge`: this thread's logit outside the chunks (minus infinity: none).
template <bool kFar, int kWarps, int kSubsets> __device__ __forceinline__ Sums join_all(Shared<kWarps, kSubsets> &sh, const Team &team, const Own<kFar> &own, float edge, float c, bool &bad)
{
    Sums all = own.sums();
    if (edge > -INFINITY) all = join<kFar>(all, Sums{edge, 1.0f, 0.0f}, c);
    bad = !(own.seen < INFINITY) || edge != edge || edge == INFINITY;
#pragma unroll
    for (int d = 16; d; d >>= 1)
        all = join<kFar>(all, Sums{__shfl_xor_sync(0xffffffffu, all.m, d), __shfl_xor_sync(0xffffffffu, all.s, d), __shfl_xor_sync(0xffffffffu, all.u, d)}, c);
    bad = __any_sync(0xffffffffu, bad) != 0;
    if ((team.t & 31) == 0) { sh.warp[team.t >> 5] = all; sh.bad[team.t >> 5] = bad; }
    if (team.t == 0) sh.n_candidates = 0;
    team.sync();
    all = sh.warp[0];
    bad = sh.bad[0] != 0;
    for (int w = 1; w < team.threads >> 5; ++w) { all = join<kFar>(all, sh.warp[w], c); bad |= sh.bad[w] != 0; }
    return all;
}

// Place of the key at `lane` of list `own` among all of `lists` falling lists (at most eight), by bisection in all at once (keys differ).
__device__ __forceinline__ void place_key(const Key (*sorted)[32], int lists, int own, int lane, Key key, int k, Key *out)
{
    if (lane >= k || !key) return;
    int larger[kMostCluster] = {};
#pragma unroll
    for (int step = 16; step; step >>= 1)
#pragma unroll
        for (int w = 0; w < kMostCluster; ++w)
            if (w < lists && sorted[w][larger[w] + step - 1] > key) larger[w] += step;
    int place = lane;
#pragma unroll
    for (int w = 0; w < kMostCluster; ++w)
        if (w < lists && w != own) place += larger[w] + (larger[w] == 31 && sorted[w][31] > key);
    if (place < k) out[place] = key;
}

// Places of the `n` keys in `list` by counting the larger ones; the first `k` go to `top` (zero: none).
template <int kWarps, int kSubsets> __device__ void rank_candidates(Shared<kWarps, kSubsets> &sh, const Team &team, int n, int k)
{
    if (team.t < kMostTop) sh.top[team.t] = 0;
    team.sync();
    for (int i = team.t; i < n; i += team.threads) {
        const Key mine = sh.candidate[i];
        int place = 0;
#pragma unroll 8
        for (int j = 0; j < n; ++j) place += sh.candidate[j] > mine;
        if (place < k && mine) sh.top[place] = mine;
    }
    team.sync();
}

// The k largest logits of this team's chunks and edges into sh.top; after join_all.  A thread's chunks are first, first + stride, ...; its
// subsets, `each` of them one after the other, have the keys `key`.
template <typename T, int kWarps, int kSubsets>
__device__ void team_top(Shared<kWarps, kSubsets> &sh, const Team &team, const Row<T> &row, const Key (&key)[kSubsets], float edge, int edge_index, int first, int stride, int each, int k)
{
    const int t = team.t, lane = t & 31, warp = t >> 5, warps = team.threads >> 5;
    constexpr int kSize = Chunk<T>::kSize;
    // The k-th largest of 32 groups' largest keys: k subsets at least reach it, and seldom many more (all of a warp's lanes
    // are a group each, k exactly).  A full order of the subsets' maxima took 1.5 us here.
    const int group = team.threads >> 5;
    Key most = 0;
#pragma unroll
    for (int s = 0; s < kSubsets; ++s) most = max(most, key[s]);
    for (int d = 1; d < group; d <<= 1) most = max(most, __shfl_xor_sync(0xffffffffu, most, d));
    if ((t & (group - 1)) == 0) sh.group[t / group] = most;
    if (t == 0) sh.n_chosen = 0;
    team.sync();
    most = sh.group[lane];
    int larger = 0;
#pragma unroll 8
    for (int j = 0; j < 32; ++j) larger += sh.group[j] > most;
    const uint32_t kth = __ballot_sync(0xffffffffu, most && larger == k - 1);
    const Key least = kth ? __shfl_sync(0xffffffffu, most, __ffs((int)kth) - 1) : 1;
#pragma unroll
    for (int s = 0; s < kSubsets; ++s)
        if (key[s] >= least) sh.chosen[atomicAdd(&sh.n_chosen, 1)] = first + s * each * stride;
    if (edge > -INFINITY) {
        const int at = atomicAdd(&sh.n_candidates, 1);
        sh.candidate[at] = make_key(edge, (uint32_t)edge_index);     // (the first few: there is room)
    }
    team.sync();
    // the chosen subsets' chunks, dealt out over all threads, four loads of a thread under way at once
    const int items = sh.n_chosen * each;
    for (int i0 = t; i0 < items; i0 += 4 * team.threads) {
        Chunk<T> e[4];
        int chunk[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            const int i = i0 + a * team.threads, j = i / each;
            chunk[a] = i < items ? sh.chosen[j] + (i - j * each) * stride : row.chunks;
            if (chunk[a] < row.chunks) e[a] = row.load(chunk[a]);
        }
#pragma unroll
        for (int a = 0; a < 4; ++a) {
            if (chunk[a] >= row.chunks) continue;
#pragma unroll
            for (int q = 0; q < kSize; ++q) {
                const float v = to_float(e[a].v[q]);
                if (v > -INFINITY && make_key(v, (uint32_t)chunk[a]) >= least) {
                    const int at = atomicAdd(&sh.n_candidates, 1);
                    if (at < kCandidates) sh.candidate[at] = make_key(v, (uint32_t)row.index(chunk[a], q));
                }
            }
        }
    }
    team.sync();
    const int n = sh.n_candidates;
    if (n <= kCandidates) {
        rank_candidates(sh, team, n, k);
        return;
    }
    // a row whose large logits all lie in a few subsets: one alternative after the other
    Key last = ~(Key)0;
    for (int r = 0; r < kMostTop; ++r) {
        Key found = 0;
        if (r < k) {
            if (edge > -INFINITY && make_key(edge, (uint32_t)edge_index) < last) found = make_key(edge, (uint32_t)edge_index);
            for (int i = first; i < row.chunks; i += stride) {
                const Chunk<T> e = row.load(i);
#pragma unroll
                for (int q = 0; q < kSize; ++q) {
                    const float v = to_float(e.v[q]);
                    const Key mine = v > -INFINITY ? make_key(v, (uint32_t)row.index(i, q)) : 0;
                    if (mine < last && mine > found) found = mine;
                }
            }
        }
#pragma unroll
        for (int d = 16; d; d >>= 1) found = max(found, __shfl_xor_sync(0xffffffffu, found, d));
        team.sync();
        if (lane == 0) sh.found[warp] = found;
        team.sync();
        found = 0;
        for (int w = 0; w < warps; ++w) found = max(found, sh.found[w]);
        if (t == 0) sh.top[r] = found;
        last = found;
    }
    team.sync();
}

// by one thread for each alternative at least
template <int kWarps, int kSubsets> __device__ __forceinline__ void write_results(const LogProbParams &p, const Shared<kWarps, kSubsets> &sh, const Given &given, int64_t row_index, Sums all, bool bad, int t)
{
    const RowResult r = row_result(all, bad);
    if (t == 0) write_row(p, r, given, row_index);
    if (t < p.top) {
        const Key key = sh.top[t];
        write_alternative(p, r, row_index, t, key != 0, key_index(key), from_ordered((uint32_t)(key >> 32)));
    }
    if (p.votes && t == 0 && !bad && sh.top[0]) atomicAdd(p.votes + key_index(sh.top[0]), 1);
}

// few rows: a block or a cluster of them for a row.  kFar: tiny factors, any number of rows
template <typename T, bool kFar> __global__ void __launch_bounds__(kThreads) k_log_probs(const __grid_constant__ LogProbParams p)
{
    __shared__ Shared<kThreads / 32> sh;
    const Team team{(int)threadIdx.x, (int)blockDim.x, 0};
    const int t = team.t, threads = team.threads, rank = p.cluster > 1 ? (int)(blockIdx.x % (unsigned)p.cluster) : 0;
    const int64_t row_index = blockIdx.x / (unsigned)p.cluster;
    const Row<T> row(static_cast<const T *>(p.logits) + row_index * p.ld, p.vocab);
    const int stride = threads * p.cluster, first = rank * threads + t, edge_index = rank == 0 && t < 32 ? row.edge(t) : -1;
    const float c = p.scale2, edge = edge_index >= 0 ? to_float(row.at[edge_index]) : -INFINITY;
    const Given given = given_of(p, row.at, row_index, rank == 0 && t == 0);
    Own<kFar> own;
    constexpr int kAhead = 4;
    for (int i0 = first; i0 < row.chunks; i0 += kAhead * stride) {
        Chunk<T> e[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (i0 + a * stride < row.chunks) e[a] = row.load(i0 + a * stride);
        own.add(e, (row.chunks - i0 + stride - 1) / stride, i0, stride, c, p.least, p.limit);
    }
    bool bad;
    Sums all = join_all(sh, team, own, edge, c, bad);
    const int k = max(p.top, p.votes ? 1 : 0);
    const Key key[1] = {own.subset()};
    if (k) team_top<T>(sh, team, row, key, edge, edge_index, first, stride, (row.chunks + stride - 1) / stride, k);
    if (p.cluster > 1) {
        if (t == 0) { sh.block = all; sh.block_bad = bad; }
        cluster_sync();
        if (rank == 0) {
            for (int b = 1; t < 32 && b < p.cluster; ++b) {      // the first warp writes the results
                const uint32_t from = in_block(&sh.block, b);
                all = join<kFar>(all, Sums{__uint_as_float(read_remote(from)), __uint_as_float(read_remote(from + 4)), __uint_as_float(read_remote(from + 8))}, c);
                bad |= read_remote(in_block(&sh.block_bad, b)) != 0;
            }
            if (k) {
                Key (*const sorted)[32] = reinterpret_cast<Key (*)[32]>(sh.candidate);
                const int list = t / kMostTop, lane = t % kMostTop;
                Key key = 0;
                if (list < p.cluster) {
                    const uint32_t from = in_block(&sh.top[lane], list);
                    key = (Key)read_remote(from + 4) << 32 | read_remote(from);
                    sorted[list][lane] = key;
                }
                team.sync();
                if (t < kMostTop) sh.top[t] = 0;             // (this block's own list has been copied)
                team.sync();
                if (list < p.cluster) place_key(sorted, p.cluster, list, lane, key, k, sh.top);
                team.sync();
            }
        }
        cluster_sync();
        if (rank) return;
    }
    write_results(p, sh, given, row_index, all, bad, t);
}

// rows of middling length: a warp for a row
constexpr int kRowWarps = 4;
template <typename T> __global__ void __launch_bounds__(32 * kRowWarps) k_log_probs_warp(const __grid_constant__ LogProbParams p)
{
    __shared__ Shared<1> shared[kRowWarps];
    Shared<1> &sh = shared[threadIdx.x >> 5];
    const Team team{(int)threadIdx.x & 31, 32, -1};
    const int t = team.t, k = max(p.top, p.votes ? 1 : 0);
    const float c = p.scale2;
    const int64_t r = (int64_t)blockIdx.x * kRowWarps + (threadIdx.x >> 5);
    if (r >= p.rows) return;
    const Row<T> row(static_cast<const T *>(p.logits) + r * p.ld, p.vocab);
    const int edge_index = row.edge(t);
    const float edge = edge_index >= 0 ? to_float(row.at[edge_index]) : -INFINITY;
    const Given given = given_of(p, row.at, r, t == 0);
    Own<false> own;
    constexpr int kAhead = 4;
    for (int i0 = t; i0 < row.chunks; i0 += 32 * kAhead) {
        Chunk<T> e[kAhead];
#pragma unroll
        for (int a = 0; a < kAhead; ++a)
            if (i0 + a * 32 < row.chunks) e[a] = row.load(i0 + a * 32);
        own.add(e, (row.chunks - i0 + 31) / 32, i0, 32, c, p.least, p.limit);
    }
    bool bad;
    const Sums all = join_all(sh, team, own, edge, c, bad);
    const Key key[1] = {own.subset()};
    if (k) team_top<T>(sh, team, row, key, edge, edge_index, t, 32, (row.chunks + 31) / 32, k);
    write_results(p, sh, given, r, all, bad, t);
}

// many rows: eight warps that work and one that copies
static_assert(kCandidates >= 512, "two keys for each thread");
constexpr int kStreamThreads = 256, kPieces = 4, kPieceBytes = 16384, kStreamBlocks = 3, kStreamSubsets = 2;
template <typename T> __global__ void __launch_bounds__(kStreamThreads + 32, kStreamBlocks) k_log_probs_stream(const __grid_constant__ LogProbParams p)
{
    extern __shared__ __align__(128) uint8_t pieces[];
    __shared__ Shared<kStreamThreads / 32, kStreamSubsets> sh;
    __shared__ __align__(8) uint64_t full[kPieces], empty[kPieces];
    __shared__ int failed;
    if (threadIdx.x == 0) {
        for (int i = 0; i < kPieces; ++i) { tc::mbar_init(tc::smem_u32(&full[i]), 1); tc::mbar_init(tc::smem_u32(&empty[i]), kStreamThreads / 32); }
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        failed = 0;
    }
    __syncthreads();
    const T *logits = static_cast<const T *>(p.logits);
    constexpr int kPieceChunks = kPieceBytes / 16;
    int slot = 0, use = 0;
    if (threadIdx.x >= kStreamThreads) {
        if (threadIdx.x == kStreamThreads) {
            int64_t issued = 0;
            for (int64_t r = blockIdx.x; r < p.rows && !failed; r += gridDim.x) {
                const Row<T> row(logits + r * p.ld, p.vocab);
                for (int from = 0; from < row.chunks; from += kPieceChunks) {
                    if (use && !wait_limited(tc::smem_u32(&empty[slot]), (uint32_t)(use - 1) & 1u, &failed)) { count_timeout(&timeouts); break; }
                    const uint32_t bytes = 16u * (uint32_t)min(kPieceChunks, row.chunks - from), bar = tc::smem_u32(&full[slot]);
                    tc::mbar_expect_tx(bar, bytes);
                    tc::bulk_g2s(tc::smem_u32(pieces + slot * kPieceBytes), reinterpret_cast<const uint8_t *>(row.body()) + 16 * (int64_t)from, bytes, bar);
                    ++issued;
                    if (++slot == kPieces) { slot = 0; ++use; }
                }
            }
            // after a failure copies may still be under way
            if (failed)
                for (int64_t i = issued > kPieces ? issued - kPieces : 0; i < issued; ++i) {
                    int again = 0;
                    wait_limited(tc::smem_u32(&full[i % kPieces]), (uint32_t)(i / kPieces) & 1u, &again);
                }
        }
        return;
    }
    const Team team{(int)threadIdx.x, kStreamThreads, 1};
    const int t = team.t, k = max(p.top, p.votes ? 1 : 0);
    const float c = p.scale2;
    for (int64_t r = blockIdx.x; r < p.rows; r += gridDim.x) {
        const Row<T> row(logits + r * p.ld, p.vocab);
        const int edge_index = t < 32 ? row.edge(t) : -1;
        const float edge = edge_index >= 0 ? to_float(row.at[edge_index]) : -INFINITY;
        const Given given = given_of(p, row.at, r, t == 0);
        Own<false> own;
        // two subsets a thread: what is read again for the alternatives is half.  Their keys wait where the candidates will be: there
        // are no registers for them
        const int n_pieces = (row.chunks + kPieceChunks - 1) / kPieceChunks, per_subset = (n_pieces + kStreamSubsets - 1) / kStreamSubsets, each = per_subset * (kPieceChunks / kStreamThreads);
        int left_in_subset = per_subset, at_subset = t;
        sh.candidate[t + kStreamThreads] = 0;
        for (int from = 0; from < row.chunks; from += kPieceChunks) {
            if (!wait_limited(tc::smem_u32(&full[slot]), (uint32_t)use & 1u, &failed)) { count_timeout(&timeouts); own.seen = NAN; }
            const int left = row.chunks - from - t;
            // (int8: one chunk has 16 logits, and there are no registers for more)
            constexpr int kN = kPieceChunks / kStreamThreads, kTogether = sizeof(T) == 1 ? 1 : kN;
#pragma unroll 1
            for (int i0 = 0; i0 < kN; i0 += kTogether) {
                Chunk<T> e[kTogether];
#pragma unroll
                for (int i = 0; i < kTogether; ++i) e[i] = *reinterpret_cast<const Chunk<T> *>(pieces + slot * kPieceBytes + 16 * ((i0 + i) * kStreamThreads + t));
                const int here = left - i0 * kStreamThreads;
                if (here > (kTogether - 1) * kStreamThreads) own.add(e, kTogether, from + i0 * kStreamThreads + t, kStreamThreads, c, p.least, p.limit);
                else if (here > 0) own.add(e, (here + kStreamThreads - 1) / kStreamThreads, from + i0 * kStreamThreads + t, kStreamThreads, c, p.least, p.limit);
            }
            __syncwarp();
            if ((t & 31) == 0) tc::mbar_arrive(tc::smem_u32(&empty[slot]));
            if (++slot == kPieces) { slot = 0; ++use; }
            if (--left_in_subset == 0 || from + kPieceChunks >= row.chunks) {
                sh.candidate[at_subset] = own.subset();
                at_subset += kStreamThreads;
                left_in_subset = per_subset;
            }
        }
        bool bad;
        const Sums all = join_all(sh, team, own, edge, c, bad);
        if (k) {
            const Key key[kStreamSubsets] = {sh.candidate[t], sh.candidate[t + kStreamThreads]};
            team_top<T>(sh, team, row, key, edge, edge_index, t, kStreamThreads, each, k);
        }
        write_results(p, sh, given, r, all, bad, t);
        team.sync();
    }
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
        const Given given = given_of(p, row, row_index, mine && lane == 0);
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
                const float z = fmaxf(times_difference<true>(x[e], m, c), kFloorZ), ez = exp2_fast(z);
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
        if (mine && lane == 0) write_row(p, r, given, row_index);
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

// The range of largest logits for the short way: single precision holds all differences, and (kMasked - m) c, the exponent that a
// mask gets there, is kFloorZ at most, so that its exponential is zero.  bf16's and fp32's kMasked is out of reach down to factors of
// 1e-28, but fp16's is near: m has to be above -65,400 at a factor of 1, and no m around zero is far enough below one of 0.0016.  Chunks
// without masks go the short way there too (4,096 x 131,072 fp16 at 0.001: 262 us, at 1 248; with masks 518).  int8 has no masks.
template <typename T> void set_range(LogProbParams &p)
{
    p.limit = p.scale2 < 1e8f ? 1e29f : -1e29f;
    p.least = -1e29f;
    if (sizeof(T) > 1) p.least = std::max(p.least, (float)std::min((double)Finite<T>::kMasked - (double)kFloorZ / (double)p.scale2, 3e38));
}

template <typename T> cudaError_t launch_log_probs(const Device &dev, LogProbParams p, cudaStream_t st)
{
    set_range<T>(p);
    if (p.vocab <= 64) {
        const int lanes = p.vocab <= 16 ? 1 : 8;
        const int64_t per_block = kGroupThreads / lanes;
        const unsigned grid = (unsigned)std::min<int64_t>((p.rows + per_block - 1) / per_block, 8 * dev.n_sms);
        if (lanes == 1) k_log_probs_group<T, 1, 16><<<grid, kGroupThreads, 0, st>>>(p);
        else k_log_probs_group<T, 8, 8><<<grid, kGroupThreads, 0, st>>>(p);
        return cudaGetLastError();
    }
    // Factors so small that logits further apart than single precision's range weigh something: one form for all rows, with the arithmetic for
    // that, so that the others need none (in them it cost 2 % of a long row).  fp16 and int8 have no such logits.
    const bool far = p.scale2 < kTinyFactor && (std::is_same<T, float>::value || std::is_same<T, __nv_bfloat16>::value);
    // (a warp takes 16 chunks a lane in the time that a block's barriers take)
    if (!far && (p.vocab <= 4096 || (p.vocab <= 16384 && p.rows >= 16 * dev.n_sms))) {
        k_log_probs_warp<T><<<(unsigned)((p.rows + kRowWarps - 1) / kRowWarps), 32 * kRowWarps, 0, st>>>(p);
        return cudaGetLastError();
    }
    if (!far && p.rows >= 2 * kStreamBlocks * dev.n_sms) {
        const cudaError_t e = cudaFuncSetAttribute(k_log_probs_stream<T>, cudaFuncAttributeMaxDynamicSharedMemorySize, kPieces * kPieceBytes);
        if (e != cudaSuccess) return e;
        k_log_probs_stream<T><<<(unsigned)(kStreamBlocks * dev.n_sms), kStreamThreads + 32, kPieces * kPieceBytes, st>>>(p);
        return cudaGetLastError();
    }
    const int chunks = (int)(p.vocab * (int64_t)sizeof(T) / 16);
    // (more rows than SMs: smaller blocks, so that all are at work at once)
    const int threads = chunks >= 4 * kThreads && p.rows <= dev.n_sms ? kThreads : chunks >= 2 * kThreads ? kThreads / 2 : kThreads / 4;
    p.cluster = 1;
    while (p.cluster < kMostCluster && p.rows * p.cluster * 2 <= 4 * dev.n_sms && chunks >= 4 * threads * p.cluster) p.cluster *= 2;
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
    if constexpr (std::is_same<T, float>::value || std::is_same<T, __nv_bfloat16>::value)
        if (far) return cudaLaunchKernelEx(&cfg, k_log_probs<T, true>, p);
    return cudaLaunchKernelEx(&cfg, k_log_probs<T, false>, p);
}

}  // namespace

namespace ops {
cudaError_t log_probs_timeouts(cudaStream_t st, uint32_t *count) { return read_timeouts(timeouts, st, count); }
}  // namespace ops
}  // namespace isc

extern "C" int isc_log_probs(const void *logits, int64_t ld, int type, int64_t rows, int64_t vocab, float scale, const int64_t *targets, int top,
                             float *out_log_probs, float *out_entropy, int32_t *out_top_ids, float *out_top_log_probs, int32_t *votes, void *cuda_stream)
{
    using namespace isc;
    using namespace isc::ops;
    if (rows < 0 || vocab < 1 || (!is_float_type(type) && type != ISC_I8) || !(scale > 0.0f) || scale > 1e38f || top < 0 || top > kMostTop) return ISC_ERR_ARG;
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
