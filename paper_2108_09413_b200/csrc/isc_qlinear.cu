// Rows of int8 times an int8 matrix on the tensor cores, beside the low-rank adapters of many requests (isc_quant_linear).
//
//   y_tn = s_t (u_n sum_k x_tk W_nk + c_a sum_r B_anr sum_k A_ark x_tk) + bias_n,   a = id_t
//
// Two kernels.  k_adapter_rows computes the inner sums of the rows that have an adapter; k_quant_linear streams W through
// tcgen05 kind::i8 and adds the outer product in its epilogue, so y is written once.  The second starts while the first runs
// (programmatic launch) and waits for it only before its first epilogue.
//
// k_quant_linear.  The matrix is the MMA's M side (128 outputs), rows are its N side (16 to 256 rows, whatever divides them
// best), so a call of one row pays for 16 columns of the tensor core and not for 128.  Operands come by tensor copies of 128 bytes of k
// (128-byte swizzle; outside the matrices zeros).  One warp copies, one issues, eight requantise; accumulators
// alternate between two ranges of tensor memory, so one tile's epilogue runs under the next one's products.  Where there are
// fewer tiles than SMs, a cluster of up to eight blocks shares a tile: each takes a part of k, leaves its int32 sums
// in shared memory and finishes its share of the tile from all of them; integers add up exactly in any order.
//
// Forms.  k_quant_linear<kTiles>: persistent blocks with tile after tile.  <kPart>: a tile for a block or a cluster, narrow ones (few rows) two
// to an SM.  k_quant_linear_one: a single row, without the tensor cores.  plan() chooses by a count of cycles.
//
// The adapters' outer product, in single precision by two-number FMAs.  kTiles: on the accumulators' fragments, as tensor memory gives
// them: a thread has 4 outputs x 4 rows, so an inner sum that it loads serves four products, a value of B another four.  The tile's
// inner sums and its adapter's B lie in shared memory (with 200 KB of it in use the first-level cache is next to
// nothing, and what a step loads from memory it waits for); a row that does not share its neighbours' adapter loads its own.
// kPart, whose rows may each have another adapter: groups of lanes share an output's ranks, straight from memory, while W is on its way.
//
// Measured (us; rank 0 is without adapters): 8,192 rows, k = n = 4,096: rank 0 100, 16 133, 32 159, 64 254; k = n = 8,192, rank 32: 502 (410 without: 2.68
// POP/s, the rate that the card's power lets cuBLAS's bf16 sustain, twice over); 64 rows, k = 4,096, n = 12,288, 32 adapters of rank 16: 27 (17 without).
// What bounds it: few rows the copies' start and end around W's bytes; many, the tensor pipe, and from rank 32 on the
// epilogue's FMAs beside it.
//
// Two other ways were measured.  mma.sync in the epilogue: beside tcgen05 products that keep the tensor pipe busy each one waits for
// hundreds of cycles (k = n = 8,192, rank 32: 604 us).  tcgen05 kind::f16 into a third accumulator, inner sums as sums of bf16 numbers,
// operands written by helper warps: tensor memory then has room for tiles of 160 rows only, and those alone cost more than the
// FMAs (k = n = 4,096: rank 0 177, 16 212, 32 242, 64 317 us).
#include <cuda.h>
#include <cuda_runtime.h>
#include <math.h>
#include <stdint.h>

#include <algorithm>

#include "isc_conv.cuh"
#include "isc_ops.cuh"
#include "isc_ops.h"

namespace isc {
namespace {

using namespace ops;
using namespace tc;

__device__ uint32_t timeouts;            // bounded waits that have run out

constexpr int kTileM = 128, kBlockK = 128;
constexpr int kEpilogueWarps = 8, kThreads = 32 * (2 + kEpilogueWarps);
constexpr int kMostStages = 12, kMostTileN = 256, kMostSplit = 8;
constexpr uint32_t kRingBytes = 192 * 1024, kRingBytesNarrow = 72 * 1024;
constexpr uint32_t kStageRow = 80, kStageRowWide = 144;      // bytes from row to row of a warp's output staging (16-bit, 32-bit)
constexpr uint32_t kStaging = 8 * kStageRowWide;
constexpr size_t kSmemBeside = kEpilogueWarps * kStaging + 1024;       // beside the stages
constexpr int kOuterAhead = 4;          // of a warp's items, whose outer products are computed ahead (kPart)
constexpr size_t kSmemMost = 231936;
// A tile's inner sums, and its adapter's B, in shared memory: bytes from row to row and from output to output, so that the four rows and the
// eight outputs that a warp reads at once lie in different banks.
__host__ __device__ constexpr uint32_t inner_pitch(int ranks) { return (uint32_t)ranks * 4u + 16u; }
__host__ __device__ constexpr uint32_t left_pitch(int ranks) { return (uint32_t)ranks * 2u + 8u; }
constexpr size_t adapter_bytes(int ranks, int width) { return ranks ? width * inner_pitch(ranks) + kTileM * left_pitch(ranks) : 0; }
// the widest tile that leaves them room beside three stages
constexpr int widest_tile(int ranks)
{
    int width = kMostTileN;
    while (width > 16 && (size_t)(3 * (kTileM + width) * kBlockK) + kSmemBeside + adapter_bytes(ranks, width) > kSmemMost) width -= 16;
    return width;
}

enum Form { kTiles, kPart };

struct LinearParams {
    CUtensorMap map_w, map_x;
    Form form;
    const float *x_scale, *w_scale, *bias;
    const void *b;                      // adapters: [adapter][n][rank]
    const int32_t *ids;
    const float *inner;                 // [row][ranks]: inner sums times the adapter's scale, zeros behind its rank
    void *y;
    int64_t ldy;
    int rows, n, k_blocks, rank, ranks, n_adapters, y_type;    // ranks: rank in whole sixteens
    int tile_n, tiles_m, tiles_n, split, stages;
    uint32_t ring_bytes, acc_stride;    // shared memory of the stages; tensor-memory columns of an accumulator
    bool vec_y;
};

struct OneParams {
    const int8_t *x, *w;
    const float *x_scale, *w_scale, *bias, *inner;
    const void *b;
    const int32_t *ids;
    void *y;
    int64_t ldw;
    int n, k, rank, n_adapters, y_type;
};

__device__ __forceinline__ void copy_tile(uint32_t dst, const CUtensorMap *map, int x, int y, uint32_t bar)
{
    asm volatile("cp.async.bulk.tensor.2d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];"
                 ::"r"(dst), "l"(reinterpret_cast<uint64_t>(map)), "r"(x), "r"(y), "r"(bar) : "memory");
}
// K-major operand of 128-byte rows, swizzled over 128 bytes, 1024 bytes from one group of eight rows to the next
__device__ __forceinline__ uint64_t operand(uint32_t addr)
{
    return (uint64_t)((addr & 0x3FFFFu) >> 4) | (uint64_t)1 << 16 | (uint64_t)(1024 >> 4) << 32 | (uint64_t)1 << 46 | (uint64_t)2 << 61;
}
template <bool kHalf> __device__ __forceinline__ void mma16(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1)
{
    if (kHalf)
        asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
    else
        asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
            : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ void cluster_sync()
{
    __syncwarp();
    asm volatile("barrier.cluster.arrive.release.aligned;\n\tbarrier.cluster.wait.acquire.aligned;" ::: "memory");
}
__device__ __forceinline__ uint32_t in_block(uint32_t addr, int rank)
{
    uint32_t a;
    asm("mapa.shared::cluster.u32 %0, %1, %2;" : "=r"(a) : "r"(addr), "r"(rank));
    return a;
}
__device__ __forceinline__ int4 read_remote_v4(uint32_t addr)
{
    int4 v;
    asm volatile("ld.shared::cluster.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(v.x), "=r"(v.y), "=r"(v.z), "=r"(v.w) : "r"(addr) : "memory");
    return v;
}
__device__ __forceinline__ int read_remote(uint32_t addr)
{
    int v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(addr) : "memory");
    return v;
}

// the epilogue's warps
__device__ __forceinline__ void epilogue_sync()
{
    __syncwarp();
    asm volatile("barrier.cta.sync.aligned 1, %0;" ::"n"(32 * kEpilogueWarps) : "memory");
}

// What a warp's lane needs for its four outputs of a 32-output strip: fragment rows lane / 4 + 8 i.
struct Strip {
    int n0;
    float w_scale[4], bias[4];
    __device__ __forceinline__ void load(const LinearParams &p, int first, int lane)
    {
        n0 = first;
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            const int n = first + (lane >> 2) + 8 * i;
            w_scale[i] = n < p.n ? __ldg(p.w_scale + n) : 0.0f;
            bias[i] = p.bias && n < p.n ? __ldg(p.bias + n) : 0.0f;
        }
    }
};

// 16 rows as a lane of an epilogue warp meets them: it has rows row0 + 8 e + 2 (lane mod 4) + j.
struct Rows {
    int id[2][2];
    float scale[2][2];
    template <bool kAdapters> __device__ __forceinline__ void load(const LinearParams &p, int row0, int lane)
    {
#pragma unroll
        for (int e = 0; e < 2; ++e)
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                const int row = row0 + 8 * e + 2 * (lane & 3) + j;
                id[e][j] = kAdapters && row < p.rows ? __ldg(p.ids + row) : -1;
                const float s = row < p.rows ? __ldg(p.x_scale + row) : 0.0f;
                scale[e][j] = kAdapters && id[e][j] >= p.n_adapters ? NAN : s;
            }
    }
};

// Sixteen ranks of B for a lane's four outputs (lane / 4 + 8 i of a strip), as they lie in memory.
struct Left {
    uint2 v[4][4];
    __device__ __forceinline__ void load(const LinearParams &p, int a, int n0, int block, int lane)
    {
        const uint16_t *b = static_cast<const uint16_t *>(p.b) + ((int64_t)a * p.n + n0 + (lane >> 2)) * p.rank + 16 * block;
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int q = 0; q < 4; ++q)
                v[i][q] = 16 * block + 4 * q < p.rank && n0 + (lane >> 2) + 8 * i < p.n ? __ldg(reinterpret_cast<const uint2 *>(b + (int64_t)8 * i * p.rank + 4 * q)) : make_uint2(0, 0);
    }
};
__device__ __forceinline__ void load_kept(Left &left, const uint8_t *kept, uint32_t pitch, int block, int lane)
{
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int q = 0; q < 4; ++q) left.v[i][q] = *reinterpret_cast<const uint2 *>(kept + (uint32_t)((lane >> 2) + 8 * i) * pitch + (uint32_t)(32 * block + 8 * q));
}
template <bool kHalf> __device__ __forceinline__ Pair widen_pair(uint32_t w)
{
    if (kHalf) {
        const float2 f = __half22float2(*reinterpret_cast<const __half2 *>(&w));
        return make_pair(f.x, f.y);
    }
    return make_pair(__uint_as_float(w << 16), __uint_as_float(w & 0xFFFF0000u));
}

// Sums of products over ranks, even and odd ones apart.
struct Outer {
    Pair v[4][2][2];
    __device__ __forceinline__ void clear()
    {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int e = 0; e < 2; ++e) v[i][e][0] = v[i][e][1] = 0;
    }
    // sixteen ranks of all rows (kOne < 0) or of row kOne alone; inner(e, j, q): four inner sums of a row
    template <bool kHalf, int kOne, typename Inner> __device__ __forceinline__ void add(const Left &left, Inner inner)
    {
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            Pair b[4][2];
#pragma unroll
            for (int i = 0; i < 4; ++i) { b[i][0] = widen_pair<kHalf>(left.v[i][q].x); b[i][1] = widen_pair<kHalf>(left.v[i][q].y); }
#pragma unroll
            for (int e = 0; e < 2; ++e)
#pragma unroll
                for (int j = 0; j < 2; ++j) {
                    if (kOne >= 0 && kOne != 2 * e + j) continue;
                    const float4 in = inner(e, j, q);
                    const Pair lo = make_pair(in.x, in.y), hi = make_pair(in.z, in.w);
#pragma unroll
                    for (int i = 0; i < 4; ++i) v[i][e][j] = fma2(b[i][1], hi, fma2(b[i][0], lo, v[i][e][j]));
                }
        }
    }
    __device__ __forceinline__ float sum(int i, int e, int j) const
    {
        float a, b;
        split(v[i][e][j], a, b);
        return a + b;
    }
};

// one row of several in a strip: its own adapter's ranks
template <bool kHalf, int kOne, typename Inner> __device__ __forceinline__ void add_own(const LinearParams &p, const Rows &rows, int n0, int block, int lane, Inner inner, Outer &outer)
{
    const int a = rows.id[kOne >> 1][kOne & 1];
    if ((unsigned)a >= (unsigned)p.n_adapters) return;
    Left left;
    left.load(p, a, n0, block, lane);
    outer.template add<kHalf, kOne>(left, inner);
}
template <bool kHalf, typename Inner> __device__ __forceinline__ void add_each(const LinearParams &p, const Rows &rows, int n0, int block, int lane, Inner inner, Outer &outer)
{
    add_own<kHalf, 0>(p, rows, n0, block, lane, inner, outer);
    add_own<kHalf, 1>(p, rows, n0, block, lane, inner, outer);
    add_own<kHalf, 2>(p, rows, n0, block, lane, inner, outer);
    add_own<kHalf, 3>(p, rows, n0, block, lane, inner, outer);
}

// Results of 32 outputs x 8 rows (f: outputs lane / 4 + 8 i, rows row0 + 2 (lane mod 4) + j) to y.  `staging`: this warp's.
__device__ __forceinline__ void store_rows(const LinearParams &p, const Strip &s, int row0, int lane, const float (&f)[4][2], uint32_t staging)
{
    const int c = lane & 3;
    const int row = row0 + (lane >> 2);
    __syncwarp();                       // the strip before has been read
    if (p.y_type != ISC_F32) {
        uint32_t v[4];
#pragma unroll
        for (int i = 0; i < 4; ++i) {
            if (p.y_type == ISC_BF16) { const __nv_bfloat162 t = __floats2bfloat162_rn(f[i][0], f[i][1]); v[i] = *reinterpret_cast<const uint32_t *>(&t); }
            else { const __half2 t = __floats2half2_rn(f[i][0], f[i][1]); v[i] = *reinterpret_cast<const uint32_t *>(&t); }
        }
        // four 8 x 8 matrices, transposed: a row of y holds its 32 outputs side by side
        asm volatile("stmatrix.sync.aligned.m8n8.x4.trans.shared.b16 [%0], {%1,%2,%3,%4};"
                     ::"r"(staging + (uint32_t)(lane & 7) * kStageRow + (uint32_t)(lane >> 3) * 16u), "r"(v[0]), "r"(v[1]), "r"(v[2]), "r"(v[3]) : "memory");
        __syncwarp();
        if (p.vec_y && s.n0 + 32 <= p.n) {
            const uint4 out = ld_shared_v4(staging + (uint32_t)(lane >> 2) * kStageRow + (uint32_t)c * 16u);
            if (row < p.rows) *reinterpret_cast<uint4 *>(static_cast<uint16_t *>(p.y) + (int64_t)row * p.ldy + s.n0 + 8 * c) = out;
        } else {
            // a lane for an output: adjacent bytes all the same
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                uint16_t v;
                asm volatile("ld.shared.u16 %0, [%1];" : "=h"(v) : "r"(staging + (uint32_t)r * kStageRow + (uint32_t)lane * 2u));
                if (row0 + r < p.rows && s.n0 + lane < p.n) static_cast<uint16_t *>(p.y)[(int64_t)(row0 + r) * p.ldy + s.n0 + lane] = v;
            }
        }
    } else {
#pragma unroll
        for (int i = 0; i < 4; ++i)
#pragma unroll
            for (int j = 0; j < 2; ++j)
                asm volatile("st.shared.f32 [%0], %1;" ::"r"(staging + (uint32_t)(2 * c + j) * kStageRowWide + (uint32_t)((lane >> 2) + 8 * i) * 4u), "f"(f[i][j]) : "memory");
        __syncwarp();
        if (p.vec_y && s.n0 + 32 <= p.n) {
#pragma unroll
            for (int e = 0; e < 2; ++e) {
                const uint4 out = ld_shared_v4(staging + (uint32_t)(lane >> 2) * kStageRowWide + (uint32_t)(c + 4 * e) * 16u);
                if (row < p.rows) *reinterpret_cast<uint4 *>(static_cast<uint32_t *>(p.y) + (int64_t)row * p.ldy + s.n0 + 4 * c + 16 * e) = out;
            }
        } else {
#pragma unroll
            for (int r = 0; r < 8; ++r) {
                const uint32_t v = lds32(staging + (uint32_t)r * kStageRowWide + (uint32_t)lane * 4u);
                if (row0 + r < p.rows && s.n0 + lane < p.n) static_cast<uint32_t *>(p.y)[(int64_t)(row0 + r) * p.ldy + s.n0 + lane] = v;
            }
        }
    }
}

// The sums' scales, the adapters' part and the offset.  acc: fragments of 16 outputs each, e: which eight rows.
template <bool kAdapters> __device__ __forceinline__ void finish(const LinearParams &p, const Strip &s, const Rows &rows, const Outer &outer, int row0, int e, int lane,
                                                                const int (&acc)[2][4], uint32_t staging)
{
    float f[4][2];
#pragma unroll
    for (int i = 0; i < 4; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
            const float sum = (float)acc[i >> 1][2 * (i & 1) + j];
            const float v = kAdapters ? fmaf(s.w_scale[i], sum, outer.sum(i, e, j)) : s.w_scale[i] * sum;
            f[i][j] = fmaf(v, rows.scale[e][j], s.bias[i]);
        }
    store_rows(p, s, row0 + 8 * e, lane, f, staging);
}

// One row's outer product with 32 outputs of its adapter: kLanes lanes share an output's ranks, eight each, so that a load covers 512
// adjacent bytes of B; their sums are joined while they are dealt out, which leaves each lane with one output, output_of(lane).
template <int kLanes> __device__ __forceinline__ int output_of(int lane) { return (lane & (kLanes - 1)) * (32 / kLanes) + lane / kLanes; }
template <bool kHalf, int kLanes> __device__ __forceinline__ float outer_of(const LinearParams &p, int a, int row, int n0, int lane)
{
    const int rank0 = 8 * (lane & (kLanes - 1)), n = n0 + lane / kLanes;
    const bool there = rank0 < p.rank, second = rank0 + 4 < p.rank;
    const uint16_t *b = static_cast<const uint16_t *>(p.b) + ((int64_t)a * p.n + n) * p.rank + rank0;
    const float4 *in = reinterpret_cast<const float4 *>(p.inner + (int64_t)row * p.ranks + rank0);
    const float4 zero = make_float4(0.0f, 0.0f, 0.0f, 0.0f), s0 = there ? __ldcg(in) : zero, s1 = there ? __ldcg(in + 1) : zero;
    const Pair in2[4] = {make_pair(s0.x, s0.y), make_pair(s0.z, s0.w), make_pair(s1.x, s1.y), make_pair(s1.z, s1.w)};
    float v[kLanes];
    constexpr int kBatch = kLanes < 8 ? kLanes : 8, kStep = 32 / kLanes;
#pragma unroll
    for (int first = 0; first < kLanes; first += kBatch) {
        uint2 w[kBatch][2];
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const bool mine = there && n + (first + i) * kStep < p.n;
            const uint16_t *from = b + (int64_t)(first + i) * kStep * p.rank;
            if (p.rank % 8 == 0) {
                const uint4 q = mine ? __ldg(reinterpret_cast<const uint4 *>(from)) : make_uint4(0, 0, 0, 0);
                w[i][0] = make_uint2(q.x, q.y);
                w[i][1] = make_uint2(q.z, q.w);
            } else {
                w[i][0] = mine ? __ldg(reinterpret_cast<const uint2 *>(from)) : make_uint2(0, 0);
                w[i][1] = mine && second ? __ldg(reinterpret_cast<const uint2 *>(from + 4)) : make_uint2(0, 0);
            }
        }
#pragma unroll
        for (int i = 0; i < kBatch; ++i) {
            const Pair sum = fma2(widen_pair<kHalf>(w[i][1].y), in2[3], fma2(widen_pair<kHalf>(w[i][1].x), in2[2], fma2(widen_pair<kHalf>(w[i][0].y), in2[1], mul2(widen_pair<kHalf>(w[i][0].x), in2[0]))));
            float x, y;
            split(sum, x, y);
            v[first + i] = x + y;
        }
    }
#pragma unroll
    for (int d = kLanes / 2; d; d >>= 1) {
        const bool upper = lane & d;
#pragma unroll
        for (int i = 0; i < d; ++i) {
            const float give = upper ? v[i] : v[i + d], keep = upper ? v[i + d] : v[i];
            v[i] = keep + __shfl_xor_sync(0xffffffffu, give, d);
        }
    }
    return v[0];
}

// Eight rows' sums of one output from the kSplit blocks that share a tile.
template <int kSplit> __device__ __forceinline__ void gather(uint32_t at, int (&sum)[8], int first = 0)
{
    int4 v[kSplit][2];
#pragma unroll
    for (int b = 0; b < kSplit; ++b) {
        const uint32_t from = in_block(at, first + b);
        v[b][0] = read_remote_v4(from);
        v[b][1] = read_remote_v4(from + 16u);
    }
#pragma unroll
    for (int b = 0; b < kSplit; ++b) {
        sum[0] += v[b][0].x; sum[1] += v[b][0].y; sum[2] += v[b][0].z; sum[3] += v[b][0].w;
        sum[4] += v[b][1].x; sum[5] += v[b][1].y; sum[6] += v[b][1].z; sum[7] += v[b][1].w;
    }
}

// The outer products of 32 outputs x 8 rows, each row with its own adapter, to shared memory ([row][output], single precision).
template <bool kHalf, int kLanes> __device__ __forceinline__ void outer_rows_by(const LinearParams &p, int row0, int n0, int lane, uint32_t to)
{
    const int mine = row0 + (lane & 7), id = mine < p.rows ? __ldg(p.ids + mine) : -1;
    constexpr int kTogether = kLanes < 8 ? 8 / kLanes : 1;       // rows whose operands are loaded together
#pragma unroll 1
    for (int t0 = 0; t0 < 8; t0 += kTogether) {
        float outer[kTogether];
#pragma unroll
        for (int u = 0; u < kTogether; ++u) {
            const int a = __shfl_sync(0xffffffffu, id, t0 + u);
            outer[u] = (unsigned)a < (unsigned)p.n_adapters ? outer_of<kHalf, kLanes>(p, a, row0 + t0 + u, n0, lane) : 0.0f;
        }
#pragma unroll
        for (int u = 0; u < kTogether; ++u)
            asm volatile("st.shared.f32 [%0], %1;" ::"r"(to + (uint32_t)((t0 + u) * 32 + output_of<kLanes>(lane)) * 4u), "f"(outer[u]) : "memory");
    }
    __syncwarp();
}
template <bool kHalf> __device__ __forceinline__ void outer_rows(const LinearParams &p, int row0, int n0, int lane, uint32_t to)
{
    if (p.rank <= 16) outer_rows_by<kHalf, 2>(p, row0, n0, lane, to);
    else if (p.rank <= 32) outer_rows_by<kHalf, 4>(p, row0, n0, lane, to);
    else if (p.rank <= 64) outer_rows_by<kHalf, 8>(p, row0, n0, lane, to);
    else outer_rows_by<kHalf, 16>(p, row0, n0, lane, to);
}

// 32 outputs x 8 rows of a tile whose sums lie in the shared memory of the blocks that share it ([output][row], at `sums`); `outer`: where
// outer_rows has put theirs.  A lane has an output.
template <bool kAdapters> __device__ __forceinline__ void finish_part(const LinearParams &p, int row0, int n0, uint32_t sums, uint32_t outer, int lane, bool failed)
{
    const int n = n0 + lane, mine = row0 + (lane & 7);
    const float w_scale = n < p.n ? __ldg(p.w_scale + n) : 0.0f, bias = p.bias && n < p.n ? __ldg(p.bias + n) : 0.0f;
    const int id = kAdapters && mine < p.rows ? __ldg(p.ids + mine) : -1;
    const float x_scale = failed || (kAdapters && id >= p.n_adapters) ? NAN : mine < p.rows ? __ldg(p.x_scale + mine) : 0.0f;
    int sum[8] = {};
    const uint32_t from = sums + (uint32_t)lane * 32u;
    if (p.split == 1) gather<1>(from, sum);
    else if (p.split == 2) gather<2>(from, sum);
    else if (p.split == 4) gather<4>(from, sum);
    else { gather<4>(from, sum); gather<4>(from, sum, 4); }
#pragma unroll
    for (int t = 0; t < 8; ++t) {
        const float part = kAdapters ? __uint_as_float(lds32(outer + (uint32_t)(t * 32 + lane) * 4u)) : 0.0f;
        const float f = fmaf(fmaf(w_scale, (float)sum[t], part), __shfl_sync(0xffffffffu, x_scale, t), bias);
        if (row0 + t >= p.rows || n >= p.n) continue;
        const int64_t at = (int64_t)(row0 + t) * p.ldy + n;
        if (p.y_type == ISC_F32) static_cast<float *>(p.y)[at] = f;
        else if (p.y_type == ISC_F16) static_cast<__half *>(p.y)[at] = __float2half_rn(f);
        else static_cast<__nv_bfloat16 *>(p.y)[at] = __float2bfloat16_rn(f);
    }
}

// The adapters' operands of a block's first tile into the second-level cache: what a call of few rows otherwise waits for at its end.
// Warp `w` of those of all the blocks that share the tile takes every n-th row.  (64 rows of 16 adapters of rank 64, k = 4,096, n = 12,288:
// 49 us where each block fetches for all of its tile's rows, 45 so.)
__device__ __forceinline__ void prefetch_adapters(const LinearParams &p, int n0, int m0, int w, int lane)
{
    const int bytes = min(kTileM, p.n - m0) * p.rank * 2;
    for (int t0 = 0; t0 < p.tile_n && n0 + t0 < p.rows; t0 += 32) {
        const int id = t0 + lane < p.tile_n && n0 + t0 + lane < p.rows ? __ldg(p.ids + n0 + t0 + lane) : -1, before = __shfl_up_sync(0xffffffffu, id, 1);
        uint32_t fresh = __ballot_sync(0xffffffffu, (unsigned)id < (unsigned)p.n_adapters && (lane == 0 || id != before) && (t0 + lane) % (kEpilogueWarps * p.split) == w);
        while (fresh) {
            const int a = __shfl_sync(0xffffffffu, id, __ffs((int)fresh) - 1);
            fresh &= fresh - 1;
            const char *b = static_cast<const char *>(p.b) + ((int64_t)a * p.n + m0) * p.rank * 2;
            for (int at = 128 * lane; at < bytes; at += 128 * 32) asm volatile("prefetch.global.L2 [%0];" ::"l"(b + at));
        }
    }
}

// kForm kTiles: persistent blocks with tile after tile.  kPart: a tile, or a part of k of one, for a block, two blocks to an SM if
// the tile is narrow.
template <Form kForm, bool kAdapters, bool kHalf> __global__ void __launch_bounds__(kThreads, kForm == kPart ? 2 : 1) k_quant_linear(const __grid_constant__ LinearParams p)
{
    extern __shared__ uint8_t smem_raw[];
    __shared__ __align__(8) uint64_t bar_full[kMostStages], bar_free[kMostStages], bar_acc_full[2], bar_acc_free[2], bar_end;
    __shared__ uint32_t tmem_addr;
    __shared__ int failed;
    const int warp = (int)warp_uniform(threadIdx.x >> 5), lane = threadIdx.x & 31;
    const uint32_t ring = (smem_u32(smem_raw) + 1023u) & ~1023u, staging = ring + p.ring_bytes, outer_at = staging;     // (kPart has no other use for it)
    const uint32_t stage_bytes = (uint32_t)(kTileM + p.tile_n) * kBlockK;
    const int rank = p.split > 1 ? (int)(blockIdx.x % (unsigned)p.split) : 0;
    const int first_tile = (int)(blockIdx.x / (unsigned)p.split), tile_step = (int)(gridDim.x / (unsigned)p.split), tiles = p.tiles_m * p.tiles_n;
    const int kb0 = (int)((int64_t)p.k_blocks * rank / p.split), kb1 = (int)((int64_t)p.k_blocks * (rank + 1) / p.split);
    if (threadIdx.x == 0) {
        for (int s = 0; s < p.stages; ++s) { mbar_init(smem_u32(&bar_full[s]), 1); mbar_init(smem_u32(&bar_free[s]), 1); }
        for (int b = 0; b < 2; ++b) { mbar_init(smem_u32(&bar_acc_full[b]), 1); mbar_init(smem_u32(&bar_acc_free[b]), kEpilogueWarps); }
        mbar_init(smem_u32(&bar_end), 1);
        asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
        failed = 0;
    }
    if (warp == 1) tmem_alloc(smem_u32(&tmem_addr), 2 * p.acc_stride);
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = tmem_addr;

    if (warp == 0) {
        if (lane == 0) {
            int s = 0, use = 0, issued = 0;
            for (int tile = first_tile; tile < tiles && !failed; tile += tile_step) {
                const int m0 = tile % p.tiles_m * kTileM, n0 = tile / p.tiles_m * p.tile_n;
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (use && !wait_limited(smem_u32(&bar_free[s]), (uint32_t)(use - 1) & 1u, &failed)) { count_timeout(&timeouts); break; }
                    const uint32_t bar = smem_u32(&bar_full[s]), at = ring + (uint32_t)s * stage_bytes;
                    mbar_expect_tx(bar, (uint32_t)(kTileM + p.tile_n) * kBlockK);
                    copy_tile(at, &p.map_w, kb * kBlockK, m0, bar);
                    copy_tile(at + kTileM * kBlockK, &p.map_x, kb * kBlockK, n0, bar);
                    ++issued;
                    if (++s == p.stages) { s = 0; ++use; }
                }
            }
            // after a failure copies may still be under way
            if (failed)
                for (int i = max(0, issued - p.stages); i < issued; ++i) {
                    int again = 0;
                    wait_limited(smem_u32(&bar_full[i % p.stages]), (uint32_t)(i / p.stages) & 1u, &again);
                }
        }
        __syncwarp();
    } else if (warp == 1) {
        if (lane == 0) {
            const uint32_t idesc = (2u << 4) | (1u << 7) | (1u << 10) | ((uint32_t)(p.tile_n >> 3) << 17) | ((uint32_t)(kTileM >> 4) << 24);
            int s = 0, use = 0, j = 0;
            for (int tile = first_tile; tile < tiles && !failed; tile += tile_step, ++j) {
                const int buf = j & 1;
                if (j >= 2 && !wait_limited(smem_u32(&bar_acc_free[buf]), (uint32_t)((j >> 1) - 1) & 1u, &failed)) { count_timeout(&timeouts); break; }
                tc_fence_after();
                for (int kb = kb0; kb < kb1; ++kb) {
                    if (!wait_limited(smem_u32(&bar_full[s]), (uint32_t)use & 1u, &failed)) { count_timeout(&timeouts); break; }
                    tc_fence_after();
                    const uint64_t a = operand(ring + (uint32_t)s * stage_bytes), b = operand(ring + (uint32_t)s * stage_bytes + kTileM * kBlockK);
#pragma unroll
                    for (int q = 0; q < kBlockK / 32; ++q) conv::mma_i8(tmem + (uint32_t)buf * p.acc_stride, a + 2 * q, b + 2 * q, idesc, kb > kb0 || q > 0);
                    conv::commit_to(smem_u32(&bar_free[s]));
                    if (++s == p.stages) { s = 0; ++use; }
                }
                if (!failed) conv::commit_to(smem_u32(&bar_acc_full[buf]));
            }
            if (failed) {               // products may still be under way: tensor memory and operands stay until they are done
                int again = 0;
                conv::commit_to(smem_u32(&bar_end));
                wait_limited(smem_u32(&bar_end), 0, &again);
            }
        }
        __syncwarp();
    } else {
        const int w = warp - 2, quarter = warp & 3, half = w >> 2;
        const uint32_t mine = staging + (uint32_t)w * kStaging;
        Strip strip;
        if constexpr (kForm == kPart) {
            // what the end needs: scales, offsets and ids into the second-level cache
            const int n = first_tile % p.tiles_m * kTileM + 32 * w + lane, row = first_tile / p.tiles_m * p.tile_n + 32 * w + lane;
            if (w < 4 && n < p.n) {
                asm volatile("prefetch.global.L2 [%0];" ::"l"(p.w_scale + n));
                if (p.bias) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.bias + n));
            }
            if (32 * w < p.tile_n && row < p.rows) {
                asm volatile("prefetch.global.L2 [%0];" ::"l"(p.x_scale + row));
                if (kAdapters) asm volatile("prefetch.global.L2 [%0];" ::"l"(p.ids + row));
            }
        }
        if (kAdapters && first_tile < tiles) prefetch_adapters(p, first_tile / p.tiles_m * p.tile_n, first_tile % p.tiles_m * kTileM, w + kEpilogueWarps * rank, lane);
        if constexpr (kForm == kTiles) {
            const uint32_t in_pitch = inner_pitch(p.ranks), b_pitch = left_pitch(p.ranks), inner_at = staging + kEpilogueWarps * kStaging, left_at = inner_at + (uint32_t)p.tile_n * in_pitch;
            const uint8_t *const inner_s = smem_raw + (inner_at - smem_u32(smem_raw)), *const left_s = smem_raw + (left_at - smem_u32(smem_raw));
            if (kAdapters) conv::chain_wait();
            int j = 0;
            for (int tile = first_tile; tile < tiles; tile += tile_step, ++j) {
                const int buf = j & 1, m0 = tile % p.tiles_m * kTileM, n0 = tile / p.tiles_m * p.tile_n;
                strip.load(p, m0 + 32 * quarter, lane);
                Rows rows;
                rows.load<kAdapters>(p, n0 + 16 * half, lane);
                int kept = -1;
                if (kAdapters) {
                    // Under the tile's products: all of its rows' inner sums, and B of the adapter that its middle row has
                    const int e = threadIdx.x - 64, words = p.ranks >> 2;
                    kept = __ldg(p.ids + min(n0 + p.tile_n / 2, p.rows - 1));
                    if ((unsigned)kept >= (unsigned)p.n_adapters) kept = -1;
                    epilogue_sync();                    // the tile before has been read
                    for (int i = e; i < p.tile_n * words; i += 32 * kEpilogueWarps) {
                        const int row = i / words, at = i - row * words;
                        conv::cp_async16(inner_at + (uint32_t)row * in_pitch + 16u * (uint32_t)at, p.inner + (int64_t)min(n0 + row, p.rows - 1) * p.ranks + 4 * at);
                    }
                    if (kept >= 0) {
                        const uint16_t *b = static_cast<const uint16_t *>(p.b) + ((int64_t)kept * p.n + m0) * p.rank;
                        for (int i = e; i < kTileM * words; i += 32 * kEpilogueWarps) {
                            const int row = i / words, at = 4 * (i - row * words);
                            const bool there = at < p.rank && m0 + row < p.n;
                            asm volatile("cp.async.ca.shared.global [%0], [%1], 8, %2;"
                                         ::"r"(left_at + (uint32_t)row * b_pitch + 2u * (uint32_t)at), "l"(there ? b + (int64_t)row * p.rank + at : b), "r"(there ? 8 : 0) : "memory");
                        }
                    }
                    conv::cp_async_wait_all();
                    epilogue_sync();
                }
                const bool ok = __all_sync(0xffffffffu, wait_limited(smem_u32(&bar_acc_full[buf]), (uint32_t)(j >> 1) & 1u, &failed)) != 0;
                if (!ok) {              // nothing of the tile can be told
                    count_timeout(&timeouts);
#pragma unroll
                    for (int i = 0; i < 4; ++i) strip.w_scale[i] = strip.bias[i] = NAN;
                }
                tc_fence_after();
                const uint32_t acc = tmem + (uint32_t)buf * p.acc_stride + ((uint32_t)(32 * quarter) << 16);
                for (int q = half; q < p.tile_n / 16; q += 2) {
                    const int row0 = n0 + 16 * q;
                    int v[2][8];
                    tmem_ld_frag(acc + 16u * (uint32_t)q, v[0]);
                    tmem_ld_frag(acc + (16u << 16) + 16u * (uint32_t)q, v[1]);
                    Rows next;
                    next.load<kAdapters>(p, row0 + 32, lane);
                    Outer outer;
                    if (kAdapters) {
                        outer.clear();
                        const int a = rows.id[0][0];
                        const int a0 = __shfl_sync(0xffffffffu, a, 0);
                        const bool same = __all_sync(0xffffffffu, (a == a0) & (a == rows.id[0][1]) & (a == rows.id[1][0]) & (a == rows.id[1][1])) != 0;
                        const uint8_t *from = inner_s + (uint32_t)(16 * q + 2 * (lane & 3)) * in_pitch;
#pragma unroll 1
                        for (int r = 0; r < p.ranks >> 4; ++r, from += 64) {
                            const auto inner = [&](int e, int jj, int quad) { return *reinterpret_cast<const float4 *>(from + (uint32_t)(8 * e + jj) * in_pitch + 16u * (uint32_t)quad); };
                            if (!same) add_each<kHalf>(p, rows, strip.n0, r, lane, inner, outer);
                            else if ((unsigned)a < (unsigned)p.n_adapters) {
                                Left left;
                                if (a == kept) load_kept(left, left_s + (uint32_t)(32 * quarter) * b_pitch, b_pitch, r, lane);
                                else left.load(p, a, strip.n0, r, lane);
                                outer.template add<kHalf, -1>(left, inner);
                            }
                        }
                    }
                    tmem_ld_frag_wait(v[0]);
                    tmem_ld_frag_wait(v[1]);
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const int part[2][4] = {{v[0][4 * e], v[0][4 * e + 1], v[0][4 * e + 2], v[0][4 * e + 3]}, {v[1][4 * e], v[1][4 * e + 1], v[1][4 * e + 2], v[1][4 * e + 3]}};
                        if (row0 + 8 * e < p.rows) finish<kAdapters>(p, strip, rows, outer, row0, e, lane, part, mine);
                    }
                    rows = next;
                }
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(smem_u32(&bar_acc_free[buf]));
            }
        } else {
            if (kAdapters) {
                // the first items' outer products, under W's copies and products: they need the inner sums only
                conv::chain_wait();
                for (int i = 0; i < kOuterAhead; ++i) {
                    const int item = rank + p.split * (w + kEpilogueWarps * i), row0 = first_tile / p.tiles_m * p.tile_n + item % (p.tile_n / 8) * 8, strip_n = first_tile % p.tiles_m * kTileM + 32 * (item / (p.tile_n / 8));
                    if (item < kTileM / 32 * (p.tile_n / 8) && row0 < p.rows && strip_n < p.n) outer_rows<kHalf>(p, row0, strip_n, lane, outer_at + (uint32_t)(w * kOuterAhead + i) * 1024u);
                }
            }
            // this block's sums to its shared memory; its ring is empty: all products are done
            const bool ok = __all_sync(0xffffffffu, wait_limited(smem_u32(&bar_acc_full[0]), 0, &failed)) != 0;
            if (!ok) count_timeout(&timeouts);
            tc_fence_after();
            for (int q = half; q < p.tile_n / 16; q += 2) {
                int v[16];
                tmem_ld16_issue(tmem + ((uint32_t)(32 * quarter) << 16) + 16u * (uint32_t)q, v);
                asm volatile("tcgen05.wait::ld.sync.aligned;" : "+r"(v[0]), "+r"(v[1]), "+r"(v[2]), "+r"(v[3]), "+r"(v[4]), "+r"(v[5]), "+r"(v[6]), "+r"(v[7]),
                             "+r"(v[8]), "+r"(v[9]), "+r"(v[10]), "+r"(v[11]), "+r"(v[12]), "+r"(v[13]), "+r"(v[14]), "+r"(v[15]) :: "memory");
                // [strip][eight rows][output][row]: a lane that finishes eight rows of an output reads two times 16 bytes
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (ok) st_shared_v4(ring + (uint32_t)((quarter * (p.tile_n / 8) + 2 * q + (e >> 1)) * 32 + lane) * 32u + 16u * (uint32_t)(e & 1),
                                         make_uint4((uint32_t)v[4 * e], (uint32_t)v[4 * e + 1], (uint32_t)v[4 * e + 2], (uint32_t)v[4 * e + 3]));
            }
            tc_fence_before();
        }
    }
    if constexpr (kForm == kPart) {
        __syncwarp();
        if (p.split > 1) cluster_sync();
        else __syncthreads();
        if (warp >= 2) {
            const int w = warp - 2, per_quarter = p.tile_n / 8;
            bool bad = false;
            for (int b = 0; b < p.split; ++b) bad |= read_remote(in_block(smem_u32(&failed), b)) != 0;
            int i = 0;
            for (int item = rank + p.split * w; item < kTileM / 32 * per_quarter; item += p.split * kEpilogueWarps, ++i) {
                const int at = item % per_quarter * 8, row0 = first_tile / p.tiles_m * p.tile_n + at, strip = item / per_quarter, n0 = first_tile % p.tiles_m * kTileM + 32 * strip;
                if (row0 >= p.rows || n0 >= p.n) continue;
                const uint32_t outer = outer_at + (uint32_t)(w * kOuterAhead + i % kOuterAhead) * 1024u;
                if (kAdapters && i >= kOuterAhead) outer_rows<kHalf>(p, row0, n0, lane, outer);
                finish_part<kAdapters>(p, row0, n0, ring + (uint32_t)item * 1024u, outer, lane, bad);
            }
        }
        __syncwarp();
        if (p.split > 1) cluster_sync();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    if (warp == 1) tmem_dealloc(tmem, 2 * p.acc_stride);
}

// sixteen codes of a row, zeros behind its end (which is read no further: it may be the tensor's)
__device__ __forceinline__ uint4 load_codes(const int8_t *at, int left)
{
    if (left >= 16) return __ldg(reinterpret_cast<const uint4 *>(at));
    uint32_t w[4] = {0, 0, 0, 0};
#pragma unroll
    for (int e = 0; e < 16; ++e)
        if (e < left) w[e >> 2] |= (uint32_t)(uint8_t)at[e] << 8 * (e & 3);
    return make_uint4(w[0], w[1], w[2], w[3]);
}

// ---- one row: W's rows straight into registers

// A warp for an output, products by dp4a.  A tile of the tensor cores' form costs a fixed time (tensor memory, descriptors, barriers, a
// cluster's join) that a call of one row does not get back, and reads W in pieces of 128 bytes; here a warp has 4 KB of a row of W under way
// at once.  Bound by W's bytes: k = 8,192, n = 28,672 in 41 us, 5.8 TB/s; k = n = 4,096 in 6.4 us against 9.9 with tiles.
// (dp4a is slow here, about eleven a clock and SM: two rows took 16.5 us where tiles take 10.)
constexpr int kOneThreads = 256;
template <bool kHalf> __global__ void __launch_bounds__(kOneThreads) k_quant_linear_one(const __grid_constant__ OneParams p)
{
    const int lane = threadIdx.x & 31, n = (int)(blockIdx.x * (unsigned)(kOneThreads / 32) + (threadIdx.x >> 5));
    if (n >= p.n) return;
    // what the end needs, ahead of the products; the adapter's share of this output: the first 32 ranks, a rank to a lane
    const float w_scale = __ldg(p.w_scale + n), x_scale = __ldg(p.x_scale), bias = p.bias ? __ldg(p.bias + n) : 0.0f;
    const int id = p.rank ? __ldg(p.ids) : -1;
    const bool adapted = (unsigned)id < (unsigned)p.n_adapters;
    const uint16_t *b = static_cast<const uint16_t *>(p.b) + ((int64_t)id * p.n + n) * p.rank;
    const uint32_t b_first = adapted && lane < p.rank ? __ldg(b + lane) : 0u;
    const int8_t *w = p.w + (int64_t)n * p.ldw;
    int sum = 0;
    constexpr int kAhead = 8;
    for (int k0 = 16 * lane; k0 < p.k; k0 += 512 * kAhead) {
        uint4 v[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u) v[u] = load_codes(w + k0 + 512 * u, p.k - k0 - 512 * u);
#pragma unroll
        for (int u = 0; u < kAhead; ++u) {
            const uint4 x = load_codes(p.x + k0 + 512 * u, p.k - k0 - 512 * u);
            sum = __dp4a((int)x.x, (int)v[u].x, sum);
            sum = __dp4a((int)x.y, (int)v[u].y, sum);
            sum = __dp4a((int)x.z, (int)v[u].z, sum);
            sum = __dp4a((int)x.w, (int)v[u].w, sum);
        }
    }
    sum = __reduce_add_sync(0xffffffffu, sum);
    float outer = 0.0f;
    if (p.rank) {
        conv::chain_wait();
        if (adapted) {
            for (int r = lane; r < p.rank; r += 32) {
                const uint32_t v = r < 32 ? b_first : __ldg(b + r);
                outer = fmaf(kHalf ? __half2float(__ushort_as_half((unsigned short)v)) : __uint_as_float(v << 16), p.inner[r], outer);
            }
#pragma unroll
            for (int d = 16; d; d >>= 1) outer += __shfl_xor_sync(0xffffffffu, outer, d);
        }
    }
    if (lane) return;
    const float f = p.rank && id >= p.n_adapters ? NAN : fmaf(fmaf(w_scale, (float)sum, outer), x_scale, bias);
    if (p.y_type == ISC_F32) static_cast<float *>(p.y)[n] = f;
    else if (p.y_type == ISC_F16) static_cast<__half *>(p.y)[n] = __float2half_rn(f);
    else static_cast<__nv_bfloat16 *>(p.y)[n] = __float2bfloat16_rn(f);
}

// ---- the adapters' inner sums

struct InnerParams {
    const int8_t *x;
    const void *a;                      // [adapter][rank][k]
    const float *scale;
    const int32_t *ids;
    float *inner;
    int64_t ldx;
    int rows, k, rank, ranks, n_adapters, split;
    bool vec_a;
};

constexpr int kInnerThreads = 256;

// four int8 as four 16-bit numbers, exactly
template <bool kHalf> __device__ __forceinline__ uint2 widen(uint32_t v)
{
    if (kHalf) {
        // 1024 + (v + 128), less 1152
        const uint32_t u = v ^ 0x80808080u, lo = __byte_perm(u, 0x64646464u, 0x4140), hi = __byte_perm(u, 0x64646464u, 0x4342);
        const __half2 off = __halves2half2(__ushort_as_half(0x6480), __ushort_as_half(0x6480));
        const __half2 a = __hsub2(*reinterpret_cast<const __half2 *>(&lo), off), b = __hsub2(*reinterpret_cast<const __half2 *>(&hi), off);
        return make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
    }
    // v = (128 + (v & 127)) - (128 or 256), both of them bf16 numbers whose last bits are v's
    const uint32_t lo = __byte_perm(v, 0x43434343u, 0x4140), hi = __byte_perm(v, 0x43434343u, 0x4342);
    const uint32_t p0 = lo & 0xFF7FFF7Fu, q0 = lo & 0xFF80FF80u, p1 = hi & 0xFF7FFF7Fu, q1 = hi & 0xFF80FF80u;
    const __nv_bfloat162 a = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&p0), *reinterpret_cast<const __nv_bfloat162 *>(&q0)),
                         b = __hsub2(*reinterpret_cast<const __nv_bfloat162 *>(&p1), *reinterpret_cast<const __nv_bfloat162 *>(&q1));
    return make_uint2(*reinterpret_cast<const uint32_t *>(&a), *reinterpret_cast<const uint32_t *>(&b));
}

// kRowBlocks x 8 rows and kRankBlocks x 16 ranks for a block (a cluster where k is split): every warp takes one of the rows' adapters and a
// part of k, ranks on the MMA's M side; the warps' sums meet in shared memory in a fixed order.
template <bool kHalf, int kRowBlocks, int kRankBlocks> __global__ void __launch_bounds__(kInnerThreads) k_adapter_rows(const __grid_constant__ InnerParams p)
{
    constexpr int kRows = 8 * kRowBlocks, kWarps = kInnerThreads / 32, kRanks = 16 * kRankBlocks;
    __shared__ float4 sums[kWarps][kRankBlocks * kRowBlocks][32];
    __shared__ float total[kRows][kRanks];
    __shared__ int ids[kRows], slot_of[kRows], adapter[kRows], n_distinct;
    conv::chain_start();
    const int t = threadIdx.x, warp = t >> 5, lane = t & 31, g = lane >> 2, c = lane & 3;
    const int part = p.split > 1 ? (int)(blockIdx.x % (unsigned)p.split) : 0, row0 = (int)(blockIdx.x / (unsigned)p.split) * kRows, rank0 = blockIdx.y * kRanks;
    if (warp == 0) {
        int id = lane < kRows && row0 + lane < p.rows ? p.ids[row0 + lane] : -1;
        if (id >= p.n_adapters) id = -1;
        uint32_t pending = __ballot_sync(0xffffffffu, id >= 0);
        int n = 0, slot = -1;
        while (pending) {
            const int a = __shfl_sync(0xffffffffu, id, __ffs((int)pending) - 1);
            const uint32_t same = __ballot_sync(0xffffffffu, id == a);
            if (id == a) slot = n;
            if (lane == 0) adapter[n] = a;
            pending &= ~same;
            ++n;
        }
        if (lane < kRows) { ids[lane] = id; slot_of[lane] = slot; }
        if (lane == 0) n_distinct = n;
    }
    for (int i = t; i < kRows * kRanks; i += kInnerThreads) total[i / kRanks][i % kRanks] = 0.0f;
    __syncthreads();
    const int distinct = n_distinct;
    const int chunks = (p.k + 63) >> 6, chunk0 = (int)((int64_t)chunks * part / p.split), chunk1 = (int)((int64_t)chunks * (part + 1) / p.split);
    // blocks along z deal the adapters out, two at a time, where there are few rows
    const int at_once = gridDim.z > 1 ? 2 : kWarps;
    for (int first = (int)blockIdx.z * at_once; first < distinct; first += at_once * (int)gridDim.z) {
        const int here = min(distinct - first, at_once);
        const int width = here > 4 ? 8 : here > 2 ? 4 : here;        // slots; warps w, w + width, ... share one
        const int slot = warp % width, share = warp / width, shares = kWarps / width;
        float acc[kRankBlocks][kRowBlocks][4] = {};
        if (slot < here) {
            const int a = adapter[first + slot];
            const uint16_t *ar[kRankBlocks][2];
#pragma unroll
            for (int r = 0; r < kRankBlocks; ++r)
#pragma unroll
                for (int h = 0; h < 2; ++h) {
                    const int rank = rank0 + 16 * r + 8 * h + g;
                    ar[r][h] = rank < p.rank ? static_cast<const uint16_t *>(p.a) + ((int64_t)a * p.rank + rank) * p.k : nullptr;
                }
            const int lo = chunk0 + (int)((int64_t)(chunk1 - chunk0) * share / shares), hi = chunk0 + (int)((int64_t)(chunk1 - chunk0) * (share + 1) / shares);
            constexpr int kAhead = kRankBlocks * kRowBlocks == 1 ? 4 : 2;
#pragma unroll kAhead
            for (int ch = lo; ch < hi; ++ch) {
                const int k0 = 64 * ch + 16 * c;
                uint4 xv[kRowBlocks];
#pragma unroll
                for (int b = 0; b < kRowBlocks; ++b) {
                    const int row = row0 + 8 * b + g;
                    xv[b] = row < p.rows ? load_codes(p.x + (int64_t)row * p.ldx + k0, p.k - k0) : make_uint4(0, 0, 0, 0);
                }
                uint32_t av[kRankBlocks][2][8];
#pragma unroll
                for (int r = 0; r < kRankBlocks; ++r)
#pragma unroll
                    for (int h = 0; h < 2; ++h) {
                        if (p.vec_a) {
#pragma unroll
                            for (int q = 0; q < 2; ++q) {
                                const uint4 v = ar[r][h] && k0 + 8 * q < p.k ? __ldg(reinterpret_cast<const uint4 *>(ar[r][h] + k0 + 8 * q)) : make_uint4(0, 0, 0, 0);
                                av[r][h][4 * q] = v.x; av[r][h][4 * q + 1] = v.y; av[r][h][4 * q + 2] = v.z; av[r][h][4 * q + 3] = v.w;
                            }
                        } else {
#pragma unroll
                            for (int q = 0; q < 8; ++q) {
                                const uint32_t e0 = ar[r][h] && k0 + 2 * q < p.k ? ar[r][h][k0 + 2 * q] : 0u, e1 = ar[r][h] && k0 + 2 * q + 1 < p.k ? ar[r][h][k0 + 2 * q + 1] : 0u;
                                av[r][h][q] = e0 | e1 << 16;
                            }
                        }
                    }
#pragma unroll
                for (int s = 0; s < 4; ++s)
#pragma unroll
                    for (int b = 0; b < kRowBlocks; ++b) {
                        const uint2 xb = widen<kHalf>(s == 0 ? xv[b].x : s == 1 ? xv[b].y : s == 2 ? xv[b].z : xv[b].w);
#pragma unroll
                        for (int r = 0; r < kRankBlocks; ++r) {
                            const uint32_t left[4] = {av[r][0][2 * s], av[r][1][2 * s], av[r][0][2 * s + 1], av[r][1][2 * s + 1]};
                            mma16<kHalf>(acc[r][b], left, xb.x, xb.y);
                        }
                    }
            }
        }
#pragma unroll
        for (int r = 0; r < kRankBlocks; ++r)
#pragma unroll
            for (int b = 0; b < kRowBlocks; ++b) sums[warp][r * kRowBlocks + b][lane] = make_float4(acc[r][b][0], acc[r][b][1], acc[r][b][2], acc[r][b][3]);
        __syncthreads();
        for (int i = t; i < kRows * kRanks; i += kInnerThreads) {
            const int row = i / kRanks, rank = i % kRanks, s = slot_of[row] - first;
            if (s < 0 || s >= here) continue;
            const int l = (rank & 7) * 4 + ((row & 7) >> 1), e = 2 * ((rank >> 3) & 1) + (row & 1);
            float v = 0.0f;
            for (int w = s; w < kWarps; w += width) v += reinterpret_cast<const float *>(&sums[w][(rank >> 4) * kRowBlocks + (row >> 3)][l])[e];
            total[row][rank] = v;
        }
        __syncthreads();
    }
    if (p.split > 1) cluster_sync();
    if (part == 0) {
        for (int i = t; i < kRows * kRanks; i += kInnerThreads) {
            const int row = i / kRanks, rank = i % kRanks;
            float v = total[row][rank];
            for (int b = 1; b < p.split; ++b) v += __int_as_float(read_remote(in_block(smem_u32(&total[row][rank]), b)));
            const int id = ids[row];
            const bool mine = id >= 0 && slot_of[row] / at_once % (int)gridDim.z == (int)blockIdx.z;
            if (mine && rank0 + rank < p.ranks) p.inner[(int64_t)(row0 + row) * p.ranks + rank0 + rank] = rank0 + rank < p.rank ? v * p.scale[id] : 0.0f;
        }
    }
    if (p.split > 1) cluster_sync();
}

// a row's inner sums, in single precision and whole sixteens of ranks
int64_t work_bytes_of(int64_t rows, int rank) { return (int64_t)((rank + 15) & ~15) * rows * 4; }

typedef CUresult (*EncodeFn)(CUtensorMap *, CUtensorMapDataType, cuuint32_t, void *, const cuuint64_t *, const cuuint64_t *, const cuuint32_t *, const cuuint32_t *, CUtensorMapInterleave,
                             CUtensorMapSwizzle, CUtensorMapL2promotion, CUtensorMapFloatOOBfill);

bool encode_rows(void *encode, CUtensorMap *map, const int8_t *base, int64_t k, int64_t rows, int64_t ld, int box_rows)
{
    const cuuint64_t dims[2] = {(cuuint64_t)k, (cuuint64_t)rows}, strides[1] = {(cuuint64_t)ld};
    const cuuint32_t box[2] = {kBlockK, (cuuint32_t)box_rows}, step[2] = {1, 1};
    return ((EncodeFn)encode)(map, CU_TENSOR_MAP_DATA_TYPE_UINT8, 2, const_cast<int8_t *>(base), dims, strides, box, step, CU_TENSOR_MAP_INTERLEAVE_NONE, CU_TENSOR_MAP_SWIZZLE_128B,
                              CU_TENSOR_MAP_L2_PROMOTION_L2_256B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Row tile, and blocks that share a tile: what takes the fewest cycles by a rough count.  A block of k costs 2.1 cycles for each
// operand row; an epilogue 25 cycles a row and 25 more for every sixteen ranks (50 where the tile is split), under the next tile's
// products where there is one; starting, and joining the blocks that share a tile, a few thousand, and eight of them
// far more the wider the tile (200 rows, k = 4,096, n = 1,024: 9.9 us with four blocks to a tile, 18.6 with eight; 16 rows, k = 8,192: 10.7 and 8.6).
void plan(LinearParams &p, int n_sms)
{
    p.tiles_m = (p.n + kTileM - 1) / kTileM;
    const int most = widest_tile(p.ranks), widest = p.rows <= 1024 ? kMostTileN : most, least = (p.rows + widest - 1) / widest;
    int64_t best = INT64_MAX;
    for (int t = least; t <= std::min(4 * least + 4, least + 64); ++t) {
        const int width = ((p.rows + t - 1) / t + 15) & ~15, tiles_n = (p.rows + width - 1) / width;
        // Narrow tiles are bound by W's bytes: two blocks to an SM, so that one's copies run under the other's start and end (16 rows,
        // k = 8,192, n = 28,672, no adapters: 49 us with one block and 192 KB of stages, 43 us with two of 96 KB; beside adapters they have 72 KB).
        const bool narrow = width <= 64 && tiles_n == 1;
        const int64_t tiles = (int64_t)p.tiles_m * tiles_n, slots = narrow ? 2 * n_sms : n_sms;
        for (int split = 1; split <= kMostSplit && (split == 1 || (tiles * split <= slots && p.k_blocks >= 4 * split)); split *= 2) {
            const bool part = narrow || split > 1;
            if (!part && width > most) continue;
            const int64_t rounds = (tiles * split + slots - 1) / slots;
            const double products = 2.1 * ((p.k_blocks + split - 1) / split) * (width + kTileM), end = (25.0 + (part ? 50.0 : 25.0) * (p.ranks >> 4)) * width / split + (split > 1 ? 4000.0 : 0.0) + (split == 8 ? 100.0 * width : 0.0);
            const int64_t cost = (int64_t)(part ? rounds * (products + end + 3000.0) : rounds * std::max(products, end) + std::min(products, end) + 3000.0);
            if (cost < best) {
                best = cost;
                p.tile_n = width;
                p.tiles_n = tiles_n;
                p.split = split;
                p.form = part ? kPart : kTiles;
                p.ring_bytes = narrow ? (p.ranks ? kRingBytesNarrow : kRingBytesNarrow + 24 * 1024) : part ? kRingBytes : (uint32_t)(kSmemMost - kSmemBeside - adapter_bytes(p.ranks, width)) & ~1023u;
            }
        }
    }
    p.acc_stride = p.tile_n > 128 ? 256 : p.tile_n > 64 ? 128 : 64;
    p.stages = std::min<int>(kMostStages, p.ring_bytes / ((kTileM + p.tile_n) * kBlockK));
}

template <typename P> cudaError_t launch(void (*kernel)(P), const P &p, dim3 grid, int threads, size_t smem, int cluster, bool chained, cudaStream_t st)
{
    cudaLaunchAttribute attr[2];
    int n = 0;
    if (cluster > 1) {
        attr[n].id = cudaLaunchAttributeClusterDimension;
        attr[n].val.clusterDim.x = (unsigned)cluster;
        attr[n].val.clusterDim.y = attr[n].val.clusterDim.z = 1;
        ++n;
    }
    if (chained) {
        attr[n].id = cudaLaunchAttributeProgrammaticStreamSerialization;
        attr[n].val.programmaticStreamSerializationAllowed = 1;
        ++n;
    }
    cudaLaunchConfig_t cfg = {};
    cfg.gridDim = grid;
    cfg.blockDim = dim3((unsigned)threads);
    cfg.dynamicSmemBytes = smem;
    cfg.stream = st;
    cfg.attrs = attr;
    cfg.numAttrs = (unsigned)n;
    return cudaLaunchKernelEx(&cfg, kernel, p);
}

cudaError_t launch_inner(InnerParams p, int type, int n_sms, cudaStream_t st)
{
    const int row_blocks = p.rows >= 1024 ? 4 : 1, rank_blocks = p.rank <= 16 ? 1 : 2;
    const int64_t groups = (p.rows + 8 * row_blocks - 1) / (8 * row_blocks), ranks = (p.rank + 16 * rank_blocks - 1) / (16 * rank_blocks);
    p.split = 1;
    while (p.split < kMostSplit && groups * ranks * p.split * 2 <= 2 * n_sms && p.k >= 64 * 8 * p.split) p.split *= 2;
    void (*const kernels[2][2][2])(InnerParams) = {{{k_adapter_rows<false, 1, 1>, k_adapter_rows<false, 1, 2>}, {k_adapter_rows<false, 4, 1>, k_adapter_rows<false, 4, 2>}},
                                                   {{k_adapter_rows<true, 1, 1>, k_adapter_rows<true, 1, 2>}, {k_adapter_rows<true, 4, 1>, k_adapter_rows<true, 4, 2>}}};
    // (16 rows of 14 adapters of rank 16, k = n = 4,096: 21.3 us for the whole call with a block for all of a group's adapters)
    const unsigned deal = row_blocks == 1 && groups * ranks * p.split * 4 <= 4 * n_sms ? 4 : 1;
    return launch(kernels[type == ISC_F16][row_blocks == 4][rank_blocks == 2], p, dim3((unsigned)(groups * p.split), (unsigned)ranks, deal), kInnerThreads, 0, p.split, false, st);
}

}  // namespace

namespace ops {
cudaError_t linear_timeouts(cudaStream_t st, uint32_t *count) { return read_timeouts(timeouts, st, count); }
}  // namespace ops
}  // namespace isc

extern "C" int isc_quant_linear_work_space(int64_t rows, int rank, int64_t *out_bytes)
{
    if (rows < 0 || rank < 0 || rank > 128 || !out_bytes) return ISC_ERR_ARG;
    if (rows >= INT32_MAX / 2) return ISC_ERR_UNSUPPORTED;
    *out_bytes = isc::work_bytes_of(rows, rank);
    return ISC_OK;
}

extern "C" int isc_quant_linear(const int8_t *x, int64_t ldx, const float *x_scale, int64_t rows, const int8_t *w, int64_t ldw, const float *w_scale, int64_t k, int64_t n, const float *bias,
                                const isc_adapters *adapters, void *y, int64_t ldy, int y_type, void *work, int64_t work_bytes, void *cuda_stream)
{
    using namespace isc;
    using namespace isc::ops;
    if (rows < 0 || k < 1 || n < 1 || !is_float_type(y_type)) return ISC_ERR_ARG;
    if (rows == 0) return ISC_OK;
    if (!x || !x_scale || !w || !w_scale || !y || ldx < k || ldw < k || ldy < n) return ISC_ERR_ARG;
    if (!aligned(x_scale, 4) || !aligned(w_scale, 4) || !aligned(bias, 4) || !aligned(y, type_bytes(y_type))) return ISC_ERR_ARG;
    const isc_adapters *ad = adapters;
    if (ad) {
        if (!ad->a || !ad->b || !ad->scale || !ad->ids || ad->n_adapters < 1 || ad->rank < 1 || (ad->type != ISC_BF16 && ad->type != ISC_F16)) return ISC_ERR_ARG;
        if (!aligned(ad->scale, 4) || !aligned(ad->ids, 4) || !work || !aligned(work, 16)) return ISC_ERR_ARG;
        if (ad->rank % 4 || ad->rank > 128 || !aligned(ad->a, 16) || !aligned(ad->b, 16)) return ISC_ERR_UNSUPPORTED;
        if (rows < INT32_MAX / 2 && work_bytes < isc::work_bytes_of(rows, ad->rank)) return ISC_ERR_ARG;
    }
    // a single row has no pitch
    if (rows == 1) ldx = (k + 15) & ~(int64_t)15;
    if (n == 1) ldw = (k + 15) & ~(int64_t)15;
    // (k: the sums' 32 bits; the rest: 32-bit tile and coordinate arithmetic)
    if (k > 65536 || rows >= INT32_MAX / 2 || n >= INT32_MAX / 2 || !aligned(x, 16) || !aligned(w, 16) || ldx % 16 || ldw % 16) return ISC_ERR_UNSUPPORTED;
    Device dev;
    cudaError_t e = current_device(&dev);
    if (e != cudaSuccess) return status_of(e, "device");
    LinearParams p = {};
    p.x_scale = x_scale; p.w_scale = w_scale; p.bias = bias;
    p.y = y; p.ldy = ldy; p.y_type = y_type;
    p.rows = (int)rows; p.n = (int)n; p.k_blocks = (int)((k + kBlockK - 1) / kBlockK);
    p.vec_y = aligned(y, 16) && ldy * type_bytes(y_type) % 16 == 0;
    const cudaStream_t st = (cudaStream_t)cuda_stream;
    const bool half = ad && ad->type == ISC_F16;
    if (ad) {
        p.b = ad->b; p.ids = ad->ids; p.inner = static_cast<float *>(work);
        p.rank = ad->rank; p.ranks = (ad->rank + 15) & ~15; p.n_adapters = ad->n_adapters;
    }
    if (rows > 1) {                     // (before anything is launched: it may refuse)
        plan(p, dev.n_sms);
        if ((int64_t)p.tiles_m * p.tiles_n > INT32_MAX / kMostSplit) return ISC_ERR_UNSUPPORTED;
    }
    if (ad) {
        InnerParams q = {};
        q.x = x; q.a = ad->a; q.scale = ad->scale; q.ids = ad->ids;
        q.inner = static_cast<float *>(work);
        q.ranks = p.ranks;
        q.ldx = ldx; q.rows = (int)rows; q.k = (int)k; q.rank = ad->rank; q.n_adapters = ad->n_adapters;
        q.vec_a = k % 8 == 0;
        e = launch_inner(q, ad->type, dev.n_sms, st);
        if (e != cudaSuccess) return status_of(e, "quant_linear, inner sums");
    }
    if (rows == 1) {
        const OneParams one = {x, w, x_scale, w_scale, bias, p.inner, p.b, p.ids, y, ldw, p.n, (int)k, p.rank, p.n_adapters, y_type};
        e = launch(half ? k_quant_linear_one<true> : k_quant_linear_one<false>, one, dim3((unsigned)((n + kOneThreads / 32 - 1) / (kOneThreads / 32))), kOneThreads, 0, 1, ad != nullptr, st);
        return status_of(e, "quant_linear");
    }
    if (!dev.encode || !encode_rows(dev.encode, &p.map_w, w, k, n, ldw, kTileM) || !encode_rows(dev.encode, &p.map_x, x, k, rows, ldx, p.tile_n)) return ISC_ERR_CUDA;
    void (*const kernel)(LinearParams) =
        p.form == kPart ? (!ad ? k_quant_linear<kPart, false, false> : half ? k_quant_linear<kPart, true, true> : k_quant_linear<kPart, true, false>) :
        !ad ? k_quant_linear<kTiles, false, false> : half ? k_quant_linear<kTiles, true, true> : k_quant_linear<kTiles, true, false>;
    e = cudaFuncSetAttribute(kernel, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)kSmemMost);
    if (e != cudaSuccess) return status_of(e, "quant_linear");
    const int tiles = p.tiles_m * p.tiles_n;
    const unsigned grid = p.form == kPart ? (unsigned)(tiles * p.split) : (unsigned)std::min(tiles, dev.n_sms);
    e = launch(kernel, p, dim3(grid), kThreads, p.ring_bytes + kSmemBeside + (p.form == kTiles ? adapter_bytes(p.ranks, p.tile_n) : ad ? kEpilogueWarps * (kOuterAhead * 1024 - kStaging) : 0), p.split, ad != nullptr, st);
    return status_of(e, "quant_linear");
}
