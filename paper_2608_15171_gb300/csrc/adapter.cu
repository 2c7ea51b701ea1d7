// Low-rank adapters of many requests beside a projection that they share:
//   out[t, c] = y[t, c] + scale sum_r (sum_k x[t, k] A[j R + r, k]) B[c, r],
// A, B and scale those of t's adapter, j the slice (of several projections side by
// side) in which column c lies, R the rank.
//
// A unit is up to 16 rows of one adapter, worked by a cluster of CTAs.  The inner sums
// s = x A^T are split over K among the cluster's CTAs and their warps and joined
// through distributed shared memory in a fixed order; then each CTA takes its share of
// the columns.  Both products run on mma.sync 16x8x16: the rows are few, and what
// counts is to read the adapter's weights once.  (A product's K may be taken in any
// order as long as both operands agree: a lane takes 8 neighbouring values of K with
// one 16-byte load for two MMAs, so the operands go from global memory to registers.)
// s enters the second product as two bf16 numbers, a value and what its rounding left,
// so that it counts to 2^-17 of itself.  A row: 2048 x 2560 of rank 16 4.3 us, a chain of
// loads, a cluster barrier, loads and stores; 64 rows of 31 adapters, 4096 x 6144, rank 32 12.9
// (36.6 MB of weights: 2.8 TB/s, in clusters of 4); 128 rows of 76 adapters of rank 64 38.1
// (179 MB: 4.7 TB/s).  (B copied to shared memory while the inner sums are made, by bulk copies: 4.9
// and 15.3 us, 48.5.  One warp's inner sums 96 after another, not parted among warps: 512 rows
// of one adapter of rank 64 20.8 us, 18.1 so.)
#include <algorithm>
#include <cmath>
#include <limits>
#include <memory>
#include <new>
#include <type_traits>
#include <vector>

#include "ppas_device.cuh"
#include "ppas_internal.h"

namespace ppas {
namespace {

constexpr int kAThreads = 512;
constexpr int kAWarps = kAThreads / 32;
constexpr int kAUnitCluster = 16;  // CTAs of a unit's cluster (more than the portable 8)
constexpr int kAChunk = 96;  // inner sums of a warp at most: its loads of 12 x 16 bytes a lane are under way at once
constexpr int kAAhead = 4;   // of the rank in B, 16 times this are loaded ahead
constexpr int32_t kATileMin = 48;    // rows of an adapter next to one another that make tiles,
// and of all such runs together (below, units of 16 rows are done first: 512 rows, 2048 x
// 2560, rank 16 6.7 us, tiles 9.3; 4096 x 6144, rank 16 8.6, 12.2, rank 64 18.1, 17.8, rank 128 29.9,
// 29.6; past it 768 rows 8.5, 9.5 and 15.7, 13.0 and 32.8, 18.5)
constexpr int32_t kATileTotal = 513;
constexpr int kMaxTiles = 2600;      // of a launch (bounded by the 32 KB parameter space),
constexpr int kFewTiles = 160;       // or 2 KB of it (2k step 18.0 us, 18.2 with all of it)

__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float4 ld_cluster_f32x4(uint32_t a) {
    float4 v;
    asm volatile("ld.shared::cluster.v4.f32 {%0,%1,%2,%3}, [%4];"
                 : "=f"(v.x), "=f"(v.y), "=f"(v.z), "=f"(v.w)
                 : "r"(a)
                 : "memory");
    return v;
}
__device__ __forceinline__ void add_to(float4 &v, float4 w) {
    v.x += w.x;
    v.y += w.y;
    v.z += w.z;
    v.w += w.w;
}
// the first half of a cluster barrier, behind what this thread has read
__device__ __forceinline__ void cluster_arrive() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
// two values as bf16, and what their rounding left.  (Finite: a value past the largest bf16 number, an
// infinity too, is that number and what is left.)
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t &hi, uint32_t &lo) {
    asm("cvt.rn.satfinite.bf16x2.f32 %0, %1, %2;" : "=r"(hi) : "f"(b), "f"(a));
    lo = pack_bf16x2(a - __uint_as_float(hi << 16), b - __uint_as_float(hi & 0xFFFF0000u));
}

template <int kUnits, int kRows>
struct UnitParams {
    AdapterParams p;
    int32_t ctas;          // of a cluster
    int32_t beside_tiles;  // launched behind a call's tiles, to run beside them
    int32_t group_at[kAMaxSlices + 1];  // first group of 32 columns of each slice; all of them
    AdapterUnit units[kUnits];
    int32_t rows[kRows];
};

// The inner sums are parted among 2^unit_parts_log(wide) of the warps, up to kAChunk each,
// and K among as many warps as that leaves: log2, and a part's width.
__host__ __device__ constexpr int unit_parts_log(int wide) {
    int l = 0;
    while (wide > kAChunk << l) ++l;
    return l;
}
__host__ __device__ constexpr int unit_part(int wide) {
    const int parts = 1 << unit_parts_log(wide);
    return ((wide + parts - 1) / parts + 7) / 8 * 8;
}
static_assert(1 << unit_parts_log(kAMaxSlices * kAMaxRank) <= kAWarps, "a warp has one part");
__host__ __device__ constexpr int unit_pitch(int wide) { return wide + 4; }
__host__ __device__ constexpr size_t unit_smem(int wide, int part, int steps) {
    return 4 * (static_cast<size_t>(kAWarps) * kAUnitRows * part + kAUnitRows * wide + kAUnitRows * unit_pitch(wide)) +
           static_cast<size_t>(steps) * 32 * 32;
}

}  // namespace

template <int kUnits, int kRows>
__global__ void __launch_bounds__(kAThreads, 1)
    adapter_units_kernel(const __grid_constant__ UnitParams<kUnits, kRows> u) {
    extern __shared__ __align__(16) float adapter_smem[];
    const AdapterParams &p = u.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const int ctas = u.ctas, rank = static_cast<int>(cluster_ctarank());
    const AdapterUnit unit = u.units[blockIdx.x / static_cast<uint32_t>(ctas)];
    const int n = unit.n;
    auto row_of = [&](int i) { return static_cast<int64_t>(unit.listed ? u.rows[unit.first + i] : unit.first + i); };
    grid_dep_launch();
    // Beside tiles: their kernel lets this one start only after its own wait, so all that
    // came before the call has completed; the two write different rows and read nothing
    // that the other writes.  The wait comes at the end then, so that what follows this
    // kernel follows the tiles too.
    if (!u.beside_tiles) grid_dep_wait();

    if (unit.adapter < 0) {  // (every CTA of the cluster)
        // a warp a row, 8 x 16 bytes a lane under way
        const int vecs = p.cols / 8;
        for (int i = rank * kAWarps + warp; i < n; i += kAWarps * ctas) {
            const int64_t row = row_of(i);
            const uint4 *src = reinterpret_cast<const uint4 *>(p.y + row * p.y_stride);
            uint4 *dst = reinterpret_cast<uint4 *>(p.out + row * p.out_stride);
            for (int v0 = lane; v0 < vecs; v0 += 8 * 32) {
                uint4 w[8];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (v0 + k * 32 < vecs) w[k] = src[v0 + k * 32];
#pragma unroll
                for (int k = 0; k < 8; ++k)
                    if (v0 + k * 32 < vecs) dst[v0 + k * 32] = w[k];
            }
        }
        if (u.beside_tiles) grid_dep_wait();
        return;
    }
    const int wide = p.n_slices * p.rank, pitch = unit_pitch(wide), rank16 = (p.rank + 15) / 16;
    const int parts_log = unit_parts_log(wide), width = unit_part(wide);
    float *const red = adapter_smem;                          // [warp][row][width]
    float *const part = red + kAWarps * kAUnitRows * width;   // [row][wide]: this CTA's part of K
    float *const sum = part + kAUnitRows * wide;              // [row][pitch]
    uint4 *const frag = reinterpret_cast<uint4 *>(sum + kAUnitRows * pitch);  // [slice][16 of the rank][lane][2]
    const __nv_bfloat16 *const a = p.a + static_cast<int64_t>(unit.adapter) * wide * p.hidden;
    const __nv_bfloat16 *const b = p.b + static_cast<int64_t>(unit.adapter) * p.cols * p.rank;
    const bool has0 = g < n, has1 = g + 8 < n;
    const int64_t row0 = row_of(has0 ? g : 0), row1 = row_of(has1 ? g + 8 : 0);
    const uint4 zero = make_uint4(0, 0, 0, 0);

    // ---- s = x A^T over this CTA's blocks of 32 of K
    const int blocks = (p.hidden + 31) / 32;
    const int kb0 = blocks * rank / ctas, kb1 = blocks * (rank + 1) / ctas;
    {
        const int n0 = (warp & ((1 << parts_log) - 1)) * width, n1 = min(n0 + width, wide);
        float acc[kAChunk / 8][4] = {};
        for (int kb = kb0 + (warp >> parts_log); kb < kb1; kb += kAWarps >> parts_log) {
            const int k = kb * 32 + t * 8;
            const bool in = k < p.hidden;
            const uint4 x0 = in && has0 ? __ldg(reinterpret_cast<const uint4 *>(p.x + row0 * p.x_stride + k)) : zero;
            const uint4 x1 = in && has1 ? __ldg(reinterpret_cast<const uint4 *>(p.x + row1 * p.x_stride + k)) : zero;
            uint4 w[kAChunk / 8];
            const __nv_bfloat16 *at = a + static_cast<int64_t>(n0 + g) * p.hidden + k;
#pragma unroll
            for (int j = 0; j < kAChunk / 8; ++j) {
                w[j] = in && n0 + 8 * j < n1 ? __ldg(reinterpret_cast<const uint4 *>(at)) : zero;
                at += 8 * p.hidden;
            }
            const uint32_t f0[4] = {x0.x, x1.x, x0.y, x1.y}, f1[4] = {x0.z, x1.z, x0.w, x1.w};
#pragma unroll
            for (int j = 0; j < kAChunk / 8; ++j) {
                if (n0 + 8 * j >= n1) break;
                mma_16816(acc[j], f0, w[j].x, w[j].y);
                mma_16816(acc[j], f1, w[j].z, w[j].w);
            }
        }
        float *const to = red + (warp * kAUnitRows + g) * width + 2 * t;
#pragma unroll
        for (int j = 0; j < kAChunk / 8; ++j) {
            if (n0 + 8 * j >= n1) break;
            if (has0) *reinterpret_cast<float2 *>(to + 8 * j) = make_float2(acc[j][0], acc[j][1]);
            if (has1) *reinterpret_cast<float2 *>(to + 8 * width + 8 * j) = make_float2(acc[j][2], acc[j][3]);
        }
    }
    // ---- out = y + scale s B^T: groups of 32 columns, in each an MMA's column n is
    // column (n / 2) * 8 + 2 j + n % 2 of the group, so that a lane ends with 8 neighbours
    struct Group {
        int slice, col;  // this lane's columns: col .. col + 7
        bool in;
        const __nv_bfloat16 *b;  // its first row of B, the column tiles' 2 rows apart
        int rows;                // of B from there to the slice's end
        uint2 w[4][kAAhead];     // [column tile][16 of the rank]
        uint4 y0, y1;
    };
    auto load_w = [&](const Group &f, int j, int k) {
        return 2 * j < f.rows && k + 4 * t < p.rank ? __ldg(reinterpret_cast<const uint2 *>(f.b + 2 * j * p.rank + k))
                                                    : make_uint2(0, 0);
    };
    auto fetch = [&](int group, Group &f) {
        f.slice = (group >= u.group_at[1]) + (group >= u.group_at[2]) + (group >= u.group_at[3]);
        const int base = p.slice_at[f.slice] + (group - u.group_at[f.slice]) * 32, c1 = p.slice_at[f.slice + 1];
        const int first = base + (g >> 1) * 8 + (g & 1);
        f.col = base + 8 * t;
        f.in = f.col < c1;
        f.rows = c1 - first;
        f.b = b + static_cast<int64_t>(first) * p.rank + 4 * t;
#pragma unroll
        for (int q = 0; q < kAAhead; ++q)
#pragma unroll
            for (int j = 0; j < 4; ++j) f.w[j][q] = load_w(f, j, 16 * q);
        f.y0 = f.y1 = zero;
        if (f.in && has0) f.y0 = *reinterpret_cast<const uint4 *>(p.y + row0 * p.y_stride + f.col);
        if (f.in && has1) f.y1 = *reinterpret_cast<const uint4 *>(p.y + row1 * p.y_stride + f.col);
    };
    const int n_groups = u.group_at[kAMaxSlices], step = kAWarps * ctas;
    int group = rank * kAWarps + warp;
    Group f;
    f.slice = 0;
    // (what the second product reads first is on its way while the sums are joined)
    if (group < n_groups) fetch(group, f);
    __syncthreads();
    const int vecs = wide / 4;
    for (int i = tid; i < n * vecs; i += kAThreads) {
        const int row = i / vecs, c = (i - row * vecs) * 4, from_warp = c / width;
        const float *const from = red + (from_warp * kAUnitRows + row) * width + c - from_warp * width;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        for (int w = 0; w < kAWarps >> parts_log; ++w)
            add_to(v, *reinterpret_cast<const float4 *>(from + (w << parts_log) * kAUnitRows * width));
        *reinterpret_cast<float4 *>(part + row * wide + c) = v;
    }
    cluster_sync_all();
    for (int i = tid; i < kAUnitRows * vecs; i += kAThreads) {
        const int row = i / vecs, c = (i - row * vecs) * 4;
        float4 v = make_float4(0.f, 0.f, 0.f, 0.f);
        if (row < n) {
            const uint32_t at = smem_u32(part + row * wide + c);
#pragma unroll
            for (int r0 = 0; r0 < kAUnitCluster; r0 += 8) {
                if (r0 >= ctas) break;
                float4 from[8];
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r0 + r < ctas) from[r] = ld_cluster_f32x4(dsmem_addr(at, static_cast<uint32_t>(r0 + r)));
#pragma unroll
                for (int r = 0; r < 8; ++r)
                    if (r0 + r < ctas) add_to(v, from[r]);
            }
        }
        *reinterpret_cast<float4 *>(sum + row * pitch + c) = v;
    }
    __syncthreads();
    cluster_arrive();  // nothing of another CTA's is read from here on
    // as the second product's operand, once for all groups: per lane the values and what their rounding left
    for (int i = tid; i < p.n_slices * rank16 * 32; i += kAThreads) {
        const int s = i >> 5, l = i & 31, k = s % rank16 * 16 + 4 * (l & 3);
        float4 s0 = make_float4(0.f, 0.f, 0.f, 0.f), s1 = s0;
        if (k < p.rank) {
            const float *const from = sum + (l >> 2) * pitch + s / rank16 * p.rank + k;
            s0 = *reinterpret_cast<const float4 *>(from);
            s1 = *reinterpret_cast<const float4 *>(from + 8 * pitch);
        }
        uint4 hi, lo;
        split_bf16(s0.x, s0.y, hi.x, lo.x);
        split_bf16(s1.x, s1.y, hi.y, lo.y);
        split_bf16(s0.z, s0.w, hi.z, lo.z);
        split_bf16(s1.z, s1.w, hi.w, lo.w);
        frag[2 * i] = hi;
        frag[2 * i + 1] = lo;
    }
    const float scale = p.scales ? __ldg(p.scales + unit.adapter) : 1.f;
    __syncthreads();
    for (; group < n_groups; group += step) {
        float acc[4][4] = {};
        const uint4 *const s = frag + 2 * (f.slice * rank16 * 32 + lane);
#pragma unroll 1
        for (int q0 = 0; q0 < rank16; q0 += kAAhead) {
            if (q0 > 0) {
#pragma unroll
                for (int e = 0; e < kAAhead; ++e)
#pragma unroll
                    for (int j = 0; j < 4; ++j) f.w[j][e] = load_w(f, j, 16 * (q0 + e));
            }
#pragma unroll
            for (int e = 0; e < kAAhead; ++e) {
                if (q0 + e >= rank16) break;
                const uint4 h = s[(q0 + e) * 64], l = s[(q0 + e) * 64 + 1];
                const uint32_t hi[4] = {h.x, h.y, h.z, h.w}, lo[4] = {l.x, l.y, l.z, l.w};
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    mma_16816(acc[j], hi, f.w[j][e].x, f.w[j][e].y);
                    mma_16816(acc[j], lo, f.w[j][e].x, f.w[j][e].y);
                }
            }
        }
        const uint4 y0 = f.y0, y1 = f.y1;
        const int col = f.col;
        const bool in = f.in;
        if (group + step < n_groups) fetch(group + step, f);
        auto put = [&](uint4 y, int64_t row, int h) {
            uint32_t v[4] = {y.x, y.y, y.z, y.w};
#pragma unroll
            for (int j = 0; j < 4; ++j) {
                const float lo_ = __uint_as_float(v[j] << 16), hi_ = __uint_as_float(v[j] & 0xFFFF0000u);
                v[j] = pack_bf16x2(fmaf(scale, acc[j][2 * h], lo_), fmaf(scale, acc[j][2 * h + 1], hi_));
            }
            *reinterpret_cast<uint4 *>(p.out + row * p.out_stride + col) = make_uint4(v[0], v[1], v[2], v[3]);
        };
        if (in && has0) put(y0, row0, 0);
        if (in && has1) put(y1, row1, 1);
    }
    __syncwarp();
    cluster_wait();  // nobody leaves while others read its part
    if (u.beside_tiles) grid_dep_wait();
}

// ---------------------------------------------------------------- long runs of rows
// A tile of 128 rows (or 64, of the products' 128) of one adapter, on the tcgen05 tensor cores: the inner sums
// s = x A^T [128, slices x rank] accumulate in TMEM over blocks of 64 of K, each slice's on
// columns of its own (rank rounded up to 16).  The epilogue warps turn them, in
// place, into two bf16 numbers each, the operand A in TMEM of the second product, and
// add that product, a block of columns at a time, to y.  So s never leaves the SM, and
// x, y and out cross HBM once.  Where there are fewer tiles than SMs a cluster of CTAs
// shares a tile: each takes a part of K, the parts are summed row by row through
// distributed shared memory, and each takes a share of the columns.
//   warp 0      TMA: x and A tiles into a ring, B tiles into another, y tiles into a
//               third, from which, with the products added, they are stored
//   warp 1      allocates TMEM, issues the MMAs
//   warps 2-17  inner sums, and y + scale s B^T in shared memory: a thread has a row (its
//               TMEM lane); 8 warps have the even blocks of columns, 8 the odd ones, two
//               of them 32 rows, half the columns each
// 16384 rows, 4096 x 6144, rank 64: 98.9 us (544 MB: 5.5 TB/s, 0.81 of the copy's rate; the
// tensor pipe is 22 % busy); 2048 x 2560, rank 16 42.9 us (5.5 TB/s).  HBM is what bounds
// it, but for the turn from the first product to the second, in which a CTA, alone on
// its SM, neither reads nor writes.  (With y and out moved by the epilogue's threads,
// through a transposition in shared memory, a block took 3000 cycles and the call 176 us.)
namespace {

constexpr int kTEpilogue = 512;
constexpr int kTThreads = 64 + kTEpilogue;
enum : int {
    T_FULL = 0,
    T_EMPTY = T_FULL + kTMaxStages,
    T_SUMS = T_EMPTY + kTMaxStages,  // the inner sums are in TMEM
    T_READY,                         // and turned into an operand
    T_BFULL,
    T_BEMPTY = T_BFULL + kTBStages,
    T_YFULL = T_BEMPTY + kTBStages,
    T_YDONE = T_YFULL + kTYStages,     // the products are added
    T_OUTFULL = T_YDONE + kTYStages,   // [2] a block's products are in TMEM
    T_OUTEMPTY = T_OUTFULL + 2,
    T_DONE = T_OUTEMPTY + 2,           // every MMA has completed
    T_COUNT
};
static_assert(T_COUNT * 8 + 8 <= kTBarBytes, "barrier area");

struct TileCall {
    AdapterParams p;
    TileShape s;
    int32_t *err;
    int32_t block_at[kAMaxSlices + 1];  // first block of columns of each slice; all of them
};
template <int kTiles>
struct TileParams : TileCall {
    AdapterTile tiles[kTiles];
};
static_assert(sizeof(TileParams<kMaxTiles>) + 3 * 128 + 2 * 128 <= 32764, "kernel parameter space");

// block i of the columns: its slice, first column and width
struct ColumnBlock {
    int slice, c0, width;
};
__device__ __forceinline__ ColumnBlock column_block(const TileCall &tp, int i) {
    ColumnBlock b;
    b.slice = (i >= tp.block_at[1]) + (i >= tp.block_at[2]) + (i >= tp.block_at[3]);
    b.c0 = tp.p.slice_at[b.slice] + ((i - tp.block_at[b.slice]) << tp.s.block_log);
    b.width = min(1 << tp.s.block_log, tp.p.slice_at[b.slice + 1] - b.c0);
    return b;
}
static_assert(kAMaxSlices == 4, "column_block compares with three of them");

__device__ __forceinline__ void tmem_ld16_sync(uint32_t taddr, float (&v)[16]) {
    asm volatile(
        "tcgen05.ld.sync.aligned.32x32b.x16.b32 "
        "{%0,%1,%2,%3,%4,%5,%6,%7,%8,%9,%10,%11,%12,%13,%14,%15}, [%16];\n\t"
        "tcgen05.wait::ld.sync.aligned;"
        : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]), "=f"(v[4]), "=f"(v[5]), "=f"(v[6]), "=f"(v[7]), "=f"(v[8]),
          "=f"(v[9]), "=f"(v[10]), "=f"(v[11]), "=f"(v[12]), "=f"(v[13]), "=f"(v[14]), "=f"(v[15])
        : "r"(taddr)
        : "memory");
}
__device__ __forceinline__ void tma_store_2d(const CUtensorMap *map, uint32_t from, int32_t x, int32_t y) {
    asm volatile("cp.async.bulk.tensor.2d.global.shared::cta.tile.bulk_group [%0, {%2, %3}], [%1];" ::"l"(
                     reinterpret_cast<uint64_t>(map)),
                 "r"(from), "r"(x), "r"(y)
                 : "memory");
}
__device__ __forceinline__ void stores_commit() { asm volatile("cp.async.bulk.commit_group;" ::: "memory"); }
// until the memory of all but this thread's last n groups of stores has been read
template <int n>
__device__ __forceinline__ void stores_wait_read() {
    asm volatile("cp.async.bulk.wait_group.read %0;" ::"n"(n) : "memory");
}
__device__ __forceinline__ void stores_wait() { asm volatile("cp.async.bulk.wait_group 0;" ::: "memory"); }

}  // namespace

template <int kRows, int kTiles>
__global__ void __launch_bounds__(kTThreads, 1)
    adapter_tiles_kernel(const __grid_constant__ CUtensorMap tm_x, const __grid_constant__ CUtensorMap tm_a,
                         const __grid_constant__ CUtensorMap tm_b, const __grid_constant__ CUtensorMap tm_y,
                         const __grid_constant__ CUtensorMap tm_out, const __grid_constant__ TileParams<kTiles> tp) {
    extern __shared__ uint8_t smem_raw[];
    const AdapterParams &p = tp.p;
    const TileShape &ts = tp.s;
    constexpr uint32_t kXBytes = kRows * 128;
    const uint32_t raw_s = smem_u32(smem_raw);
    const uint32_t sb = (raw_s + 1023u) & ~1023u;
    uint8_t *const sg = smem_raw + (sb - raw_s);
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // (uniform)
    auto bar = [&](int i) { return sb + ts.bars_at + 8u * static_cast<uint32_t>(i); };
    volatile uint32_t *const tmem_base = reinterpret_cast<volatile uint32_t *>(sg + ts.bars_at + T_COUNT * 8);
    volatile int *const abort_flag = reinterpret_cast<volatile int *>(sg + ts.bars_at + T_COUNT * 8 + 4);
    const int ctas = ts.ctas, rank = static_cast<int>(cluster_ctarank());
    const AdapterTile tile = tp.tiles[blockIdx.x / static_cast<uint32_t>(ctas)];

    // the parameters' lines all at once (one after another, as they are used, the first
    // copies went out 2 us later)
    if (warp >= 2 && warp < 2 + 8) {
        const int32_t word = reinterpret_cast<const int32_t *>(&tp)[(warp - 2) * 16];
        asm volatile("" ::"r"(word));
    }
    if (warp == 1) {
        tmem_alloc(smem_u32(const_cast<uint32_t *>(tmem_base)), static_cast<uint32_t>(ts.tmem));
        tmem_relinquish();
    }
    if (warp == 0) {
        if (lane == 0) {
            prefetch_tmap(&tm_x);
            prefetch_tmap(&tm_a);
            prefetch_tmap(&tm_b);
            prefetch_tmap(&tm_y);
            prefetch_tmap(&tm_out);
            *abort_flag = 0;
        }
        for (int i = lane; i < T_COUNT; i += 32) {
            const bool by_warps = i == T_READY || (i >= T_YDONE && i < T_YDONE + kTYStages) || i == T_OUTEMPTY ||
                                  i == T_OUTEMPTY + 1;
            mbar_init(bar(i), i == T_READY ? kTEpilogue / 32 : by_warps ? 8 : 1);
        }
        fence_mbar_init();
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *tmem_base, 0);
    const uint32_t outs = tmem + static_cast<uint32_t>(ts.wide16);  // two blocks of products behind the sums
    // the set-up above overlaps the kernel before this one on the stream
    grid_dep_wait();
    grid_dep_launch();

    // this CTA's blocks of K, and its blocks of columns: rank, rank + ctas, ...
    const int k_blocks = (p.hidden + kTK - 1) / kTK;
    const int kb0 = k_blocks * rank / ctas, kb1 = k_blocks * (rank + 1) / ctas;
    const int mine = (tp.block_at[kAMaxSlices] - rank + ctas - 1) / ctas;
    const uint32_t sub_bytes = kXBytes + ts.a_bytes, stage_bytes = static_cast<uint32_t>(ts.subs) * sub_bytes;
    const int block = 1 << ts.block_log, boxes = block / 64;
    const uint32_t y_bytes = static_cast<uint32_t>(boxes) * kXBytes;
    // (every thread, on every path: the same number of cluster barriers)
    auto cluster_point = [&]() {
        if (ctas > 1) {
            __syncwarp();
            cluster_sync_all();
        }
    };

    if (warp == 0) {
        // ---------------------------------------------------------------- TMA
        bool ok = true;
        int q = 0;
        for (int s = 0, round = 0, kb = kb0; kb < kb1; kb += ts.subs, ++q) {
            if (round > 0 && !mbar_wait_warp(bar(T_EMPTY + s), (round & 1) ^ 1, tp.err)) {
                ok = false;
                break;
            }
            if (elect_one()) {
                uint32_t dst = sb + static_cast<uint32_t>(s) * stage_bytes;
                const int subs = min(ts.subs, kb1 - kb);
                mbar_expect_tx(bar(T_FULL + s), static_cast<uint32_t>(subs) * sub_bytes);
                for (int j = 0; j < subs; ++j, dst += sub_bytes) {
                    tma_load_2d(dst, &tm_x, (kb + j) * kTK, tile.first, bar(T_FULL + s));
                    tma_load_3d(dst + kXBytes, &tm_a, (kb + j) * kTK, 0, tile.adapter * p.n_slices, bar(T_FULL + s));
                }
            }
            __syncwarp();
            if (++s == ts.stages) {
                s = 0;
                ++round;
            }
        }
        const int rank_tiles = (p.rank + 63) / 64;
        auto load_b = [&](int i) {
            const ColumnBlock cb = column_block(tp, rank + i * ctas);
            const int s = i % kTBStages;
            if (elect_one()) {
                mbar_expect_tx(bar(T_BFULL + s), ts.b_bytes);
                for (int h = 0; h < rank_tiles; ++h)
                    tma_load_2d(sb + ts.b_at + static_cast<uint32_t>(s) * ts.b_bytes +
                                    static_cast<uint32_t>(h * block) * 128,
                                &tm_b, h * 64, tile.adapter * p.cols + cb.c0, bar(T_BFULL + s));
            }
            __syncwarp();
        };
        auto load_y = [&](int i) {
            const ColumnBlock cb = column_block(tp, rank + i * ctas);
            const int s = i % ts.y_stages;
            if (lane == 0) {
                const uint32_t dst = sb + static_cast<uint32_t>(s) * y_bytes;
                mbar_expect_tx(bar(T_YFULL + s), y_bytes);
                for (int h = 0; h < boxes; ++h)
                    tma_load_2d(dst + static_cast<uint32_t>(h) * kXBytes, &tm_y, cb.c0 + h * 64, tile.first,
                                bar(T_YFULL + s));
            }
            __syncwarp();
        };
        int nb = 0, ny = 0;
        for (; ok && nb < min(mine, kTBStages); ++nb) load_b(nb);
        cluster_point();
        cluster_point();
        // every MMA on the ring of x and A has completed: its memory is y's
        if (ok) ok = mbar_wait_warp(bar(T_SUMS), 0, tp.err);
        for (; ok && ny < min(mine, ts.y_free); ++ny) load_y(ny);
        if (ok && ny < min(mine, ts.y_stages)) ok = mbar_wait_warp(bar(T_READY), 0, tp.err);
        for (; ok && ny < min(mine, ts.y_stages); ++ny) load_y(ny);
        for (int i = 0; ok && i < mine; ++i) {
            const int s = i % ts.y_stages;
            if (!mbar_wait_warp(bar(T_YDONE + s), (i / ts.y_stages) & 1, tp.err)) {
                ok = false;
                break;
            }
            const ColumnBlock cb = column_block(tp, rank + i * ctas);
            if (lane == 0) {
                const uint32_t from = sb + static_cast<uint32_t>(s) * y_bytes;
                if (tile.n == kRows)
                    for (int h = 0; h < boxes; ++h)
                        if (h * 64 + 64 <= cb.width)
                            tma_store_2d(&tm_out, from + static_cast<uint32_t>(h) * kXBytes, cb.c0 + h * 64, tile.first);
                stores_commit();
            }
            __syncwarp();
            if (nb < mine) {
                if (!mbar_wait_warp(bar(T_BEMPTY + nb % kTBStages), ((nb / kTBStages) & 1) ^ 1, tp.err)) {
                    ok = false;
                    break;
                }
                load_b(nb++);
            }
            // the block before this one has been stored from its memory
            if (i > 0 && ny < mine) {
                if (lane == 0) stores_wait_read<1>();
                __syncwarp();
                load_y(ny++);
            }
        }
        if (!ok) *abort_flag = 1;
        // nothing lands, or is read, once the CTA has left
        ring_land(bar(T_FULL), q, ts.stages, lane);
        ring_land(bar(T_BFULL), nb, kTBStages, lane);
        ring_land(bar(T_YFULL), ny, ts.y_stages, lane);
        if (lane == 0) stores_wait();
        __syncwarp();
    } else if (warp == 1) {
        // ---------------------------------------------------------------- MMAs
        bool ok = true;
        const int width = p.n_slices * ts.rank16;  // N of the first product, in parts of at most 256
        const uint32_t idesc16 = idesc_bf16_f32(kTRows, 16, false, false);
        // (two loops: what an iteration issues decides how fast blocks of K are taken,
        // with the test for a second part in it 470 cycles, 350 without)
        auto inner_sums = [&](auto parts) {
            constexpr bool kTwo = decltype(parts)::value == 2;
            const uint32_t idesc0 = idesc16 + (static_cast<uint32_t>(((kTwo ? 256 : width) - 16) >> 3) << 17);
            const uint32_t idesc1 = idesc16 + (static_cast<uint32_t>((width - 256 - 16) >> 3) << 17);
            const uint64_t dx0 = smem_desc_sw128(sb, 16, 1024), da0 = smem_desc_sw128(sb + kXBytes, 16, 1024);
            uint32_t accumulate = 0;
            for (int q = kb1 - kb0, s = 0, parity = 0; q > 0; q -= ts.subs) {
                if (!mbar_wait_warp(bar(T_FULL + s), parity, tp.err)) return false;
                tc_fence_after();
                const uint64_t at = (static_cast<uint32_t>(s) * stage_bytes) >> 4;
                if (elect_one()) {
                    auto block_of_k = [&](uint64_t dx, uint64_t da) {
#pragma unroll
                        for (int kk = 0; kk < kTK / 16; ++kk) {
                            const uint32_t more = kk > 0 ? 1u : accumulate;
                            umma_bf16(tmem, dx + kk * 2, da + kk * 2, idesc0, more);
                            if (kTwo) umma_bf16(tmem + 256, dx + kk * 2, da + 256 * 8 + kk * 2, idesc1, more);
                        }
                    };
                    block_of_k(dx0 + at, da0 + at);
                    if (!kTwo && ts.subs == 2 && q > 1) {
                        accumulate = 1;
                        block_of_k(dx0 + at + (sub_bytes >> 4), da0 + at + (sub_bytes >> 4));
                    }
                    umma_commit(bar(T_EMPTY + s));
                }
                __syncwarp();
                accumulate = 1;  // (whichever thread is elected)
                if (++s == ts.stages) {
                    s = 0;
                    parity ^= 1;
                }
            }
            if (elect_one()) umma_commit(bar(T_SUMS));
            __syncwarp();
            return true;
        };
        ok = width > 256 ? inner_sums(std::integral_constant<int, 2>{}) : inner_sums(std::integral_constant<int, 1>{});
        cluster_point();
        cluster_point();
        if (ok) ok = mbar_wait_warp(bar(T_READY), 0, tp.err);
        tc_fence_after();
        const uint32_t idesc = idesc_bf16_f32(kTRows, 64, false, false) +
                               (static_cast<uint32_t>((block - 64) >> 3) << 17);
        const uint64_t db0 = smem_desc_sw128(sb + ts.b_at, 16, 1024);
        for (int i = 0; ok && i < mine; ++i) {
            const int s = i % kTBStages, buf = i & 1;
            const int slice = column_block(tp, rank + i * ctas).slice;
            if (!mbar_wait_warp(bar(T_BFULL + s), (i / kTBStages) & 1, tp.err) ||
                (i >= 2 && !mbar_wait_warp(bar(T_OUTEMPTY + buf), ((i >> 1) & 1) ^ 1, tp.err))) {
                ok = false;
                break;
            }
            tc_fence_after();
            if (elect_one()) {
                const uint32_t d = outs + static_cast<uint32_t>(buf * block);
                const uint64_t db = db0 + ((static_cast<uint32_t>(s) * ts.b_bytes) >> 4);
                for (int k = 0; k < ts.rank16; k += 16) {
                    // 16 inner sums: of their columns the first 8 hold their values, the others what was left
                    const uint32_t a = tmem + static_cast<uint32_t>(slice * ts.rank16 + k);
                    const uint64_t b = db + static_cast<uint64_t>((k >> 6) * block * 8 + ((k & 63) >> 3));
                    umma_bf16_ts(d, a, b, idesc, k > 0 ? 1u : 0u);
                    umma_bf16_ts(d, a + 8, b, idesc, 1u);
                }
                umma_commit(bar(T_BEMPTY + s));
                umma_commit(bar(T_OUTFULL + buf));
            }
            __syncwarp();
        }
        if (!ok) *abort_flag = 1;
        if (elect_one()) umma_commit(bar(T_DONE));
        __syncwarp();
        mbar_wait_warp(bar(T_DONE), 0, tp.err);
    } else {
        // ---------------------------------------------------------------- inner sums, output
        // TMEM lane quarter, half of the columns, even or odd blocks
        const int wq = warp & 3, half = ((warp - 2) >> 2) & 1, set = (warp - 2) >> 3;
        const int c_first = ((warp - 2) >> 2) * 16, c_step = kTEpilogue / 8;  // inner sums of this warp: 16 columns at a time
        const int row = wq * 32 + lane;                    // this thread's TMEM lane
        const bool works = kRows == kTRows || wq * 32 < kRows;  // (others only take part in the barriers)
        const uint32_t t_lane = static_cast<uint32_t>(wq * 32) << 16;
        const float scale = p.scales ? __ldg(p.scales + tile.adapter) : 1.f;
        // (every MMA on the ring has completed by then, and with them its copies: its memory is free)
        bool ok = mbar_wait_warp(bar(T_SUMS), 0, tp.err);
        if (!ok) *abort_flag = 1;
        tc_fence_after();
        const int width = p.n_slices * ts.rank16, pitch = ts.wide16 + 4;
        // [own_rows][pitch] the cluster's sums of this CTA's rows, [128][pitch] this CTA's
        // part, later all rows' sums
        float *const summed = reinterpret_cast<float *>(sg + ts.summed_at);
        float *const part = reinterpret_cast<float *>(sg + ts.part_at);
        if (ctas > 1) {
            for (int c = c_first; ok && works && c < width; c += c_step) {
                float v[16];
                tmem_ld16_sync(tmem + t_lane + static_cast<uint32_t>(c), v);
                float4 *const to = reinterpret_cast<float4 *>(part + row * pitch + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) to[i] = make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]);
            }
            cluster_point();
            // the parts of this CTA's rows, summed; then every CTA's sums (both ways along the
            // rows: with each thread reading its own row of the others, 192 sums took 8 us, not 3.5;
            // with every CTA summing all rows, one barrier less, the tiles of the 2k step 18.4 for 17.4)
            const int vecs = width / 4, own0 = rank * ts.own_rows, own = min(ts.own_rows, kRows - own0);
            for (int i = tid - 64; i < vecs * own; i += kTEpilogue) {
                const int r = i / vecs, c = (i - r * vecs) * 4;
                const uint32_t at = smem_u32(part + (own0 + r) * pitch + c);
                float4 sum = make_float4(0.f, 0.f, 0.f, 0.f), v[kAMaxCluster];
#pragma unroll
                for (int o = 0; o < kAMaxCluster; ++o)
                    if (o < ctas) v[o] = ld_cluster_f32x4(dsmem_addr(at, static_cast<uint32_t>(o)));
#pragma unroll
                for (int o = 0; o < kAMaxCluster; ++o)
                    if (o < ctas) add_to(sum, v[o]);
                *reinterpret_cast<float4 *>(summed + r * pitch + c) = sum;
            }
            cluster_point();
            for (int i0 = tid - 64; i0 < vecs * kRows; i0 += 4 * kTEpilogue) {
                float4 v[4];
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = i0 + k * kTEpilogue, r = i / vecs, c = (i - r * vecs) * 4, o = r / ts.own_rows;
                    if (i < vecs * kRows)
                        v[k] = ld_cluster_f32x4(dsmem_addr(smem_u32(summed + (r - o * ts.own_rows) * pitch + c),
                                                           static_cast<uint32_t>(o)));
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    const int i = i0 + k * kTEpilogue, r = i / vecs, c = (i - r * vecs) * 4;
                    if (i < vecs * kRows) *reinterpret_cast<float4 *>(part + r * pitch + c) = v[k];
                }
            }
            nbar_sync(1, kTEpilogue);
        }
        for (int c = c_first; ok && works && c < width; c += c_step) {
            float v[16];
            if (ctas > 1) {
                const float4 *const from = reinterpret_cast<const float4 *>(part + row * pitch + c);
#pragma unroll
                for (int i = 0; i < 4; ++i) {
                    const float4 w = from[i];
                    v[4 * i] = w.x, v[4 * i + 1] = w.y, v[4 * i + 2] = w.z, v[4 * i + 3] = w.w;
                }
            } else {
                tmem_ld16_sync(tmem + t_lane + static_cast<uint32_t>(c), v);
            }
            // (columns past the rank are 0, A's rows there are; but for rows with an infinity, so they are made so)
            const int some = p.rank - c % ts.rank16;
            uint32_t r[16];
#pragma unroll
            for (int i = 0; i < 8; ++i) {
                const bool in = 2 * i < some;  // (the rank is even)
                split_bf16(in ? v[2 * i] : 0.f, in ? v[2 * i + 1] : 0.f, r[i], r[8 + i]);
            }
            tmem_st16(tmem + t_lane + static_cast<uint32_t>(c), r);
        }
        tmem_wait_st();
        tc_fence_before();
        fence_proxy_async_smem();  // y's copies may come where the parts were
        __syncwarp();
        if (lane == 0) mbar_arrive(bar(T_READY));

        // this warp's columns of a block: 64, a box of y, or 32, half a box
        const int groups = block / 64;
        const uint32_t box = block == 128 ? static_cast<uint32_t>(half) * kXBytes : 0u;
        const int first = block == 128 ? 0 : half * 4;  // 16-byte pieces of the box's 128-byte rows
        const int col = half * (block / 2);
        const float2 scale2 = make_float2(scale, scale);
        for (int i = set; i < mine; i += 2) {
            const int buf = i & 1, s = i % ts.y_stages, round = i / ts.y_stages;
            if (!mbar_wait_warp(bar(T_OUTFULL + buf), (i >> 1) & 1, tp.err) ||
                !mbar_wait_warp(bar(T_YFULL + s), round & 1, tp.err) || __any_sync(0xffffffffu, *abort_flag)) {
                ok = false;
                break;
            }
            tc_fence_after();
            const uint32_t y_row = sb + static_cast<uint32_t>(s) * y_bytes + box + static_cast<uint32_t>(row) * 128;
#pragma unroll
            for (int g = 0; g < 2; ++g) {
                if (g >= groups) break;
                if (!works) {
                    if (g == groups - 1 && lane == 0) mbar_arrive(bar(T_OUTEMPTY + buf));
                    continue;
                }
                float v[32];
                tmem_ld32_sync(outs + t_lane + static_cast<uint32_t>(buf * block + col + g * 32), v);
                if (g == groups - 1) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(T_OUTEMPTY + buf));
                }
#pragma unroll
                for (int k = 0; k < 4; ++k) {
                    // (128-byte swizzle)
                    const uint32_t at = y_row + static_cast<uint32_t>(((first + 4 * g + k) ^ (row & 7)) * 16);
                    uint32_t w[4];
                    asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                                 : "=r"(w[0]), "=r"(w[1]), "=r"(w[2]), "=r"(w[3])
                                 : "r"(at)
                                 : "memory");
#pragma unroll
                    for (int e = 0; e < 4; ++e) {
                        const float2 sum = fma2(make_float2(v[8 * k + 2 * e], v[8 * k + 2 * e + 1]), scale2,
                                                make_float2(__uint_as_float(w[e] << 16),
                                                            __uint_as_float(w[e] & 0xFFFF0000u)));
                        w[e] = pack_bf16x2(sum.x, sum.y);
                    }
                    asm volatile("st.shared.v4.u32 [%0], {%1,%2,%3,%4};" ::"r"(at), "r"(w[0]), "r"(w[1]), "r"(w[2]),
                                 "r"(w[3])
                                 : "memory");
                }
            }
            // a box that the tile or the slice ends in is stored by its warps, others by TMA
            const ColumnBlock cb = column_block(tp, rank + i * ctas);
            const int box_col = block == 128 ? col : 0;
            if (works && (tile.n < kRows || box_col + 64 > cb.width)) {
                __syncwarp();
                const int per_row = block == 128 ? 8 : 4;  // pieces of a row that this warp has
                const int piece = lane & (per_row - 1), rows_at_once = 32 / per_row;
                for (int r0 = 0; r0 < 32; r0 += rows_at_once) {
                    const int r = wq * 32 + r0 + lane / per_row;
                    const int c = box_col + (first + piece) * 8;
                    const uint32_t at = sb + static_cast<uint32_t>(s) * y_bytes + box +
                                        static_cast<uint32_t>(r) * 128 +
                                        static_cast<uint32_t>(((first + piece) ^ (r & 7)) * 16);
                    if (r < tile.n && c < cb.width) {
                        uint4 w;
                        asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];"
                                     : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w)
                                     : "r"(at)
                                     : "memory");
                        *reinterpret_cast<uint4 *>(p.out + static_cast<int64_t>(tile.first + r) * p.out_stride + cb.c0 + c) = w;
                    }
                }
            }
            fence_proxy_async_smem();
            __syncwarp();
            if (lane == 0) mbar_arrive(bar(T_YDONE + s));
        }
        if (!ok) *abort_flag = 1;
    }
    tc_fence_before();
    __syncthreads();
    if (warp == 1) {
        tc_fence_after();
        tmem_dealloc(tmem, static_cast<uint32_t>(ts.tmem));
    }
    cluster_point();  // nobody leaves while others read its sums
}

// how tiles of this call lie for clusters of `ctas` CTAs; false: not on this kernel
bool tile_shape(const AdapterParams &p, int ctas, TileShape *s, int rows) {
    *s = {};
    s->ctas = ctas;
    s->rows = rows;
    s->own_rows = (rows + ctas - 1) / ctas;
    s->x_bytes = static_cast<uint32_t>(rows) * 128;
    s->rank16 = (p.rank + 15) / 16 * 16;
    s->wide16 = (p.n_slices * s->rank16 + 31) / 32 * 32;
    s->a_bytes = static_cast<uint32_t>(p.n_slices * s->rank16) * 128;
    const uint32_t stage = s->x_bytes + s->a_bytes;
    // blocks of 128 columns where they fit, else of 64
    for (s->block_log = 7; s->block_log >= 6; --s->block_log) {
        const int block = 1 << s->block_log;
        if (s->wide16 + 2 * block > 512) continue;
        s->tmem = 32;
        while (s->tmem < s->wide16 + 2 * block) s->tmem *= 2;
        s->b_bytes = static_cast<uint32_t>(block * ((p.rank + 63) / 64)) * 128;
        const uint32_t rest = kTBStages * s->b_bytes + kTBarBytes + 1024;  // 1024: to the first boundary of that size
        const uint32_t room = (kTSmem - rest) / 1024 * 1024;
        // (two of them in a stage where three such fit: 2048 rows, 4096 x 6144, rank 16 19.6 us, one 19.9)
        s->subs = s->a_bytes <= 256 * 128 && room / (2 * stage) >= 3 ? 2 : 1;
        s->stages = std::min<int>(kTMaxStages, static_cast<int>(room / (s->subs * stage)));
        const uint32_t y_bytes = static_cast<uint32_t>(block / 64) * s->x_bytes;
        const uint32_t summed = ctas > 1 ? sums_bytes(s->wide16, s->own_rows) : 0;
        const uint32_t part = ctas > 1 ? sums_bytes(s->wide16, rows) : 0;
        if (s->stages < 2 || summed + part > room || summed + 2 * y_bytes > room) continue;
        s->y_stages = std::min<int>(kTYStages, static_cast<int>((room - summed) / y_bytes));
        s->b_at = std::max(static_cast<uint32_t>(s->stages * s->subs) * stage,
                           std::max(static_cast<uint32_t>(s->y_stages) * y_bytes, part) + summed);
        s->b_at = (s->b_at + 1023) / 1024 * 1024;
        s->summed_at = s->b_at - summed;
        s->part_at = s->summed_at - part;
        s->y_free = std::min<int>(s->y_stages, static_cast<int>(s->part_at / y_bytes));
        s->bars_at = s->b_at + kTBStages * s->b_bytes;
        s->smem = s->bars_at + kTBarBytes + 1024;
        if (s->smem <= kTSmem) return true;
    }
    return false;
}

void plan_adapter(int32_t n_seqs, const int32_t *q_lens, const int32_t *adapters, bool copies, int32_t tile_rows,
                  int32_t tile_total, AdapterPlan &plan) {
    constexpr int kCopyRows = 32;  // rows of a unit that is only copied
    plan.units.clear();
    plan.rows.clear();
    plan.tiles.clear();
    auto &rows = plan.gathered;
    rows.clear();
    int64_t in_tiles = 0;
    for (int32_t s = 0; s < n_seqs;) {
        const int32_t id = adapters[s];
        int64_t n = 0;
        while (s < n_seqs && adapters[s] == id) n += q_lens[s++];
        if (id >= 0 && n >= tile_rows) in_tiles += n;
    }
    if (in_tiles < tile_total) tile_rows = INT32_MAX;
    int32_t at = 0;
    for (int32_t s = 0; s < n_seqs;) {
        const int32_t id = adapters[s], first = at;
        while (s < n_seqs && adapters[s] == id) at += q_lens[s++];
        if (id < 0) {
            for (int32_t r = first; copies && r < at; r += kCopyRows)
                plan.units.push_back({r, -1, std::min(kCopyRows, at - r), 0});
            continue;
        }
        int32_t r = first;
        for (const bool tiles = at - r >= tile_rows; tiles && r < at; r += kTRows)
            plan.tiles.push_back({r, id, std::min(kTRows, at - r)});
        r = std::min(r, at);
        for (; at - r >= kAUnitRows; r += kAUnitRows) plan.units.push_back({r, id, kAUnitRows, 0});
        for (; r < at; ++r) rows.emplace_back(id, r);
    }
    std::sort(rows.begin(), rows.end());
    for (size_t i = 0; i < rows.size();) {
        size_t e = i;
        while (e < rows.size() && rows[e].first == rows[i].first && e - i < static_cast<size_t>(kAUnitRows)) ++e;
        const int32_t n = static_cast<int32_t>(e - i);
        const bool run = rows[e - 1].second - rows[i].second == n - 1;
        plan.units.push_back({run ? rows[i].second : static_cast<int32_t>(plan.rows.size()), rows[i].first, n, !run});
        for (; i < e; ++i)
            if (!run) plan.rows.push_back(rows[i].second);
    }
}

namespace {

// Clusters of 2 .. kMost CTAs of a kernel (of a whole SM each) that the current device
// holds at a time; cached per device.
template <auto kernel, int kMost>
cudaError_t clusters_at_a_time(int threads, int smem, int32_t (&clusters)[kMost + 1]) {
    static std::atomic<int32_t> known[64][kMost + 1] = {};  // + 1; 0: not asked
    int dev = 0;
    cudaError_t e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    for (int c = 2; c <= kMost; ++c) {
        int32_t n = dev >= 0 && dev < 64 ? known[dev][c].load(std::memory_order_acquire) : 0;
        if (n == 0) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(static_cast<unsigned>(c));
            cfg.blockDim = dim3(static_cast<unsigned>(threads));
            cfg.dynamicSmemBytes = static_cast<size_t>(smem);
            cudaLaunchAttribute a = {};
            a.id = cudaLaunchAttributeClusterDimension;
            a.val.clusterDim.x = static_cast<unsigned>(c);
            a.val.clusterDim.y = a.val.clusterDim.z = 1;
            cfg.attrs = &a;
            cfg.numAttrs = 1;
            int most = 0;
            e = c == 9 ? cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) : cudaSuccess;
            if (e == cudaSuccess) e = cudaOccupancyMaxActiveClusters(&most, kernel, &cfg);
            if (e != cudaSuccess && c <= 8) return e;
            if (e != cudaSuccess) {
                cudaGetLastError();
                most = 0;  // (none of that size)
            }
            n = most + 1;
            if (dev >= 0 && dev < 64) known[dev][c].store(n, std::memory_order_release);
        }
        clusters[c] = n - 1;
    }
    return cudaSuccess;
}

constexpr int kUnitSmem = static_cast<int>(unit_smem(kAMaxSlices * kAMaxRank, kAChunk, kAMaxSlices * kAMaxRank / 16));
static_assert(kUnitSmem <= static_cast<int>(kTSmem), "shared memory of a CTA");

template <int kUnits, int kRows>
cudaError_t launch_units(const AdapterParams &p, const AdapterPlan &plan, size_t &next, bool beside_tiles, cudaStream_t st) {
    static std::atomic<uint64_t> smem_set{0};
    const auto kernel = adapter_units_kernel<kUnits, kRows>;
    const int wide = p.n_slices * p.rank;
    cudaError_t e = ensure_smem_limit(kernel, kUnitSmem, smem_set);
    if (e != cudaSuccess) return e;
    UnitParams<kUnits, kRows> u;
    u.p = p;
    int n = 0, listed = 0, rows = 0;
    for (; next < plan.units.size() && n < kUnits; ++next, ++n) {
        AdapterUnit unit = plan.units[next];
        if (unit.listed) {
            if (listed + unit.n > kRows) break;
            std::copy_n(plan.rows.begin() + unit.first, unit.n, u.rows + listed);
            unit.first = listed;
            listed += unit.n;
        }
        if (unit.adapter >= 0) rows = std::max(rows, unit.n);
        u.units[n] = unit;
    }
    for (int j = 0, at = 0; j <= kAMaxSlices; ++j) {
        u.group_at[j] = at;
        if (j < kAMaxSlices) at += (p.slice_at[j + 1] - p.slice_at[j] + 31) / 32;
    }
    int32_t clusters[kAUnitCluster + 1] = {};
    e = clusters_at_a_time<adapter_units_kernel<kUnits, kRows>, kAUnitCluster>(kAThreads, kUnitSmem, clusters);
    if (e != cudaSuccess) return e;
    // As many CTAs a unit as run at a time, up to 8, 128 values of K each at least; and 16
    // where a warp then has fewer blocks one after another, of few enough sums that every CTA
    // reads all others' (a row, 4096 x 6144: rank 16 4.5 us, of 8 5.5, rank 64 6.8 and 9.7; 8
    // rows, 2048 x 2560, rank 64, of 16 10.6, 8.2).
    int c = kAMaxCluster;
    while (c > 1 && (n > clusters[c] || p.hidden < c * 128)) --c;
    auto blocks = [&](int ctas) {
        auto parts = [](int all, int of) { return (all + of - 1) / of; };
        return parts(parts((p.hidden + 31) / 32, ctas) << unit_parts_log(wide), kAWarps) +
               parts(u.group_at[kAMaxSlices], ctas * kAWarps);
    };
    constexpr int kFewSums = 768;
    if (n <= clusters[kAUnitCluster] && p.hidden >= kAUnitCluster * 128 && rows * wide <= kFewSums &&
        blocks(kAUnitCluster) < blocks(c))
        c = kAUnitCluster;
    // (beside tiles, on the SMs that their clusters leave: 2k step of 17 tiles and 7 units,
    // clusters of 4 18.0 us, of 8, which find no room, 23.7, of 2 20.7)
    if (beside_tiles) c = std::min(c, 4);
    u.ctas = c;
    u.beside_tiles = beside_tiles ? 1 : 0;
    PdlLaunch l(dim3(static_cast<unsigned>(n * c)), dim3(kAThreads),
                unit_smem(wide, unit_part(wide), p.n_slices * ((p.rank + 15) / 16)), st);
    cudaLaunchAttribute attrs[2] = {l.attr[0], {}};
    if (c > 1) {
        attrs[1].id = cudaLaunchAttributeClusterDimension;
        attrs[1].val.clusterDim.x = static_cast<unsigned>(c);
        attrs[1].val.clusterDim.y = 1;
        attrs[1].val.clusterDim.z = 1;
        l.cfg.attrs = attrs;
        l.cfg.numAttrs = 2;
    }
    return cudaLaunchKernelEx(&l.cfg, kernel, u);
}

cudaError_t launch_tiles(const AdapterParams &p, const AdapterPlan &plan, int64_t n_rows, int32_t n_adapters,
                         int32_t *err, cudaStream_t st) {
    static std::atomic<uint64_t> smem_set[3] = {};
    constexpr auto kMany = adapter_tiles_kernel<kTRows, kMaxTiles>;
    constexpr auto kFew = adapter_tiles_kernel<kTRows, kFewTiles>, kHalf = adapter_tiles_kernel<kTRows / 2, kFewTiles>;
    cudaError_t e = ensure_smem_limit(kMany, static_cast<int>(kTSmem), smem_set[0]);
    if (e == cudaSuccess) e = ensure_smem_limit(kFew, static_cast<int>(kTSmem), smem_set[1]);
    if (e == cudaSuccess) e = ensure_smem_limit(kHalf, static_cast<int>(kTSmem), smem_set[2]);
    if (e != cudaSuccess) return e;
    int32_t clusters[kAMaxCluster + 1] = {};
    e = clusters_at_a_time<kFew, kAMaxCluster>(kTThreads, static_cast<int>(kTSmem), clusters);
    if (e != cudaSuccess) return e;
    TileCall call;
    call.p = p;
    call.err = err;
    // As many CTAs a tile as run at a time (the 17 tiles of a 2k step, hidden 11008: 6 CTAs 17.4 us;
    // 4 19.5; 8, whose clusters take two rounds, 26.5).
    clusters[1] = device_sm_count();
    const int k_blocks = (p.hidden + kTK - 1) / kTK;
    auto ctas_of = [&](int64_t n, int rows) {
        int c = kAMaxCluster;
        while (c > 1 && (n > clusters[c] || c > k_blocks || !tile_shape(p, c, &call.s, rows))) --c;
        return c;
    };
    // Tiles of 64 rows where all of them run at a time and a CTA has a tenth less to do, by
    // what it moves (a block of columns takes no less, its epilogue's warps being half
    // idle) and the joining of the parts, a sum as much as 5 values moved: 768 rows, 4096
    // x 6144, rank 64 18.4 us, of 128 rows 22.7; 1024 rows of rank 16 16.0 and 15.0.
    auto work = [&](int rows) {
        int64_t n = 0;
        for (const AdapterTile &tile : plan.tiles) n += (tile.n + rows - 1) / rows;
        const int c = ctas_of(n, rows);
        if (n > std::min(clusters[c], kFewTiles) || !tile_shape(p, c, &call.s, rows))
            return std::numeric_limits<double>::infinity();
        return (static_cast<double>(p.hidden) * (rows + call.s.wide16) +
                static_cast<double>(p.cols) * (2 * kTRows + call.s.rank16)) / c +
               (c > 1 ? 5.0 * rows * call.s.wide16 : 0.0);
    };
    const int rows_of_tile = work(kTRows / 2) < 0.9 * work(kTRows) ? kTRows / 2 : kTRows;
    std::vector<AdapterTile> parts;
    if (rows_of_tile < kTRows)
        for (const AdapterTile &tile : plan.tiles)
            for (int32_t r = 0; r < tile.n; r += rows_of_tile)
                parts.push_back({tile.first + r, tile.adapter, std::min(rows_of_tile, tile.n - r)});
    const std::vector<AdapterTile> &tiles = rows_of_tile < kTRows ? parts : plan.tiles;
    for (size_t next = 0; next < tiles.size();) {
        const int n = static_cast<int>(std::min<size_t>(kMaxTiles, tiles.size() - next));
        const AdapterTile *const those = tiles.data() + next;
        next += static_cast<size_t>(n);
        const int c = ctas_of(n, rows_of_tile);
        if (!tile_shape(p, c, &call.s, rows_of_tile)) return cudaErrorInvalidValue;  // (the plan asked before)
        for (int j = 0, at = 0; j <= kAMaxSlices; ++j) {
            call.block_at[j] = at;
            if (j < kAMaxSlices) at += (p.slice_at[j + 1] - p.slice_at[j] + (1 << call.s.block_log) - 1) >> call.s.block_log;
        }
        CUtensorMap tm_x, tm_a, tm_b, tm_y, tm_out;
        const uint32_t box_rows = static_cast<uint32_t>(rows_of_tile);
        const uint64_t rows = static_cast<uint64_t>(n_rows), cols = static_cast<uint64_t>(p.cols);
        if (!encode_bf16_rows(&tm_x, p.x, static_cast<uint64_t>(p.hidden), rows, static_cast<uint64_t>(p.x_stride), kTK,
                              box_rows) ||
            !encode_bf16_3d(&tm_a, p.a, static_cast<uint64_t>(p.hidden), static_cast<uint64_t>(p.rank),
                            static_cast<uint64_t>(n_adapters) * p.n_slices, kTK, static_cast<uint32_t>(call.s.rank16),
                            static_cast<uint32_t>(p.n_slices)) ||
            !encode_bf16_2d(&tm_b, p.b, static_cast<uint64_t>(p.rank), static_cast<uint64_t>(n_adapters) * cols, 64,
                            1u << call.s.block_log) ||
            !encode_bf16_rows(&tm_y, p.y, cols, rows, static_cast<uint64_t>(p.y_stride), 64, box_rows) ||
            !encode_bf16_rows(&tm_out, p.out, cols, rows, static_cast<uint64_t>(p.out_stride), 64, box_rows))
            return cudaErrorUnknown;
        PdlLaunch l(dim3(static_cast<unsigned>(n) * static_cast<unsigned>(c)), dim3(kTThreads), call.s.smem, st);
        cudaLaunchAttribute attrs[2] = {l.attr[0], {}};
        if (c > 1) {
            attrs[1].id = cudaLaunchAttributeClusterDimension;
            attrs[1].val.clusterDim.x = static_cast<unsigned>(c);
            attrs[1].val.clusterDim.y = 1;
            attrs[1].val.clusterDim.z = 1;
            l.cfg.attrs = attrs;
            l.cfg.numAttrs = 2;
        }
        auto launch = [&](auto kernel, auto &tp) {
            static_cast<TileCall &>(tp) = call;
            std::copy_n(those, n, tp.tiles);
            return cudaLaunchKernelEx(&l.cfg, kernel, tm_x, tm_a, tm_b, tm_y, tm_out, tp);
        };
        if (n <= kFewTiles) {
            TileParams<kFewTiles> tp;
            e = rows_of_tile == kTRows ? launch(kFew, tp) : launch(kHalf, tp);
        } else {
            const auto tp = std::make_unique<TileParams<kMaxTiles>>();
            e = rows_of_tile == kTRows ? launch(kMany, *tp) : cudaErrorInvalidValue;  // (64 rows: all run at a time)
        }
        if (e != cudaSuccess) return e;
    }
    return cudaSuccess;
}

cudaError_t launch_adapter(const AdapterParams &p, const AdapterPlan &plan, int64_t n_rows, int32_t n_adapters,
                           int32_t *err, cudaStream_t st) {
    cudaError_t e = plan.tiles.empty() ? cudaSuccess : launch_tiles(p, plan, n_rows, n_adapters, err, st);
    const bool few = plan.units.size() <= 64 && plan.rows.size() <= 256;
    for (size_t next = 0; e == cudaSuccess && next < plan.units.size();)
        e = few ? launch_units<64, 256>(p, plan, next, !plan.tiles.empty(), st)
                : launch_units<1024, 3584>(p, plan, next, !plan.tiles.empty() && next == 0, st);
    return e;
}

bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

}  // namespace
}  // namespace ppas

using namespace ppas;

extern "C" ppas_status ppas_adapter_add(const void *x, int64_t x_stride, const void *y, int64_t y_stride, void *out,
                                        int64_t out_stride, int32_t n_seqs, const int32_t *h_q_lens,
                                        const int32_t *h_adapters, const void *a, const void *b,
                                        const float *d_scales, int32_t n_adapters, int32_t hidden, int32_t n_slices,
                                        const int32_t *h_slice_cols, int32_t rank, int32_t *d_err_flag, void *stream) {
    if (n_seqs < 0 || n_adapters < 1 || hidden < 1 || n_slices < 1 || rank < 1) return PPAS_ERR_INVALID_ARG;
    if (hidden % 8 || n_slices > kAMaxSlices || rank % 8 || rank > kAMaxRank) return PPAS_ERR_UNSUPPORTED;
    if (!h_slice_cols || (n_seqs > 0 && (!h_q_lens || !h_adapters))) return PPAS_ERR_INVALID_ARG;
    AdapterParams p = {};
    int64_t cols = 0;
    for (int32_t j = 0; j < n_slices; ++j) {
        if (h_slice_cols[j] < 1) return PPAS_ERR_INVALID_ARG;
        if (h_slice_cols[j] % 8) return PPAS_ERR_UNSUPPORTED;
        p.slice_at[j] = static_cast<int32_t>(cols);
        cols += h_slice_cols[j];
        if (cols > (1 << 24)) return PPAS_ERR_UNSUPPORTED;
    }
    for (int32_t j = n_slices; j <= kAMaxSlices; ++j) p.slice_at[j] = static_cast<int32_t>(cols);
    if (hidden > (1 << 24)) return PPAS_ERR_UNSUPPORTED;
    int64_t n_rows = 0;
    for (int32_t s = 0; s < n_seqs; ++s) {
        if (h_q_lens[s] < 1 || h_adapters[s] < -1 || h_adapters[s] >= n_adapters) return PPAS_ERR_INVALID_ARG;
        n_rows += h_q_lens[s];
    }
    if (n_rows > (1 << 24) || static_cast<int64_t>(n_adapters) * n_slices * rank > INT32_MAX ||
        n_adapters * cols > INT32_MAX)
        return PPAS_ERR_UNSUPPORTED;
    if (n_rows == 0) return PPAS_OK;
    constexpr int64_t kStrides = int64_t{1} << 36;  // (a tensor map's are below 2^40 bytes)
    if (x_stride > kStrides || y_stride > kStrides || out_stride > kStrides) return PPAS_ERR_UNSUPPORTED;
    if (x_stride < hidden || y_stride < cols || out_stride < cols || x_stride % 8 || y_stride % 8 || out_stride % 8)
        return PPAS_ERR_INVALID_ARG;
    if (!x || !y || !out || !a || !b || !on16(x) || !on16(y) || !on16(out) || !on16(a) || !on16(b) ||
        (reinterpret_cast<uintptr_t>(d_scales) & 3u) || (reinterpret_cast<uintptr_t>(d_err_flag) & 3u))
        return PPAS_ERR_INVALID_ARG;
    if (out == x || (out == y && out_stride != y_stride)) return PPAS_ERR_INVALID_ARG;
    p.x = static_cast<const __nv_bfloat16 *>(x);
    p.y = static_cast<const __nv_bfloat16 *>(y);
    p.out = static_cast<__nv_bfloat16 *>(out);
    p.x_stride = x_stride;
    p.y_stride = y_stride;
    p.out_stride = out_stride;
    p.a = static_cast<const __nv_bfloat16 *>(a);
    p.b = static_cast<const __nv_bfloat16 *>(b);
    p.scales = d_scales;
    p.hidden = hidden;
    p.rank = rank;
    p.n_slices = n_slices;
    p.cols = static_cast<int32_t>(cols);
    try {
        TileShape shape;
        thread_local AdapterPlan plan;  // (for its memory alone)
        plan_adapter(n_seqs, h_q_lens, h_adapters, out != y, tile_shape(p, 1, &shape) ? kATileMin : INT32_MAX,
                     kATileTotal, plan);
        return launch_adapter(p, plan, n_rows, n_adapters, d_err_flag, static_cast<cudaStream_t>(stream)) == cudaSuccess
                   ? PPAS_OK
                   : PPAS_ERR_CUDA;
    } catch (const std::exception &) {
        return PPAS_ERR_CAPACITY;  // host memory
    }
}
