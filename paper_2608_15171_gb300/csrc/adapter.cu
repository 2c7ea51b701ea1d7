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
// so that it counts to 2^-17 of itself.
#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "ppas_device.cuh"
#include "ppas_internal.h"

namespace ppas {
namespace {

constexpr int kAThreads = 256;
constexpr int kAWarps = kAThreads / 32;
constexpr int kAChunk = 64;  // inner sums worked at a time
constexpr int kAMaxCluster = 8;

__device__ __forceinline__ void mma_16816(float (&c)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
    asm volatile(
        "mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(c[0]), "+f"(c[1]), "+f"(c[2]), "+f"(c[3])
        : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
__device__ __forceinline__ float ld_cluster_f32(uint32_t a) {
    float v;
    asm volatile("ld.shared::cluster.f32 %0, [%1];" : "=f"(v) : "r"(a) : "memory");
    return v;
}
// two values as bf16, and what their rounding left (0 of an infinity)
__device__ __forceinline__ void split_bf16(float a, float b, uint32_t &hi, uint32_t &lo) {
    hi = pack_bf16x2(a, b);
    const float ha = __uint_as_float(hi << 16), hb = __uint_as_float(hi & 0xFFFF0000u);
    lo = pack_bf16x2(fabsf(ha) < INFINITY ? a - ha : 0.f, fabsf(hb) < INFINITY ? b - hb : 0.f);
}

template <int kUnits, int kRows>
struct UnitParams {
    AdapterParams p;
    AdapterUnit units[kUnits];
    int32_t rows[kRows];
};

__host__ __device__ constexpr int unit_pitch(int wide) { return wide + 4; }
__host__ __device__ constexpr size_t unit_smem(int wide) {
    const int chunk = wide < kAChunk ? wide : kAChunk;
    return 4 * (static_cast<size_t>(kAWarps) * kAUnitRows * chunk + kAUnitRows * wide +
                kAUnitRows * unit_pitch(wide));
}

}  // namespace

template <int kUnits, int kRows>
__global__ void __launch_bounds__(kAThreads)
    adapter_units_kernel(const __grid_constant__ UnitParams<kUnits, kRows> u) {
    extern __shared__ __align__(16) float adapter_smem[];
    const AdapterParams &p = u.p;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int g = lane >> 2, t = lane & 3;
    const uint32_t ctas = cluster_nctarank(), rank = cluster_ctarank();
    const AdapterUnit &unit = u.units[blockIdx.x / ctas];
    const int n = unit.n;
    auto row_of = [&](int i) { return static_cast<int64_t>(unit.listed ? u.rows[unit.first + i] : unit.first + i); };
    grid_dep_launch();
    grid_dep_wait();

    if (unit.adapter < 0) {  // (every CTA of the cluster)
        const int vecs = p.cols / 8;
        for (int i = 0; i < n; ++i) {
            const int64_t row = row_of(i);
            const uint4 *src = reinterpret_cast<const uint4 *>(p.y + row * p.y_stride);
            uint4 *dst = reinterpret_cast<uint4 *>(p.out + row * p.out_stride);
            for (int v = static_cast<int>(rank) * kAThreads + tid; v < vecs; v += static_cast<int>(ctas) * kAThreads)
                dst[v] = src[v];
        }
        return;
    }
    const int wide = p.n_slices * p.rank, chunk = min(wide, kAChunk), pitch = unit_pitch(wide);
    float *const red = adapter_smem;                       // [warp][row][chunk]
    float *const part = red + kAWarps * kAUnitRows * chunk;  // [row][wide]: this CTA's part of K
    float *const sum = part + kAUnitRows * wide;           // [row][pitch]
    const __nv_bfloat16 *const a = p.a + static_cast<int64_t>(unit.adapter) * wide * p.hidden;
    const __nv_bfloat16 *const b = p.b + static_cast<int64_t>(unit.adapter) * p.cols * p.rank;
    const bool has0 = g < n, has1 = g + 8 < n;
    const int64_t row0 = row_of(has0 ? g : 0), row1 = row_of(has1 ? g + 8 : 0);
    const float scale = p.scales ? __ldg(p.scales + unit.adapter) : 1.f;
    const uint4 zero = make_uint4(0, 0, 0, 0);

    // ---- s = x A^T over this CTA's blocks of 32 of K
    const int blocks = (p.hidden + 31) / 32, per = (blocks + static_cast<int>(ctas) - 1) / static_cast<int>(ctas);
    const int kb1 = min(blocks, (static_cast<int>(rank) + 1) * per);
    for (int n0 = 0; n0 < wide; n0 += kAChunk) {
        float acc[kAChunk / 8][4] = {};
        for (int kb = static_cast<int>(rank) * per + warp; kb < kb1; kb += kAWarps) {
            const int k = kb * 32 + t * 8;
            const bool in = k < p.hidden;
            const uint4 x0 = in && has0 ? __ldg(reinterpret_cast<const uint4 *>(p.x + row0 * p.x_stride + k)) : zero;
            const uint4 x1 = in && has1 ? __ldg(reinterpret_cast<const uint4 *>(p.x + row1 * p.x_stride + k)) : zero;
            uint4 w[kAChunk / 8];
#pragma unroll
            for (int j = 0; j < kAChunk / 8; ++j)
                w[j] = in && n0 + 8 * j < wide
                           ? __ldg(reinterpret_cast<const uint4 *>(a + static_cast<int64_t>(n0 + 8 * j + g) * p.hidden + k))
                           : zero;
            const uint32_t f0[4] = {x0.x, x1.x, x0.y, x1.y}, f1[4] = {x0.z, x1.z, x0.w, x1.w};
#pragma unroll
            for (int j = 0; j < kAChunk / 8; ++j) {
                if (n0 + 8 * j >= wide) break;
                mma_16816(acc[j], f0, w[j].x, w[j].y);
                mma_16816(acc[j], f1, w[j].z, w[j].w);
            }
        }
#pragma unroll
        for (int j = 0; j < kAChunk / 8; ++j) {
            if (n0 + 8 * j >= wide) break;
            float *const to = red + (warp * kAUnitRows + g) * chunk + 8 * j + 2 * t;
            *reinterpret_cast<float2 *>(to) = make_float2(acc[j][0], acc[j][1]);
            *reinterpret_cast<float2 *>(to + 8 * chunk) = make_float2(acc[j][2], acc[j][3]);
        }
        __syncthreads();
        const int width = min(chunk, wide - n0);
        for (int i = tid; i < n * width; i += kAThreads) {
            const int row = i / width, c = i - row * width;
            float v = 0.f;
#pragma unroll
            for (int w = 0; w < kAWarps; ++w) v += red[(w * kAUnitRows + row) * chunk + c];
            part[row * wide + n0 + c] = v;
        }
        __syncthreads();
    }
    cluster_sync_all();
    for (int i = tid; i < kAUnitRows * wide; i += kAThreads) {
        const int row = i / wide, c = i - row * wide;
        float v = 0.f;
        if (row < n)
            for (uint32_t r = 0; r < ctas; ++r) v += ld_cluster_f32(dsmem_addr(smem_u32(part + row * wide + c), r));
        sum[row * pitch + c] = v;
    }
    cluster_sync_all();  // nothing of another CTA's is read from here on

    // ---- out = y + scale s B^T: groups of 32 columns, in each an MMA's column n is
    // column (n / 2) * 8 + 2 j + n % 2 of the group, so that a lane ends with 8 neighbours
    int group = 0;
    for (int slice = 0; slice < p.n_slices; ++slice) {
        const int c0 = p.slice_at[slice], c1 = p.slice_at[slice + 1];
        const float *const s = sum + slice * p.rank;
        for (int base = c0; base < c1; base += 32, ++group) {
            if (group % (kAWarps * static_cast<int>(ctas)) != static_cast<int>(rank) * kAWarps + warp) continue;
            const int col = base + 8 * t;
            const bool in = col < c1;
            uint4 y0 = zero, y1 = zero;
            if (in && has0) y0 = *reinterpret_cast<const uint4 *>(p.y + row0 * p.y_stride + col);
            if (in && has1) y1 = *reinterpret_cast<const uint4 *>(p.y + row1 * p.y_stride + col);
            float acc[4][4] = {};
            for (int q = 0; q < p.rank; q += 16) {
                const int k = q + 4 * t;
                const bool k_in = k < p.rank;
                float4 s0 = make_float4(0.f, 0.f, 0.f, 0.f), s1 = s0;
                if (k_in) {
                    s0 = *reinterpret_cast<const float4 *>(s + g * pitch + k);
                    s1 = *reinterpret_cast<const float4 *>(s + (g + 8) * pitch + k);
                }
                uint32_t hi[4], lo[4];
                split_bf16(s0.x, s0.y, hi[0], lo[0]);
                split_bf16(s1.x, s1.y, hi[1], lo[1]);
                split_bf16(s0.z, s0.w, hi[2], lo[2]);
                split_bf16(s1.z, s1.w, hi[3], lo[3]);
#pragma unroll
                for (int j = 0; j < 4; ++j) {
                    const int at = base + (g >> 1) * 8 + 2 * j + (g & 1);
                    const uint2 w = k_in && at < c1 ? __ldg(reinterpret_cast<const uint2 *>(
                                                          b + static_cast<int64_t>(at) * p.rank + k))
                                                    : make_uint2(0, 0);
                    mma_16816(acc[j], hi, w.x, w.y);
                    mma_16816(acc[j], lo, w.x, w.y);
                }
            }
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
    }
}

AdapterPlan plan_adapter(int32_t n_seqs, const int32_t *q_lens, const int32_t *adapters, bool copies) {
    constexpr int kCopyRows = 32;  // rows of a unit that is only copied
    AdapterPlan plan;
    std::vector<std::pair<int32_t, int32_t>> rows;  // (adapter, row) of those that are gathered
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
    return plan;
}

namespace {

template <int kUnits, int kRows>
cudaError_t launch_units(const AdapterParams &p, const AdapterPlan &plan, size_t &next, cudaStream_t st) {
    static std::atomic<uint64_t> smem_set{0};
    const auto kernel = adapter_units_kernel<kUnits, kRows>;
    const int wide = p.n_slices * p.rank;
    const cudaError_t e =
        ensure_smem_limit(kernel, static_cast<int>(unit_smem(kAMaxSlices * kAMaxRank)), smem_set);
    if (e != cudaSuccess) return e;
    UnitParams<kUnits, kRows> u;
    u.p = p;
    int n = 0, listed = 0;
    for (; next < plan.units.size() && n < kUnits; ++next, ++n) {
        AdapterUnit unit = plan.units[next];
        if (unit.listed) {
            if (listed + unit.n > kRows) break;
            std::copy_n(plan.rows.begin() + unit.first, unit.n, u.rows + listed);
            unit.first = listed;
            listed += unit.n;
        }
        u.units[n] = unit;
    }
    // as many CTAs a unit as the SMs hold twice, 128 values of K each at least
    int c = 1;
    while (c < kAMaxCluster && 2 * c * n <= 2 * device_sm_count() && p.hidden >= 2 * c * 128) c *= 2;
    PdlLaunch l(dim3(static_cast<unsigned>(n * c)), dim3(kAThreads), unit_smem(wide), st);
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

cudaError_t launch_adapter(const AdapterParams &p, const AdapterPlan &plan, cudaStream_t st) {
    cudaError_t e = cudaSuccess;
    const bool few = plan.units.size() <= 64 && plan.rows.size() <= 256;
    for (size_t next = 0; e == cudaSuccess && next < plan.units.size();)
        e = few ? launch_units<64, 256>(p, plan, next, st) : launch_units<1024, 3584>(p, plan, next, st);
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
        const AdapterPlan plan = plan_adapter(n_seqs, h_q_lens, h_adapters, out != y);
        return launch_adapter(p, plan, static_cast<cudaStream_t>(stream)) == cudaSuccess ? PPAS_OK : PPAS_ERR_CUDA;
    } catch (const std::exception &) {
        return PPAS_ERR_CAPACITY;  // host memory
    }
}
