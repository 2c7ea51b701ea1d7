// Sampling the next tokens: temperature, top-k, top-p and min-p, one given
// uniform number a row.
//
// The definition (x a row of logits, M its maximum, T its temperature):
//   z_i = (x_i - M) / T,  w_i = exp(z_i),  W_i = floor(w_i 2^40),
// tokens ordered by x descending, index ascending; kept are the first n of them,
//   n = min(k, least n with W_1 + .. + W_n >= p (W_1 + .. + W_k), #{z_i >= ln p_min}),
// and with S their sum the token drawn is the first with W_1 + .. + W_j > u S.
// The weights are whole numbers, so every sum is exact and no answer depends on
// the order of additions: the same row gives the same token whatever the batch
// and however it is split.  (2^-40 of the largest weight is a tenth of what fp32
// sums of a vocabulary round off.)
//
// A row's logits are read once: a cluster of CTAs holds the row in shared
// memory.  All three cuts are the same question, at which token a running sum
// in the order reaches a target, and need no sort: one histogram of weights over
// bins of z (linear, so the bins fill evenly and few additions collide), summed
// over the cluster, gives the bin; its tokens (a few hundred) go to the first
// CTA, which ranks them against one another.  A bin with more than that (ties,
// flat rows) is divided again, by the bits of (x, index).
#include <math.h>

#include "ppas_device.cuh"
#include "ppas_internal.h"

namespace ppas {
namespace {

constexpr int kSThreads = 512;
constexpr int kSWarps = kSThreads / 32;
constexpr int kSBins = 1024;      // bins of z
constexpr int kSFine = 512;       // bins of a bin's (x, index)
constexpr int kSList = 512;       // tokens that are ranked against one another
constexpr int kSIndexBits = 18;   // vocabularies of up to 2^18 tokens
constexpr int kSMaxCluster = 8;
constexpr float kSFloor = -28.f;  // z below this: W = 0 (exp(-28) 2^40 < 1)
constexpr int kSMaxCommands = 40;
static_assert(kSMaxVocab == 1 << kSIndexBits, "index bits");
static_assert(kSBins % (2 * kSMaxCluster) == 0 && kSFine % kSMaxCluster == 0 && kSBins == 2 * kSFine &&
                  kSBins == 2 * kSThreads && kSFine == kSThreads && kSList <= kSThreads,
              "the scans give each thread two bins or one");

enum : uint32_t { kDone, kGatherBin, kGatherRange, kDivide };

struct SCommand {
    uint32_t op, bin;
    uint64_t lo, hi;  // range of (x, index)
    uint32_t shift, pad;
};

struct SShared {
    uint32_t cnt[kSBins], wl[kSBins], wh[kSBins];  // this CTA's histogram; divided bins: the first kSFine, and
                                                   // behind them the first CTA's sums over the cluster
    uint64_t sum_w[kSBins];                        // first CTA: sums over the cluster, then running sums
    uint32_t sum_c[kSBins];
    uint2 list[kSList];                            // (key, index) of a gathered bin's tokens
    uint64_t list_w[kSList];
    float2 range[kSMaxCluster];                    // (max, min finite) of each CTA
    uint64_t above[kSMaxCluster];                  // weight with z >= ln p_min, or the lowest index of the maximum
    uint64_t warp_w[kSWarps];
    uint32_t warp_c[kSWarps];
    float2 warp_range[kSWarps];
    uint32_t n, kmin, kmax;                        // of this CTA's gathered tokens
    SCommand cmd;
    uint64_t base_w, base_c, got_w, got_mass;      // first CTA: sums before the bin, what a search found
    uint32_t got_bin, got_index;
    float got_z;
};

__device__ __forceinline__ uint32_t ld_cluster_u32(uint32_t a) {
    uint32_t v;
    asm volatile("ld.shared::cluster.u32 %0, [%1];" : "=r"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ uint64_t ld_cluster_u64(uint32_t a) {
    uint64_t v;
    asm volatile("ld.shared::cluster.u64 %0, [%1];" : "=l"(v) : "r"(a) : "memory");
    return v;
}
__device__ __forceinline__ void st_cluster_u32(uint32_t a, uint32_t v) {
    asm volatile("st.shared::cluster.u32 [%0], %1;" ::"r"(a), "r"(v) : "memory");
}
__device__ __forceinline__ void st_cluster_u64(uint32_t a, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}

// a token's place in the order: ascending keys are descending logits (no -0, no NaN)
__device__ __forceinline__ uint32_t order_key(float x) {
    const uint32_t b = __float_as_uint(x);
    return (b >> 31) ? b : ~(b | 0x80000000u);
}
__device__ __forceinline__ float key_value(uint32_t k) {
    return __uint_as_float((k >> 31) ? k : ~k & 0x7FFFFFFFu);
}

struct SRow {
    float top, inv_t, bin_scale;
    __device__ __forceinline__ float z(float x) const { return x == top ? 0.f : (x - top) * inv_t; }
    __device__ __forceinline__ int bin(float z_) const {
        return min(static_cast<int>(-z_ * bin_scale), kSBins - 1);
    }
    // tokens that can be drawn or counted (a -inf is below the floor, a NaN no comparison holds for)
    __device__ __forceinline__ static bool counts(float x, float z_) { return x > -INFINITY && z_ > kSFloor; }
    __device__ __forceinline__ static uint64_t weight(float z_) { return __float2ull_rz(expf(z_) * 0x1p40f); }
};

__device__ __forceinline__ void add_weight(uint32_t *wl, uint32_t *wh, uint64_t w) {
    const uint32_t lo = static_cast<uint32_t>(w);
    uint32_t hi = static_cast<uint32_t>(w >> 32);
    if (lo) hi += atomicAdd(wl, lo) + lo < lo ? 1u : 0u;  // the carry of this addition
    if (hi) atomicAdd(wh, hi);
}

// inclusive sums over the CTA's threads
__device__ __forceinline__ void block_scan(SShared &s, uint64_t &w, uint32_t &c) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
        const uint64_t a = __shfl_up_sync(0xffffffffu, w, o);
        const uint32_t b = __shfl_up_sync(0xffffffffu, c, o);
        if (lane >= o) {
            w += a;
            c += b;
        }
    }
    if (lane == 31) {
        s.warp_w[warp] = w;
        s.warp_c[warp] = c;
    }
    __syncthreads();
    for (int i = 0; i < warp; ++i) {
        w += s.warp_w[i];
        c += s.warp_c[i];
    }
}

// Sums the cluster's histograms and leaves the bins' sums in the first CTA:
// each CTA adds up the bins [rank * n / ctas, (rank + 1) * n / ctas).
template <bool kFine>
__device__ __forceinline__ void push_sums(SShared &s, uint32_t rank, uint32_t ctas, bool counted) {
    constexpr int n = kFine ? kSFine : kSBins;
    const int per = n / static_cast<int>(ctas);
    for (int i = threadIdx.x; i < per; i += kSThreads) {
        const int b = static_cast<int>(rank) * per + i;
        uint64_t w = 0;
        uint32_t c = 0;
        for (uint32_t r = 0; r < ctas; ++r) {
            w += static_cast<uint64_t>(ld_cluster_u32(dsmem_addr(smem_u32(&s.wl[b]), r))) +
                 (static_cast<uint64_t>(ld_cluster_u32(dsmem_addr(smem_u32(&s.wh[b]), r))) << 32);
            if (counted) c += ld_cluster_u32(dsmem_addr(smem_u32(&s.cnt[b]), r));
        }
        if (kFine) {
            st_cluster_u32(dsmem_addr(smem_u32(&s.cnt[kSFine + b]), 0), c);
            st_cluster_u32(dsmem_addr(smem_u32(&s.wl[kSFine + b]), 0), static_cast<uint32_t>(w));
            st_cluster_u32(dsmem_addr(smem_u32(&s.wh[kSFine + b]), 0), static_cast<uint32_t>(w >> 32));
        } else {
            st_cluster_u64(dsmem_addr(smem_u32(&s.sum_w[b]), 0), w);
            st_cluster_u32(dsmem_addr(smem_u32(&s.sum_c[b]), 0), c);
        }
    }
}

// what the first CTA looks for: the token at which the running weight (or count) reaches `target`
struct STarget {
    bool by_count;
    uint64_t target;
};

// The bin of z in which the target lies: got_bin, base_w, base_c.
__device__ __forceinline__ void find_bin(SShared &s, const STarget &t) {
    if (threadIdx.x == 0) s.got_bin = 0xFFFFFFFFu;
    __syncthreads();
#pragma unroll
    for (int k = 0; k < 2; ++k) {
        const int b = 2 * threadIdx.x + k;
        const uint64_t w0 = b ? s.sum_w[b - 1] : 0, w1 = s.sum_w[b];
        const uint64_t c0 = b ? s.sum_c[b - 1] : 0, c1 = s.sum_c[b];
        if (t.by_count ? (c0 < t.target && t.target <= c1) : (w0 < t.target && t.target <= w1)) {
            s.got_bin = b;
            s.base_w = w0;
            s.base_c = c0;
        }
    }
    __syncthreads();
}

// the first CTA's command, written into every CTA of the cluster (one thread)
__device__ __forceinline__ void send(SShared &s, const SCommand &c, uint32_t ctas) {
    for (uint32_t r = 0; r < ctas; ++r) {
        const uint32_t a = dsmem_addr(smem_u32(&s.cmd), r);
        st_cluster_u32(a + offsetof(SCommand, op), c.op);
        st_cluster_u32(a + offsetof(SCommand, bin), c.bin);
        st_cluster_u64(a + offsetof(SCommand, lo), c.lo);
        st_cluster_u64(a + offsetof(SCommand, hi), c.hi);
        st_cluster_u32(a + offsetof(SCommand, shift), c.shift);
    }
}

// Ranks the gathered tokens (n of them, in the cluster's lists) against one
// another: got_w (running weight up to the token found), got_mass, got_index.
__device__ __forceinline__ void rank_list(SShared &s, const SRow &row, const STarget &t, uint32_t ctas, uint32_t n) {
    const uint32_t i = threadIdx.x;
    uint2 mine = make_uint2(0, 0);
    uint64_t w = 0;
    if (i < n) {
        uint32_t at = i, r = 0;
        for (; r + 1 < ctas; ++r) {
            const uint32_t nr = ld_cluster_u32(dsmem_addr(smem_u32(&s.n), r));
            if (at < nr) break;
            at -= nr;
        }
        const uint64_t e = ld_cluster_u64(dsmem_addr(smem_u32(&s.list[at]), r));
        mine = make_uint2(static_cast<uint32_t>(e), static_cast<uint32_t>(e >> 32));
        w = SRow::weight(row.z(key_value(mine.x)));
    }
    __syncthreads();  // every entry is in registers: the first CTA's own list may be overwritten
    if (threadIdx.x == 0) s.got_index = 0xFFFFFFFFu;
    if (i < n) {
        s.list[i] = mine;
        s.list_w[i] = w;
    }
    __syncthreads();
    if (i < n) {
        uint64_t up_w = 0;  // of the tokens up to this one
        uint32_t up_c = 0;
        for (uint32_t j = 0; j < n; ++j) {
            const uint2 o = s.list[j];
            if (o.x < mine.x || (o.x == mine.x && o.y <= mine.y)) {
                up_w += s.list_w[j];
                ++up_c;
            }
        }
        const uint64_t at_w = s.base_w + up_w, at_c = s.base_c + up_c;
        if (t.by_count ? at_c == t.target : (at_w - w < t.target && t.target <= at_w)) {
            s.got_w = at_w;
            s.got_mass = w;
            s.got_index = mine.y;
            s.got_z = row.z(key_value(mine.x));
        }
    }
    __syncthreads();
}

}  // namespace

template <class T>
__global__ void __launch_bounds__(kSThreads, 2) sample_kernel(const __grid_constant__ SampleParams p) {
    extern __shared__ __align__(16) uint8_t sample_smem[];
    SShared &s = *reinterpret_cast<SShared *>(sample_smem);
    float *const xs = reinterpret_cast<float *>(sample_smem + (sizeof(SShared) + 15) / 16 * 16);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t ctas = cluster_nctarank(), rank = ctas > 1 ? cluster_ctarank() : 0;
    const int32_t r = blockIdx.x / ctas;
    for (int b = tid; b < kSBins; b += kSThreads) s.cnt[b] = s.wl[b] = s.wh[b] = 0;
    grid_dep_launch();
    grid_dep_wait();

    // ---- this CTA's part of the row, 16 bytes at a time between its first and last 16-byte boundary
    const int32_t i0 = min(static_cast<int32_t>(rank) * p.chunk, p.vocab);
    const int32_t n = min(p.chunk, p.vocab - i0);
    const T *const src = static_cast<const T *>(p.logits) + r * p.row_stride + i0;
    constexpr int kPer = 16 / sizeof(T);
    const int pad = static_cast<int>((reinterpret_cast<uintptr_t>(src) / sizeof(T)) % kPer);
    const int head = min(n, (kPer - pad) % kPer), vecs = (n - head) / kPer, tail0 = head + vecs * kPer;
    float mx = -INFINITY, mn = INFINITY;
    auto take = [&](float x) {
        x = x == x ? x + 0.f : -INFINITY;  // a NaN is no candidate; one zero
        mx = fmaxf(mx, x);
        if (x > -INFINITY) mn = fminf(mn, x);
        return x;
    };
    auto widen = [](T x) -> float {
        if constexpr (sizeof(T) == 4) return x;
        else return __bfloat162float(x);
    };
    if (tid < head) xs[pad + tid] = take(widen(src[tid]));
    if (tid < n - tail0) xs[pad + tail0 + tid] = take(widen(src[tail0 + tid]));
    const uint4 *const src4 = reinterpret_cast<const uint4 *>(src + head);
    constexpr int kLoads = 4;
    for (int v0 = tid; v0 < vecs; v0 += kLoads * kSThreads) {
        uint4 q[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k)
            if (v0 + k * kSThreads < vecs) q[k] = __ldcs(src4 + v0 + k * kSThreads);
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            if (v0 + k * kSThreads >= vecs) break;
            float4 *dst = reinterpret_cast<float4 *>(xs + pad + head) + (v0 + k * kSThreads) * (kPer / 4);
            const uint32_t w[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
            if constexpr (sizeof(T) == 4) {
                dst[0] = make_float4(take(__uint_as_float(w[0])), take(__uint_as_float(w[1])),
                                     take(__uint_as_float(w[2])), take(__uint_as_float(w[3])));
            } else {
#pragma unroll
                for (int e = 0; e < 2; ++e)
                    dst[e] = make_float4(take(__uint_as_float(w[2 * e] << 16)),
                                         take(__uint_as_float(w[2 * e] & 0xFFFF0000u)),
                                         take(__uint_as_float(w[2 * e + 1] << 16)),
                                         take(__uint_as_float(w[2 * e + 1] & 0xFFFF0000u)));
            }
        }
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
    }
    if (lane == 0) s.warp_range[warp] = make_float2(mx, mn);
    __syncthreads();
    if (tid < static_cast<int>(ctas)) {
        for (int w = 0; w < kSWarps; ++w) {
            mx = fmaxf(mx, s.warp_range[w].x);
            mn = fminf(mn, s.warp_range[w].y);
        }
        const uint32_t a = dsmem_addr(smem_u32(&s.range[rank]), tid);
        dsmem_st_f32(a, mx);
        dsmem_st_f32(a + 4, mn);
    }
    cluster_sync_all();
    for (uint32_t c = 0; c < ctas; ++c) {
        mx = fmaxf(mx, s.range[c].x);
        mn = fminf(mn, s.range[c].y);
    }
    const float temperature = p.temperature ? __ldg(p.temperature + r) : 1.f;
    if (mx == -INFINITY) {  // nothing to draw
        if (rank == 0 && tid == 0) {
            p.tokens[r] = -1;
            if (p.logprobs) p.logprobs[r] = -INFINITY;
        }
        return;
    }
    if (!(temperature > 0.f)) {  // the largest logit, the lowest index of several
        uint32_t first = 0xFFFFFFFFu;
        for (int i = tid; i < n; i += kSThreads)
            if (xs[pad + i] == mx) first = min(first, static_cast<uint32_t>(i0 + i));
        first = __reduce_min_sync(0xffffffffu, first);
        if (lane == 0) s.warp_c[warp] = first;
        __syncthreads();
        if (tid == 0) {
            for (int w = 0; w < kSWarps; ++w) first = min(first, s.warp_c[w]);
            st_cluster_u64(dsmem_addr(smem_u32(&s.above[rank]), 0), first);
        }
        cluster_sync_all();
        if (rank == 0 && tid == 0) {
            for (uint32_t c = 0; c < ctas; ++c) first = min(first, static_cast<uint32_t>(s.above[c]));
            p.tokens[r] = static_cast<int32_t>(first);
            if (p.logprobs) p.logprobs[r] = 0.f;
        }
        return;
    }

    // ---- the histogram of weights over z
    const int32_t top_k = p.top_k ? __ldg(p.top_k + r) : 0;
    const float top_p = p.top_p ? __ldg(p.top_p + r) : 1.f, min_p = p.min_p ? __ldg(p.min_p + r) : 0.f;
    const bool by_k = top_k > 0 && top_k < p.vocab, by_m = min_p > 0.f;
    const float ln_min_p = by_m ? logf(min_p) : -INFINITY;
    SRow row;
    row.top = mx;
    row.inv_t = 1.f / temperature;
    const float lowest = fmaxf(row.z(mn), kSFloor);  // (fmaxf of a NaN is the floor)
    row.bin_scale = lowest < 0.f ? (kSBins - 0.5f) / -lowest : 0.f;
    uint64_t above = 0;
    for (int i = tid; i < n; i += kSThreads) {
        const float x = xs[pad + i], z = row.z(x);
        if (!SRow::counts(x, z)) continue;
        const uint64_t w = SRow::weight(z);
        const int b = row.bin(z);
        if (by_k) atomicAdd(&s.cnt[b], 1u);
        add_weight(&s.wl[b], &s.wh[b], w);
        if (by_m && z >= ln_min_p) above += w;
    }
    if (by_m) {
#pragma unroll
        for (int o = 16; o; o >>= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
        if (lane == 0) s.warp_w[warp] = above;
        __syncthreads();
        if (tid == 0) {
            for (int w = 1; w < kSWarps; ++w) above += s.warp_w[w];
            st_cluster_u64(dsmem_addr(smem_u32(&s.above[rank]), 0), above);
        }
    }
    cluster_sync_all();
    push_sums<false>(s, rank, ctas, by_k);
    cluster_sync_all();

    // ---- the cuts and the draw, one search after the other (state of the first CTA)
    enum { kCutK, kCutP, kDraw } stage = kCutK;
    STarget want = {};
    uint64_t sum = 0;  // S so far
    // the next search that there is to do, and its first command
    auto next_search = [&]() {
        if (stage == kCutK && !(by_k && static_cast<uint32_t>(top_k) < s.sum_c[kSBins - 1])) stage = kCutP;
        if (stage == kCutP && !(top_p < 1.f)) stage = kDraw;
        if (stage == kCutK) {
            want = {true, static_cast<uint64_t>(top_k)};
        } else if (stage == kCutP) {
            const double goal = ceil(static_cast<double>(top_p) * static_cast<double>(sum));
            want = {false, goal >= 1.0 ? min(sum, static_cast<uint64_t>(goal)) : 1};
        } else {
            if (by_m) {
                uint64_t m = 0;
                for (uint32_t c = 0; c < ctas; ++c) m += s.above[c];
                sum = min(sum, max(m, uint64_t{1} << 40));
            }
            const double at = static_cast<double>(__ldg(p.uniform + r)) * static_cast<double>(sum);
            want = {false, (at >= 1.0 ? min(sum - 1, static_cast<uint64_t>(at)) : 0) + 1};
        }
        find_bin(s, want);
        if (tid == 0) {
            SCommand c = {};
            c.op = s.got_bin == 0xFFFFFFFFu ? kDone : kGatherBin;
            c.bin = s.got_bin;
            if (c.op == kDone) report_error(p.err, PPAS_DEVERR_TIMEOUT);
            send(s, c, ctas);
        }
    };
    if (rank == 0) {
        uint64_t w0 = s.sum_w[2 * tid], w1 = s.sum_w[2 * tid + 1], w = w0 + w1;
        uint32_t c0 = s.sum_c[2 * tid], c1 = s.sum_c[2 * tid + 1], c = c0 + c1;
        block_scan(s, w, c);
        s.sum_w[2 * tid] = w - w1;
        s.sum_w[2 * tid + 1] = w;
        s.sum_c[2 * tid] = c - c1;
        s.sum_c[2 * tid + 1] = c;
        __syncthreads();
        sum = s.sum_w[kSBins - 1];
        next_search();
    }
    for (int step = 0; step < kSMaxCommands; ++step) {
        // (the first CTA has read every list and count when it gets here)
        cluster_sync_all();
        const SCommand cmd = s.cmd;
        if (cmd.op == kDone) return;
        if (cmd.op == kDivide)
            for (int b = tid; b < kSFine; b += kSThreads) s.cnt[b] = s.wl[b] = s.wh[b] = 0;
        if (tid == 0) {
            s.n = 0;
            s.kmin = 0xFFFFFFFFu;
            s.kmax = 0;
        }
        __syncthreads();
        for (int i = tid; i < n + ((kSThreads - n % kSThreads) % kSThreads); i += kSThreads) {
            const float x = i < n ? xs[pad + i] : -INFINITY;
            const float z = row.z(x);
            const uint32_t key = order_key(x), index = static_cast<uint32_t>(i0 + i);
            const uint64_t place = (static_cast<uint64_t>(key) << kSIndexBits) | index;
            bool in = i < n && SRow::counts(x, z);
            if (cmd.op == kGatherBin) in = in && row.bin(z) == static_cast<int>(cmd.bin);
            else in = in && cmd.lo <= place && place <= cmd.hi;
            if (cmd.op == kDivide) {
                if (in) {
                    const uint32_t b = static_cast<uint32_t>((place - cmd.lo) >> cmd.shift);
                    if (by_k) atomicAdd(&s.cnt[b], 1u);
                    add_weight(&s.wl[b], &s.wh[b], SRow::weight(z));
                }
                continue;
            }
            const uint32_t who = __ballot_sync(0xffffffffu, in);
            if (!who) continue;
            const uint32_t lo = __reduce_min_sync(0xffffffffu, in ? key : 0xFFFFFFFFu);
            const uint32_t hi = __reduce_max_sync(0xffffffffu, in ? key : 0u);
            uint32_t at = 0;
            if (lane == 0) {
                at = atomicAdd(&s.n, static_cast<uint32_t>(__popc(who)));
                atomicMin(&s.kmin, lo);
                atomicMax(&s.kmax, hi);
            }
            at = __shfl_sync(0xffffffffu, at, 0) + __popc(who & ((1u << lane) - 1));
            if (in && at < kSList) s.list[at] = make_uint2(key, index);
        }
        cluster_sync_all();
        if (cmd.op == kDivide) {
            push_sums<true>(s, rank, ctas, by_k);
            cluster_sync_all();
        }
        if (rank != 0) continue;
        SCommand c = {};
        if (cmd.op == kDivide) {
            // the part of the range in which the target lies
            uint64_t w = static_cast<uint64_t>(s.wl[kSFine + tid]) + (static_cast<uint64_t>(s.wh[kSFine + tid]) << 32);
            const uint64_t own_w = w;
            uint32_t cc = s.cnt[kSFine + tid];
            const uint32_t own_c = cc;
            const uint64_t base_w = s.base_w, base_c = s.base_c;
            if (tid == 0) s.got_bin = 0xFFFFFFFFu;
            block_scan(s, w, cc);
            const uint64_t at_w = base_w + w, at_c = base_c + cc;
            if (want.by_count ? (at_c - own_c < want.target && want.target <= at_c)
                              : (at_w - own_w < want.target && want.target <= at_w)) {
                s.got_bin = tid;
                s.base_w = at_w - own_w;
                s.base_c = at_c - own_c;
            }
            __syncthreads();
            if (tid == 0) {
                c.op = s.got_bin == 0xFFFFFFFFu ? kDone : kGatherRange;
                c.lo = cmd.lo + (static_cast<uint64_t>(s.got_bin) << cmd.shift);
                c.hi = min(cmd.hi, c.lo + (uint64_t{1} << cmd.shift) - 1);
                if (c.op == kDone) report_error(p.err, PPAS_DEVERR_TIMEOUT);
                send(s, c, ctas);
            }
            continue;
        }
        uint32_t total = 0, kmin = 0xFFFFFFFFu, kmax = 0;
        for (uint32_t q = 0; q < ctas; ++q) {
            total += ld_cluster_u32(dsmem_addr(smem_u32(&s.n), q));
            kmin = min(kmin, ld_cluster_u32(dsmem_addr(smem_u32(&s.kmin), q)));
            kmax = max(kmax, ld_cluster_u32(dsmem_addr(smem_u32(&s.kmax), q)));
        }
        if (total > kSList) {
            __syncthreads();
            if (tid == 0) {
                c.op = kDivide;
                c.lo = static_cast<uint64_t>(kmin) << kSIndexBits;
                c.hi = (static_cast<uint64_t>(kmax) << kSIndexBits) | ((1u << kSIndexBits) - 1);
                if (cmd.op == kGatherRange) {
                    c.lo = max(c.lo, cmd.lo);
                    c.hi = min(c.hi, cmd.hi);
                }
                // at most kSFine parts of 2^shift places
                const int bits = 64 - __clzll(static_cast<long long>(c.hi - c.lo));
                c.shift = bits > 9 ? bits - 9 : 0;
                send(s, c, ctas);
            }
            continue;
        }
        rank_list(s, row, want, ctas, total);
        if (s.got_index == 0xFFFFFFFFu || stage == kDraw) {
            if (tid == 0) {
                if (s.got_index == 0xFFFFFFFFu) {
                    report_error(p.err, PPAS_DEVERR_TIMEOUT);
                } else {
                    p.tokens[r] = static_cast<int32_t>(s.got_index);
                    const uint64_t mass = s.got_mass;
                    // a likely token's log from what is left of the sum, which is accurate near 0; another's
                    // from its z, which a weight of few units of 2^-40 has lost the last bits of
                    if (p.logprobs)
                        p.logprobs[r] = 2 * mass > sum
                                            ? log1pf(-(static_cast<float>(sum - mass) / static_cast<float>(sum)))
                                            : s.got_z - logf(static_cast<float>(sum) * 0x1p-40f);
                }
                send(s, c, ctas);  // kDone
            }
            continue;
        }
        sum = s.got_w;
        stage = stage == kCutK ? kCutP : kDraw;
        next_search();
    }
}
static_assert(kSFine == 1 << 9, "shift of a divided range");

size_t sample_smem_bytes(int32_t chunk) {
    // up to 7 values of padding in front of the row's part
    return (sizeof(SShared) + 15) / 16 * 16 + (static_cast<size_t>(chunk) + 8) * sizeof(float);
}

static std::atomic<uint64_t> g_sample_smem_set[2] = {};

cudaError_t launch_sample(SampleParams p, int32_t n_rows, bool bf16, cudaStream_t st) {
    constexpr int kLimit = 232448;
    const auto kernel = bf16 ? sample_kernel<__nv_bfloat16> : sample_kernel<float>;
    const cudaError_t e = ensure_smem_limit(kernel, kLimit, g_sample_smem_set[bf16]);
    if (e != cudaSuccess) return e;
    const int32_t sms = device_sm_count();
    auto chunk_of = [&](int32_t c) { return ((p.vocab + c - 1) / c + 7) / 8 * 8; };
    // as many CTAs a row as one round of the SMs holds, at least as many as its shared memory takes
    int32_t c = 1;
    while (c < kSMaxCluster && (sample_smem_bytes(chunk_of(c)) > static_cast<size_t>(kLimit) ||
                                (2 * c * static_cast<int64_t>(n_rows) <= sms && chunk_of(c) > 1024)))
        c *= 2;
    p.chunk = chunk_of(c);
    const size_t smem = sample_smem_bytes(p.chunk);
    if (smem > static_cast<size_t>(kLimit)) return cudaErrorInvalidValue;
    PdlLaunch l(dim3(static_cast<unsigned>(n_rows) * c), dim3(kSThreads), smem, st);
    cudaLaunchAttribute attrs[2] = {l.attr[0], {}};
    if (c > 1) {
        attrs[1].id = cudaLaunchAttributeClusterDimension;
        attrs[1].val.clusterDim.x = static_cast<unsigned>(c);
        attrs[1].val.clusterDim.y = 1;
        attrs[1].val.clusterDim.z = 1;
        l.cfg.attrs = attrs;
        l.cfg.numAttrs = 2;
    }
    return cudaLaunchKernelEx(&l.cfg, kernel, p);
}

}  // namespace ppas

using namespace ppas;

extern "C" ppas_status ppas_sample_tokens(const void *logits, int32_t logits_are_bf16, int64_t row_stride,
                                          int32_t n_rows, int32_t vocab, const float *d_temperature,
                                          const int32_t *d_top_k, const float *d_top_p, const float *d_min_p,
                                          const float *d_uniform, int32_t *d_tokens, float *d_logprobs,
                                          int32_t *d_err_flag, void *stream) {
    if (n_rows < 0 || vocab < 1) return PPAS_ERR_INVALID_ARG;
    if (vocab > kSMaxVocab || n_rows > INT32_MAX / kSMaxCluster) return PPAS_ERR_UNSUPPORTED;
    if (n_rows == 0) return PPAS_OK;
    if (row_stride < vocab || !logits || !d_uniform || !d_tokens) return PPAS_ERR_INVALID_ARG;
    auto on = [](const void *x, uintptr_t n) { return (reinterpret_cast<uintptr_t>(x) & (n - 1)) == 0; };
    if (!on(logits, logits_are_bf16 ? 2 : 4) || !on(d_temperature, 4) || !on(d_top_k, 4) || !on(d_top_p, 4) ||
        !on(d_min_p, 4) || !on(d_uniform, 4) || !on(d_tokens, 4) || !on(d_logprobs, 4) || !on(d_err_flag, 4))
        return PPAS_ERR_INVALID_ARG;
    SampleParams p = {};
    p.logits = logits;
    p.row_stride = row_stride;
    p.temperature = d_temperature;
    p.top_k = d_top_k;
    p.top_p = d_top_p;
    p.min_p = d_min_p;
    p.uniform = d_uniform;
    p.tokens = d_tokens;
    p.logprobs = d_logprobs;
    p.err = d_err_flag;
    p.vocab = vocab;
    return launch_sample(p, n_rows, logits_are_bf16 != 0, static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? PPAS_OK
               : PPAS_ERR_CUDA;
}
