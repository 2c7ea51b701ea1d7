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
// A cluster of CTAs takes a row: its maximum, then a histogram, then a few of its
// tokens, three passes over logits that stay in shared memory where they fit (in
// L2 where not).  All three cuts are the same question, at which token a running
// sum in the order reaches a target, and need no sort: the histogram of weights
// over bins of z (linear, so the bins fill evenly and few additions collide),
// summed over the cluster, gives the bins of all three targets; their tokens
// (mostly some tens) go to the first CTA, which ranks them, or divides them further by the
// bits of (x, index) where they are hundreds.  Bins with more than that (ties, flat
// rows) are divided so by the whole cluster first.
//
// Few rows are bound by the chain of passes, exchanges and searches: 1 row x 152000
// 12.7 us a call, 32 x 128000 bf16 20.2, 64 x 32003 15.4.  Many are bound by phases
// that do not overlap: 256 x 152000 in 105 us, 1.5 TB/s of the logits' own bytes, at
// 42 instructions a logit (25 of them the histogram's, of which exp is 8) with the
// issue slots busy half of the time and DRAM a fifth of it, for the two CTAs of an SM
// read, add up and gather in step, and 512 CTAs take two rounds of 304.
#include <float.h>
#include <math.h>

#include <type_traits>

#include "ppas_device.cuh"
#include "ppas_internal.h"

namespace ppas {
namespace {

constexpr int kSThreads = 512;
constexpr int kSWarps = kSThreads / 32;
constexpr int kSBins = 1024;      // bins of z
constexpr int kSFine = 512;       // bins of a bin's (x, index)
// tokens of a search that the first CTA takes (64 rows of 152000 logits that vary by
// 1: 42.3 us, with 512 of them 70.4; 1 row by 0.5: 19.4 and 29.3)
constexpr int kSList = 1024;
constexpr int kOfThread = 2;      // of these a thread has
constexpr int kSRank = 128;       // tokens of a search that are ranked by comparing all pairs
constexpr int kSIndexBits = 18;   // vocabularies of up to 2^18 tokens
constexpr int kSMaxCluster = 16;
constexpr float kSFloor = -28.f;  // z below this: W = 0 (exp(-28) 2^40 < 1)
// A search divides its 50 bits of (x, index) by 2^9 until 2^10 places are left, at
// most 5 times, and gathers before and after: three searches and the end take 34.
constexpr int kSMaxCommands = 40;
enum { kCutK, kCutP, kDraw, kStages };  // the searches
static_assert(kSMaxVocab == 1 << kSIndexBits, "index bits");
static_assert(kSBins % (2 * kSMaxCluster) == 0 && kSFine % kSMaxCluster == 0 && kSBins == 2 * kSFine &&
                  kSBins == 2 * kSThreads && kSFine == kSThreads && kSList == kOfThread * kSThreads && kStages * kSRank <= kSThreads,
              "the scans give each thread two bins or one");

enum : uint32_t { kDone, kGather, kDivide };

struct SCommand {
    uint32_t op, bin;
    uint64_t lo, hi;  // range of (x, index) in the bin
    uint32_t shift;
    float x_lo, x_hi;  // no token outside these belongs
    uint32_t pad;
};

// what the histogram alone tells of all three searches
struct SBinsOf {
    int32_t lo[kStages], hi[kStages];      // the target's bin is one of these; lo > hi: no such cut
    float x_lo[kStages], x_hi[kStages];    // no token outside these is in them
};

struct SShared {
    // this CTA's histogram (divided bins: the first kSFine, and behind them the
    // first CTA's sums over the cluster), later its tokens of the three searches'
    // bins (first CTA: the cluster's)
    union {
        struct {
            uint32_t cnt[kSBins], wl[kSBins], wh[kSBins];
        };
        uint64_t lists[kStages][kSList];  // places (key, index)
        uint64_t list[kSList];            // tokens of a single search's bin
    };
    uint64_t sum_w[kSBins];                // first CTA: the bins' sums over the cluster, then their running sums
    uint32_t sum_c[kSBins];
    uint64_t run_w[kStages][kSRank];       // running weights of the ranked tokens
    // first CTA: the histogram of a list, or (place, weight) of the tokens to rank
    union {
        struct {
            uint32_t fine_c[kSFine], fine_l[kSFine], fine_h[kSFine];
        };
        ulonglong2 ranked[kStages][kSRank];
    };
    SBinsOf bins;
    uint32_t ns[kStages], at[kStages];     // tokens in the lists (first CTA: all of them), this CTA's place there
    float2 range[kSMaxCluster];            // (max, about the least finite one) of each CTA
    uint64_t above[kSMaxCluster];          // weight with z >= ln p_min, or the lowest index of the maximum
    uint64_t warp_w[kSWarps];
    uint32_t warp_c[kSWarps];
    float2 warp_range[kSWarps];
    uint32_t n;                            // of this CTA's gathered tokens
    uint32_t all_n[kSMaxCluster];          // first CTA: every CTA's
    SCommand cmd;
    uint64_t target;
    uint64_t base_w, base_c, got_w, got_mass;  // first CTA: sums before the bin, what a search found
    uint32_t got_bin, got_index, got_n;
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
__device__ __forceinline__ uint32_t atom_cluster_add(uint32_t a, uint32_t v) {
    uint32_t old;
    asm volatile("atom.shared::cluster.add.u32 %0, [%1], %2;" : "=r"(old) : "r"(a), "r"(v) : "memory");
    return old;
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

// The largest finite logit of type T, as which +inf counts.  (Of bf16 not FLT_MAX,
// which is none of its values: place_range would leave it out.)
template <class T>
constexpr float kLargest = sizeof(T) == 4 ? FLT_MAX : 0x1.FEp127f;

// The places of the logits of type T from x_hi down to x_lo.  (Of bf16 logits a
// bin of z holds one value or two, of many tokens each: with the range closed
// to them the first division tells tokens apart, and not 2^16 values that are
// not there.)
template <class T>
__device__ __forceinline__ void place_range(float x_lo, float x_hi, uint64_t &lo, uint64_t &hi) {
    if constexpr (sizeof(T) == 2) {
        const uint32_t a = __float_as_uint(x_lo), b = __float_as_uint(x_hi);
        x_lo = __uint_as_float((a & 0xFFFF0000u) + (!(a >> 31) && (a & 0xFFFFu) ? 0x10000u : 0u));
        x_hi = __uint_as_float((b & 0xFFFF0000u) + ((b >> 31) && (b & 0xFFFFu) ? 0x10000u : 0u));
    }
    lo = static_cast<uint64_t>(order_key(x_hi + 0.f)) << kSIndexBits;
    hi = (static_cast<uint64_t>(order_key(x_lo + 0.f)) << kSIndexBits) | (kSMaxVocab - 1);
}

__device__ __forceinline__ float2 both(float x) { return make_float2(x, x); }
__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return fma2(a, b, both(-0.f)); }
__device__ __forceinline__ float2 fma2_rz(float2 a, float2 b, float2 c) {
    float2 r;
    asm("{\n\t.reg .b64 ra, rb, rc, rd;\n\t"
        "mov.b64 ra, {%2, %3};\n\tmov.b64 rb, {%4, %5};\n\tmov.b64 rc, {%6, %7};\n\t"
        "fma.rz.f32x2 rd, ra, rb, rc;\n\tmov.b64 {%0, %1}, rd;\n\t}"
        : "=f"(r.x), "=f"(r.y)
        : "f"(a.x), "f"(a.y), "f"(b.x), "f"(b.y), "f"(c.x), "f"(c.y));
    return r;
}

struct SRow {
    float top, inv_t, lowest, bin_scale;  // all finite; z = lowest, and all below, is in bin kSBins - 1
    float width;                          // x a bin (infinite where there is one bin)
    __device__ __forceinline__ float z(float x) const { return (x - top) * inv_t; }
    // (conversions between floats and whole numbers share a slow unit with exp:
    // here and in weight2 additions do most of their work)
    __device__ __forceinline__ int bin(float z_) const {
        return __float_as_int(fmaf(fmaxf(z_, lowest), -bin_scale, 0x1p23f)) - 0x4B000000;
    }
    // x of the tokens in bin b, and a little more: the bins' edges in x but for roundings
    __device__ __forceinline__ void bin_range(int b, float &lo, float &hi) const {
        const float slack = 1e-5f * (fabsf(top) + (static_cast<float>(b) + 1.f) * width) + 1e-30f;
        lo = top - (static_cast<float>(b) + 0.5f) * width - slack;
        hi = top - (static_cast<float>(b) - 0.5f) * width + slack;
        if (b == kSBins - 1 || !(lo < hi)) lo = -INFINITY;
        if (b == 0 || !(lo < hi)) hi = INFINITY;
    }
    // tokens that can be drawn or counted (a -inf is below the floor)
    __device__ __forceinline__ static bool counts(float z_) { return z_ > kSFloor; }
    // floor(e 2^40), low and high half, e = exp(z) <= 1: h + 2^23 = floor(2^8 e + 2^23),
    // then 2^40 e - 2^32 h, every step exact
    __device__ __forceinline__ static uint2 weight2(float e) {
        const float h = __fmaf_rz(e, 256.f, 0x1p23f);
        return make_uint2(__float2uint_rz(fmaf(e, 0x1p40f, fmaf(h, -0x1p32f, 0x1p55f))), __float_as_uint(h) & 0x7FFFFFu);
    }
};

// SRow::z, weight2 and bin of two values, the same operations on both at once
// (256 x 152000: 108.6 -> 106.6 us)
struct SPair {
    float2 z;
    uint2 w0, w1;
    int b0, b1;
    __device__ __forceinline__ SPair(const SRow &row, float x0, float x1) {
        z = mul2(add2(make_float2(x0, x1), both(-row.top)), both(row.inv_t));
        const float2 e = make_float2(expf(z.x), expf(z.y));
        const float2 h = fma2_rz(e, both(256.f), both(0x1p23f));
        const float2 l = fma2(e, both(0x1p40f), fma2(h, both(-0x1p32f), both(0x1p55f)));
        w0 = make_uint2(__float2uint_rz(l.x), __float_as_uint(h.x) & 0x7FFFFFu);
        w1 = make_uint2(__float2uint_rz(l.y), __float_as_uint(h.y) & 0x7FFFFFu);
        const float2 b = fma2(make_float2(fmaxf(z.x, row.lowest), fmaxf(z.y, row.lowest)), both(-row.bin_scale),
                              both(0x1p23f));
        b0 = __float_as_int(b.x) - 0x4B000000;
        b1 = __float_as_int(b.y) - 0x4B000000;
    }
};

// Adds a weight's high half, and the carry of its low half (what was there before
// is `old`), where there is one of them: one predicated addition.  (Branches for
// the two took 13 instructions a logit of the histogram's 42.)
__device__ __forceinline__ void add_high(uint32_t *wh, uint32_t old, uint2 w) {
    asm volatile(
        "{\n\t.reg .pred p;\n\t.reg .u32 n, h;\n\t"
        "add.cc.u32 n, %1, %2;\n\t"
        "addc.u32 h, %3, 0;\n\t"
        "setp.ne.u32 p, h, 0;\n\t"
        "@p red.shared::cta.add.u32 [%0], h;\n\t}" ::"r"(smem_u32(wh)),
        "r"(old), "r"(w.x), "r"(w.y)
        : "memory");
}
__device__ __forceinline__ void add_weight(uint32_t *wl, uint32_t *wh, uint2 w) {
    add_high(wh, atomicAdd(wl, w.x), w);
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
    uint64_t before_w = 0;
    uint32_t before_c = 0;
#pragma unroll
    for (int i = 0; i < kSWarps; ++i) {
        const uint64_t a = s.warp_w[i];
        const uint32_t b = s.warp_c[i];
        before_w += i < warp ? a : 0;
        before_c += i < warp ? b : 0;
    }
    w += before_w;
    c += before_c;
}

// Sums the cluster's histograms and leaves the bins' sums in the first CTA:
// each CTA adds up the bins [rank * n / ctas, (rank + 1) * n / ctas).
template <bool kFine>
__device__ __forceinline__ void push_sums(SShared &s, uint32_t rank, uint32_t ctas, bool counted) {
    constexpr int n = kFine ? kSFine : kSBins;
    const int per = n / static_cast<int>(ctas);
    for (int i = threadIdx.x; i < per; i += kSThreads) {
        const int b = static_cast<int>(rank) * per + i;
        uint32_t lo[kSMaxCluster], hi[kSMaxCluster], nc[kSMaxCluster];
#pragma unroll
        for (uint32_t r = 0; r < kSMaxCluster; ++r) {
            lo[r] = hi[r] = nc[r] = 0;
            if (r < ctas) {
                lo[r] = ld_cluster_u32(dsmem_addr(smem_u32(&s.wl[b]), r));
                hi[r] = ld_cluster_u32(dsmem_addr(smem_u32(&s.wh[b]), r));
                if (counted) nc[r] = ld_cluster_u32(dsmem_addr(smem_u32(&s.cnt[b]), r));
            }
        }
        uint64_t w = 0;
        uint32_t c = 0;
#pragma unroll
        for (int r = 0; r < kSMaxCluster; ++r) {
            w += static_cast<uint64_t>(lo[r]) + (static_cast<uint64_t>(hi[r]) << 32);
            c += nc[r];
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

// The first of m <= 1024 running sums that reaches the target (the last where
// none does), by a whole warp: 32 of them, then the ones before the first of those.
template <class T>
__device__ __forceinline__ int reach(const T *sums, int m, uint64_t target) {
    const int lane = threadIdx.x & 31, stride = (m + 31) / 32;
    const uint32_t far = __ballot_sync(0xffffffffu, sums[min((lane + 1) * stride, m) - 1] >= target);
    const int first = far ? __ffs(far) - 1 : 31;
    const int at = min(first * stride + min(lane, stride - 1), m - 1);
    const uint32_t near = __ballot_sync(0xffffffffu, sums[at] >= target);
    return min(near ? first * stride + __ffs(near) - 1 : m - 1, m - 1);
}
// running weights to reach: p of S, and the draw's (64-bit floating point is
// slow here: by single warps)
__device__ __forceinline__ uint64_t cut_target(float top_p, uint64_t sum) {
    const double goal = ceil(static_cast<double>(top_p) * static_cast<double>(sum));
    return goal >= 1.0 ? min(sum, static_cast<uint64_t>(goal)) : 1;
}
__device__ __forceinline__ uint64_t draw_target(float uniform, uint64_t sum) {
    const double at = static_cast<double>(uniform) * static_cast<double>(sum);
    return (at >= 1.0 ? min(sum - 1, static_cast<uint64_t>(at)) : 0) + 1;
}

// the first CTA's command, written into every CTA of the cluster (a thread each)
__device__ __forceinline__ void send(SShared &s, const SCommand &c, uint32_t ctas) {
    if (threadIdx.x >= ctas) return;
    const uint32_t a = dsmem_addr(smem_u32(&s.cmd), threadIdx.x);
    st_cluster_u32(a + offsetof(SCommand, op), c.op);
    st_cluster_u32(a + offsetof(SCommand, bin), c.bin);
    st_cluster_u64(a + offsetof(SCommand, lo), c.lo);
    st_cluster_u64(a + offsetof(SCommand, hi), c.hi);
    st_cluster_u32(a + offsetof(SCommand, shift), c.shift);
    dsmem_st_f32(a + offsetof(SCommand, x_lo), c.x_lo);
    dsmem_st_f32(a + offsetof(SCommand, x_hi), c.x_hi);
}

// Entry `at` of the cluster's n gathered tokens (lists of all_n(rank)
// tokens each, at the same place in every CTA); behind every token past them.
template <class Count>
__device__ __forceinline__ uint64_t list_entry(const uint64_t *list, uint32_t at, uint32_t n, uint32_t ctas, Count all_n) {
    if (at >= n) return ~uint64_t{0};
    uint32_t r = 0;
    for (; r + 1 < ctas; ++r) {
        const uint32_t nr = all_n(r);
        if (at < nr) break;
        at -= nr;
    }
    return ld_cluster_u64(dsmem_addr(smem_u32(list + at), r));
}

// Finds among n gathered tokens (places v, a thread's kSThreads apart, all within
// lo .. hi) the one at which the target is reached, s.base_w and s.base_c being the sums before
// them: got_w (the running weight up to it), got_mass, got_index, got_z.  Their
// places are spread over kSFine bins, and the bin with the target again, until
// it holds one token: mostly once or twice.  (Sorting 300 of them took 4 us,
// bound by the shuffles; this takes 1.)
__device__ __forceinline__ void search_list(SShared &s, const SRow &row, const STarget &t,
                                            const uint64_t (&v)[kOfThread], uint32_t n, uint64_t lo, uint64_t hi) {
    const uint32_t i = threadIdx.x;
    float z[kOfThread];
    uint2 mass[kOfThread];
#pragma unroll
    for (int k = 0; k < kOfThread; ++k) {
        z[k] = row.z(key_value(static_cast<uint32_t>(v[k] >> kSIndexBits)));
        mass[k] = SRow::weight2(expf(z[k]));
    }
    if (i == 0) s.got_index = 0xFFFFFFFFu;
    uint64_t base_w = s.base_w, base_c = s.base_c;
    for (int level = 0; level < 8; ++level) {
        const int bits = 64 - __clzll(static_cast<long long>(hi - lo));
        const int shift = bits > 9 ? bits - 9 : 0;  // kSFine parts of 2^shift places
        s.fine_c[i] = s.fine_l[i] = s.fine_h[i] = 0;
        __syncthreads();
        if (i == 0) s.got_bin = 0xFFFFFFFFu;  // (every thread has read the one of the level before)
        uint32_t b[kOfThread];
#pragma unroll
        for (int k = 0; k < kOfThread; ++k) {
            const bool in = i + k * kSThreads < n && lo <= v[k] && v[k] <= hi;
            b[k] = in ? static_cast<uint32_t>((v[k] - lo) >> shift) : 0xFFFFFFFFu;
            if (in) {
                atomicAdd(&s.fine_c[b[k]], 1u);
                add_weight(&s.fine_l[b[k]], &s.fine_h[b[k]], mass[k]);
            }
        }
        __syncthreads();
        const uint64_t own_w = s.fine_l[i] + (static_cast<uint64_t>(s.fine_h[i]) << 32);
        const uint32_t own_c = s.fine_c[i];
        uint64_t w = own_w;
        uint32_t c = own_c;
        block_scan(s, w, c);
        const uint64_t at_w = base_w + w, at_c = base_c + c;
        if (t.by_count ? (at_c - own_c < t.target && t.target <= at_c) : (at_w - own_w < t.target && t.target <= at_w)) {
            s.got_bin = i;
            s.got_n = own_c;
            s.got_w = at_w;
            s.base_w = at_w - own_w;
            s.base_c = at_c - own_c;
        }
        __syncthreads();
        const uint32_t got = s.got_bin;
        if (got == 0xFFFFFFFFu) return;
        if (s.got_n == 1) {
#pragma unroll
            for (int k = 0; k < kOfThread; ++k)
                if (b[k] == got) {
                    s.got_mass = (static_cast<uint64_t>(mass[k].y) << 32) | mass[k].x;
                    s.got_index = static_cast<uint32_t>(v[k]) & (kSMaxVocab - 1);
                    s.got_z = z[k];
                }
            __syncthreads();
            return;
        }
        base_w = s.base_w;
        base_c = s.base_c;
        lo += static_cast<uint64_t>(got) << shift;
        hi = min(hi, lo + (uint64_t{1} << shift) - 1);
    }
}

// Puts the tokens of each search (at most kSRank) in order, with their running
// weights beside them.  (A token's rank and running weight are sums over the tokens
// up to it in the order, and of few tokens every pair can be compared: no levels, no
// scans, and all three searches at once: 32 x 128000 bf16 27.6 -> 20.5 us.)
__device__ __forceinline__ void rank_lists(SShared &s, const SRow &row) {
    const int j = threadIdx.x / kSRank, i = threadIdx.x % kSRank;
    const int n = j < kStages ? static_cast<int>(s.ns[j]) : 0;
    uint64_t v = 0;
    if (i < n) {
        v = s.lists[j][i];
        const uint2 w = SRow::weight2(expf(row.z(key_value(static_cast<uint32_t>(v >> kSIndexBits)))));
        s.ranked[j][i] = make_ulonglong2(v, (static_cast<uint64_t>(w.y) << 32) | w.x);
    }
    __syncthreads();
    if (i < n) {
        uint64_t w = 0;
        int at = -1;
#pragma unroll 4
        for (int e = 0; e < n; ++e) {
            const ulonglong2 o = s.ranked[j][e];
            const bool before = o.x <= v;
            w += before ? o.y : 0;
            at += before;
        }
        s.lists[j][at] = v;
        s.run_w[j][at] = w;
    }
    __syncthreads();
}

}  // namespace

template <int n>
using Loads = std::integral_constant<int, n>;

// kResident: the row's part stays in shared memory; otherwise each pass reads it
// again, from L2 for the most part.
template <class T, bool kResident>
__global__ void __launch_bounds__(kSThreads, 2) sample_kernel(const __grid_constant__ SampleParams p) {
    extern __shared__ __align__(16) uint8_t sample_smem[];
    SShared &s = *reinterpret_cast<SShared *>(sample_smem);
    float *const xs = reinterpret_cast<float *>(sample_smem + (sizeof(SShared) + 15) / 16 * 16);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t ctas = cluster_nctarank(), rank = ctas > 1 ? cluster_ctarank() : 0;
    const int32_t r = blockIdx.x / ctas;
    // (the other half of this barrier is before the first store to another CTA)
    cluster_arrive_relaxed();
    for (int b = tid; b < kSBins; b += kSThreads) s.cnt[b] = s.wl[b] = s.wh[b] = 0;
    grid_dep_launch();
    grid_dep_wait();
    const float temperature = p.temperature ? __ldg(p.temperature + r) : 1.f;
    const int32_t top_k = p.top_k ? __ldg(p.top_k + r) : 0;
    const float top_p = p.top_p ? __ldg(p.top_p + r) : 1.f, min_p = p.min_p ? __ldg(p.min_p + r) : 0.f;
    const float uniform = __ldg(p.uniform + r);

    // ---- this CTA's part of the row, 16 bytes at a time between its first and last 16-byte boundary
    const int32_t i0 = min(static_cast<int32_t>(rank) * p.chunk, p.vocab);
    const int32_t n = min(p.chunk, p.vocab - i0);
    const T *const src = static_cast<const T *>(p.logits) + r * p.row_stride + i0;
    constexpr int kPer = 16 / sizeof(T);
    const int pad = static_cast<int>((reinterpret_cast<uintptr_t>(src) / sizeof(T)) % kPer);
    const int head = min(n, (kPer - pad) % kPer), vecs = (n - head) / kPer, tail0 = head + vecs * kPer;
    const uint4 *const src4 = reinterpret_cast<const uint4 *>(src + head);
    const int n4 = (pad + n + 3) / 4;  // resident: four values at a time, from xs on
    const float4 *const xs4 = reinterpret_cast<const float4 *>(xs);
    auto widen = [](T x) -> float {
        if constexpr (sizeof(T) == 4) return x;
        else return __bfloat162float(x);
    };
    // f(four values, index of the first in the row) over the part as it lies in
    // global memory, in batches of kLoads x 16 bytes a thread, all under way at
    // once; then done(place of the batch in `tops`), where wanted(place) was true
    auto stream = [&](auto loads, auto &&f, auto &&wanted, auto &&done) {
        constexpr int kLoads = decltype(loads)::value;
        // what is before the first and after the last boundary, a value a thread
        const int ends = head + n - tail0;
        if (tid < ends) {
            const int at = tid < head ? tid : tail0 + tid - head;
            const float x[4] = {widen(src[at]), -INFINITY, -INFINITY, -INFINITY};
            f(x, i0 + at);
        }
        int place = tid;
        for (int v0 = tid; v0 < vecs; v0 += kLoads * kSThreads, place += kSThreads) {
            if (!wanted(place)) continue;
            uint4 q[kLoads];
#pragma unroll
            for (int k = 0; k < kLoads; ++k)
                if (v0 + k * kSThreads < vecs) q[k] = __ldg(src4 + v0 + k * kSThreads);
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                if (v0 + k * kSThreads >= vecs) break;
                const int at = i0 + head + (v0 + k * kSThreads) * kPer;
                const uint32_t w[4] = {q[k].x, q[k].y, q[k].z, q[k].w};
                if constexpr (sizeof(T) == 4) {
                    const float x[4] = {__uint_as_float(w[0]), __uint_as_float(w[1]), __uint_as_float(w[2]),
                                        __uint_as_float(w[3])};
                    f(x, at);
                } else {
#pragma unroll
                    for (int e = 0; e < 2; ++e) {
                        const float x[4] = {__uint_as_float(w[2 * e] << 16), __uint_as_float(w[2 * e] & 0xFFFF0000u),
                                            __uint_as_float(w[2 * e + 1] << 16),
                                            __uint_as_float(w[2 * e + 1] & 0xFFFF0000u)};
                        f(x, at + 4 * e);
                    }
                }
            }
            done(place);
        }
    };
    auto always = [](int) { return true; };
    auto nothing = [](int) {};
    // a pass over the part once the maximum is known
    auto pass = [&](auto loads, auto &&f) {
        if constexpr (kResident) {
            for (int i = tid; i < n4; i += kSThreads) {
                const float4 q = xs4[i];
                const float x[4] = {q.x, q.y, q.z, q.w};
                f(x, i0 - pad + 4 * i);
            }
        } else {
            stream(loads, f, always, nothing);
        }
    };
    float mx = -INFINITY, mn = INFINITY, top = -INFINITY;
    // (a maximum passes over NaNs; the least of every fourth value will do to
    // spread the bins, for what is below goes to the last one)
    stream(Loads<4>{}, [&](const float(&x)[4], int at) {
#pragma unroll
        for (int k = 0; k < 4; ++k) top = fmaxf(top, x[k]);
        if (x[0] > -INFINITY) mn = fminf(mn, x[0]);
        if constexpr (kResident) {
            const int to = at - i0 + pad;
            if (at - i0 < head || at - i0 >= tail0) xs[to] = x[0];
            else *reinterpret_cast<float4 *>(xs + to) = make_float4(x[0], x[1], x[2], x[3]);
        }
    }, always, [&](int place) {
        if constexpr (!kResident) {  // each batch's maximum, of which the gather makes use
            xs[place] = top;
            mx = fmaxf(mx, top);
            top = -INFINITY;
        }
    });
    mx = fmaxf(mx, top);
    if constexpr (kResident) {
        if (tid < pad) xs[tid] = -INFINITY;
        if (tid < 4 * n4 - pad - n) xs[pad + n + tid] = -INFINITY;
    }
#pragma unroll
    for (int o = 16; o; o >>= 1) {
        mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, o));
        mn = fminf(mn, __shfl_xor_sync(0xffffffffu, mn, o));
    }
    if (lane == 0) s.warp_range[warp] = make_float2(mx, mn);
    __syncthreads();
    // every CTA of the cluster has started: its shared memory may be written
    // (the pass over the logits hides the wait)
    cluster_wait();
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
    if (mx == -INFINITY) {  // nothing to draw
        if (rank == 0 && tid == 0) {
            p.tokens[r] = -1;
            if (p.logprobs) p.logprobs[r] = -INFINITY;
        }
        return;
    }
    const float largest = fminf(mx, kLargest<T>);
    if (!(temperature > 0.f)) {  // the largest logit, the lowest index of several
        uint32_t first = 0xFFFFFFFFu;
        pass(Loads<4>{}, [&](const float(&x)[4], int at) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (x[k] >= largest) first = min(first, static_cast<uint32_t>(at + k));
        });
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
    const bool by_k = top_k > 0 && top_k < p.vocab, by_m = min_p > 0.f;
    const float ln_min_p = by_m ? logf(min_p) : -INFINITY;
    SRow row;
    // all finite, 1 / T too
    row.top = largest;
    row.inv_t = fminf(1.f / temperature, FLT_MAX);
    mn = fminf(mn, row.top);
    // a logit as the passes see it (a NaN as -inf)
    auto logit = [](float x) { return fminf(fmaxf(x, -INFINITY), kLargest<T>); };
    // (lowest * bin_scale is 1023 but for two roundings, so that no bin is past the last)
    row.lowest = fmaxf(row.z(mn), kSFloor);
    row.bin_scale = row.lowest < 0.f ? fminf((kSBins - 1.f) / -row.lowest, 1e30f) : 0.f;
    row.width = 1.f / (row.inv_t * row.bin_scale);
    uint64_t above = 0;
    // (a weight of 0 adds nothing wherever it goes: no branch, so that the
    // additions of several values are under way at once)
    pass(Loads<4>{}, [&](const float(&x)[4], int) {
        float z[4];
        uint2 w[4];
        uint32_t old[4];
        int b[4];
#pragma unroll
        for (int k = 0; k < 4; k += 2) {
            const SPair a(row, logit(x[k]), logit(x[k + 1]));
            z[k] = a.z.x;
            z[k + 1] = a.z.y;
            w[k] = a.w0;
            w[k + 1] = a.w1;
            b[k] = a.b0;
            b[k + 1] = a.b1;
        }
        if (by_k) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if (SRow::counts(z[k])) atomicAdd(&s.cnt[b[k]], 1u);
        }
#pragma unroll
        for (int k = 0; k < 4; ++k) old[k] = atomicAdd(&s.wl[b[k]], w[k].x);
#pragma unroll
        for (int k = 0; k < 4; ++k) add_high(&s.wh[b[k]], old[k], w[k]);
        if (by_m) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                above += z[k] >= ln_min_p ? (static_cast<uint64_t>(w[k].y) << 32) | w[k].x : 0;
        }
    });
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

    // ---- the cuts and the draw (state of the first CTA)
    int stage = kCutK;
    STarget want = {};
    uint64_t sum = 0;  // S so far
    uint64_t m_sum = ~uint64_t{0};
    // a search without a result, by one thread: no old token stays
    auto found_none = [&]() {
        report_error(p.err, PPAS_DEVERR_SEARCH);
        p.tokens[r] = -1;
        if (p.logprobs) p.logprobs[r] = -INFINITY;
    };
    // the search that comes next: its stage, and what it has to reach
    auto next_target = [&]() {
        if (stage == kCutK && !(by_k && static_cast<uint32_t>(top_k) < s.sum_c[kSBins - 1])) stage = kCutP;
        if (stage == kCutP && !(top_p < 1.f)) stage = kDraw;
        if (stage == kDraw) sum = min(sum, m_sum);
        if (warp == 0) {
            const uint64_t t = stage == kCutK   ? static_cast<uint64_t>(top_k)
                               : stage == kCutP ? cut_target(top_p, sum)
                                                : draw_target(uniform, sum);
            if (lane == 0) s.target = t;
        }
        __syncthreads();
        want = {stage == kCutK, s.target};
    };
    auto next_search = [&]() {
        next_target();
        find_bin(s, want);
        SCommand c = {};
        c.op = s.got_bin == 0xFFFFFFFFu ? kDone : kGather;
        c.bin = s.got_bin;
        row.bin_range(static_cast<int>(c.bin), c.x_lo, c.x_hi);
        place_range<T>(c.x_lo, fminf(c.x_hi, row.top), c.lo, c.hi);
        if (c.op == kDone && tid == 0) found_none();
        send(s, c, ctas);
    };
    // the token that was found, by one thread
    auto write_token = [&]() {
        if (s.got_index == 0xFFFFFFFFu) {
            found_none();
            return;
        }
        p.tokens[r] = static_cast<int32_t>(s.got_index);
        const uint64_t mass = s.got_mass;
        // a likely token's log from what is left of the sum, which is accurate near 0; another's
        // from its z, which a weight of few units of 2^-40 has lost the last bits of
        if (p.logprobs)
            p.logprobs[r] = 2 * mass > sum ? log1pf(-(static_cast<float>(sum - mass) / static_cast<float>(sum)))
                                           : s.got_z - logf(static_cast<float>(sum) * 0x1p-40f);
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
        if (by_m) {
            m_sum = 0;
            for (uint32_t q = 0; q < ctas; ++q) m_sum += s.above[q];
            m_sum = max(m_sum, uint64_t{1} << 40);
        }
        if (warp == 0) {
            // After a cut in bin b, S lies between the running sums before and
            // after b; the targets grow with S.  Where its ends (even and odd
            // lanes) lead to bins b0 and b1, S itself leads to one of b0 .. b1.
            const bool end = lane & 1;
            uint64_t at = sum;
            SBinsOf o;
            auto found = [&](int j, uint64_t t) {
                if (j == kCutK) {
                    o.lo[j] = o.hi[j] = reach(s.sum_c, kSBins, t);
                } else {
                    o.lo[j] = reach(s.sum_w, kSBins, __shfl_sync(0xffffffffu, t, 0));
                    o.hi[j] = reach(s.sum_w, kSBins, __shfl_sync(0xffffffffu, t, 1));
                }
                float unused;
                row.bin_range(o.hi[j], o.x_lo[j], unused);
                row.bin_range(o.lo[j], unused, o.x_hi[j]);
                const uint64_t before = o.lo[j] ? s.sum_w[o.lo[j] - 1] : 0;
                at = min(at, max(end ? s.sum_w[o.hi[j]] : before, uint64_t{1} << 40));
            };
#pragma unroll
            for (int j = 0; j < kStages; ++j) {
                o.lo[j] = 1;
                o.hi[j] = 0;
                o.x_lo[j] = INFINITY;
                o.x_hi[j] = -INFINITY;
            }
            if (by_k && static_cast<uint32_t>(top_k) < s.sum_c[kSBins - 1])
                found(kCutK, static_cast<uint64_t>(top_k));
            if (top_p < 1.f) found(kCutP, cut_target(top_p, at));
            at = min(at, m_sum);
            found(kDraw, draw_target(uniform, at));
            if (lane < ctas) {
                const uint32_t to = dsmem_addr(smem_u32(&s.bins), lane);
#pragma unroll
                for (int j = 0; j < kStages; ++j) {
                    dsmem_st_s32(to + offsetof(SBinsOf, lo) + 4 * j, o.lo[j]);
                    dsmem_st_s32(to + offsetof(SBinsOf, hi) + 4 * j, o.hi[j]);
                    dsmem_st_f32(to + offsetof(SBinsOf, x_lo) + 4 * j, o.x_lo[j]);
                    dsmem_st_f32(to + offsetof(SBinsOf, x_hi) + 4 * j, o.x_hi[j]);
                }
            }
        }
    }
    if (tid < kStages) s.ns[tid] = 0;
    cluster_sync_all();
    // ---- one pass gathers the tokens of all three, in the first CTA
    const SBinsOf bins = s.bins;
    auto gather = [&](float x, int index) {
        const float y = logit(x) + 0.f, z = row.z(y);
        if (!SRow::counts(z)) return;
        const int b = row.bin(z);
#pragma unroll
        for (int j = 0; j < kStages; ++j)
            if (bins.lo[j] <= b && b <= bins.hi[j]) {
                const uint32_t at = atomicAdd(&s.ns[j], 1u);
                if (at < kSList)
                    s.lists[j][at] = (static_cast<uint64_t>(order_key(y)) << kSIndexBits) | static_cast<uint32_t>(index);
            }
    };
    // without the batches of which no logit is that large (64 x 152000: 42.1 -> 36.5 us,
    // 256 x 152000: 117.4 -> 109.1); where the part is resident a read costs too little for that
    auto gather_pass = [&](auto &&f) {
        if constexpr (kResident) {
            pass(Loads<4>{}, f);
        } else {
            const float least = fminf(fminf(bins.x_lo[kCutK], bins.x_lo[kCutP]), bins.x_lo[kDraw]);
            stream(Loads<4>{}, f, [&](int place) { return xs[place] >= least; }, nothing);
        }
    };
    if (bins.lo[kCutK] > bins.hi[kCutK] && bins.lo[kCutP] > bins.hi[kCutP]) {
        // (one range to compare with)
        gather_pass([&](const float(&x)[4], int first) {
#pragma unroll
            for (int k = 0; k < 4; ++k)
                if ((x[k] >= bins.x_lo[kDraw]) & (x[k] <= bins.x_hi[kDraw])) gather(x[k], first + k);
        });
    } else {
        gather_pass([&](const float(&x)[4], int first) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                bool maybe = false;  // (no short circuits: six comparisons take less than their branches)
#pragma unroll
                for (int j = 0; j < kStages; ++j) maybe |= (x[k] >= bins.x_lo[j]) & (x[k] <= bins.x_hi[j]);
                if (maybe) gather(x[k], first + k);
            }
        });
    }
    if (rank != 0) {
        __syncthreads();
        if (tid < kStages) s.at[tid] = s.ns[tid] ? atom_cluster_add(dsmem_addr(smem_u32(&s.ns[tid]), 0), s.ns[tid]) : 0;
        __syncthreads();
#pragma unroll
        for (int j = 0; j < kStages; ++j)
            for (uint32_t i = tid; i < min(s.ns[j], static_cast<uint32_t>(kSList)); i += kSThreads)
                if (s.at[j] + i < kSList)
                    st_cluster_u64(dsmem_addr(smem_u32(&s.lists[j][s.at[j] + i]), 0), s.lists[j][i]);
    }
    cluster_sync_all();
    uint32_t most = 0;
#pragma unroll
    for (int j = 0; j < kStages; ++j) most = max(most, ld_cluster_u32(dsmem_addr(smem_u32(&s.ns[j]), 0)));
    if (most <= kSList) {
        cluster_arrive_relaxed();  // this CTA has read the first one's counts
        if (rank != 0) return;
        if (most <= kSRank) {
            rank_lists(s, row);
            if (warp == 0) {
                s.got_index = 0;
#pragma unroll
                for (int j = 0; j < kStages; ++j) {
                    const int first = s.bins.lo[j], found = static_cast<int>(s.ns[j]);
                    if (first > s.bins.hi[j]) continue;
                    if (j == kDraw) sum = min(sum, m_sum);
                    const uint64_t t = j == kCutK   ? static_cast<uint64_t>(top_k)
                                       : j == kCutP ? cut_target(top_p, sum)
                                                    : draw_target(uniform, sum);
                    const uint64_t before = first > 0 ? s.sum_w[first - 1] : 0;
                    const int at = j == kCutK ? top_k - 1 - static_cast<int>(first > 0 ? s.sum_c[first - 1] : 0)
                                              : reach(s.run_w[j], max(found, 1), t - before);
                    if (at < 0 || at >= found || (j != kCutK && s.run_w[j][at] < t - before)) {
                        s.got_index = 0xFFFFFFFFu;
                        break;
                    }
                    const uint64_t to = s.run_w[j][at];
                    if (j < kDraw) {
                        sum = before + to;
                        continue;
                    }
                    const uint64_t v = s.lists[j][at];
                    s.got_index = static_cast<uint32_t>(v) & (kSMaxVocab - 1);
                    s.got_mass = at ? to - s.run_w[j][at - 1] : to;
                    s.got_z = row.z(key_value(static_cast<uint32_t>(v >> kSIndexBits)));
                }
                __syncwarp();
                if (lane == 0) write_token();
            }
        } else {
#pragma unroll 1
            for (int j = 0; j < kStages; ++j) {
                const int first = s.bins.lo[j];
                if (first > s.bins.hi[j]) continue;
                stage = j;
                if (tid == 0) {
                    s.base_w = first > 0 ? s.sum_w[first - 1] : 0;
                    s.base_c = first > 0 ? s.sum_c[first - 1] : 0;
                }
                next_target();
                uint64_t lo, hi;
                place_range<T>(s.bins.x_lo[j], fminf(s.bins.x_hi[j], row.top), lo, hi);
                const uint64_t v[kOfThread] = {s.lists[j][tid], s.lists[j][tid + kSThreads]};
                search_list(s, row, want, v, s.ns[j], lo, hi);
                if (s.got_index == 0xFFFFFFFFu) break;
                if (j < kDraw) sum = s.got_w;
            }
            if (tid == 0) write_token();
        }
        cluster_wait();
        return;
    }
    // ---- one search after the other, each bin divided while it holds too many tokens
    stage = kCutK;
    if (rank == 0) next_search();
    for (int step = 0; step < kSMaxCommands; ++step) {
        // (the first CTA has read every list and count when it gets here)
        cluster_sync_all();
        const SCommand cmd = s.cmd;
        if (cmd.op == kDone) return;
        if (cmd.op == kDivide)
            for (int b = tid; b < kSFine; b += kSThreads) s.cnt[b] = s.wl[b] = s.wh[b] = 0;
        if (tid == 0) s.n = 0;
        __syncthreads();
        pass(Loads<2>{}, [&](const float(&x)[4], int first) {
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if (!((x[k] >= cmd.x_lo) & (x[k] <= cmd.x_hi))) continue;
                const float y = logit(x[k]) + 0.f, z = row.z(y);
                if (!SRow::counts(z)) continue;
                const uint64_t place =
                    (static_cast<uint64_t>(order_key(y)) << kSIndexBits) | static_cast<uint32_t>(first + k);
                if (row.bin(z) != static_cast<int>(cmd.bin) || place < cmd.lo || place > cmd.hi) continue;
                if (cmd.op == kDivide) {
                    const uint32_t b = static_cast<uint32_t>((place - cmd.lo) >> cmd.shift);
                    if (by_k) atomicAdd(&s.cnt[b], 1u);
                    add_weight(&s.wl[b], &s.wh[b], SRow::weight2(expf(z)));
                    continue;
                }
                const uint32_t at = atomicAdd(&s.n, 1u);
                if (at < kSList) s.list[at] = place;
            }
        });
        if (cmd.op != kDivide) {
            __syncthreads();
            if (tid == 0) st_cluster_u32(dsmem_addr(smem_u32(&s.all_n[rank]), 0), s.n);
        }
        cluster_sync_all();
        if (cmd.op == kDivide) {
            push_sums<true>(s, rank, ctas, by_k);
            cluster_sync_all();
        }
        if (rank != 0) continue;
        SCommand c = cmd;
        c.op = kDone;
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
            c.op = s.got_bin == 0xFFFFFFFFu ? kDone : kGather;
            c.lo = cmd.lo + (static_cast<uint64_t>(s.got_bin) << cmd.shift);
            c.hi = min(cmd.hi, c.lo + (uint64_t{1} << cmd.shift) - 1);
            c.x_lo = key_value(static_cast<uint32_t>(c.hi >> kSIndexBits));
            c.x_hi = key_value(static_cast<uint32_t>(c.lo >> kSIndexBits));
            if (c.x_hi >= kLargest<T>) c.x_hi = INFINITY;  // (the passes compare the logits as they are)
            if (c.op == kDone && tid == 0) found_none();
            send(s, c, ctas);
            continue;
        }
        uint32_t total = 0;
        for (uint32_t q = 0; q < ctas; ++q) total += s.all_n[q];
        if (total > kSList) {
            c = cmd;
            c.op = kDivide;
            // at most kSFine parts of 2^shift places
            const int bits = 64 - __clzll(static_cast<long long>(c.hi - c.lo));
            c.shift = bits > 9 ? bits - 9 : 0;
            send(s, c, ctas);
            continue;
        }
        auto n_of = [&](uint32_t q) { return s.all_n[q]; };
        const uint64_t v[kOfThread] = {list_entry(s.list, tid, total, ctas, n_of),
                                       list_entry(s.list, tid + kSThreads, total, ctas, n_of)};
        search_list(s, row, want, v, total, cmd.lo, cmd.hi);
        if (s.got_index == 0xFFFFFFFFu || stage == kDraw) {
            if (tid == 0) write_token();
            send(s, c, ctas);  // kDone
            continue;
        }
        sum = s.got_w;
        stage = stage == kCutK ? kCutP : kDraw;
        next_search();
    }
    if (rank == 0 && tid == 0) found_none();  // out of commands
}
static_assert(kSFine == 1 << 9, "shift of a divided range");

size_t sample_smem_bytes(int32_t chunk) {
    // up to 7 values of padding in front of the row's part and 3 behind it
    return (sizeof(SShared) + 15) / 16 * 16 + (static_cast<size_t>(chunk) + 12) * sizeof(float);
}

// the maximum of each batch of the first pass (4 x 16 bytes a thread)
size_t sample_stream_smem_bytes(int32_t chunk, bool bf16) {
    const int32_t round = 4 * kSThreads * (bf16 ? 8 : 4);
    return (sizeof(SShared) + 15) / 16 * 16 + static_cast<size_t>((chunk + round - 1) / round) * kSThreads * sizeof(float);
}

// two CTAs share an SM
constexpr int kHalfSm = 115712;
constexpr int kPortableCluster = 8;

using SampleKernel = void (*)(SampleParams);
SampleKernel sample_kernel_of(bool bf16, bool resident) {
    return bf16 ? (resident ? sample_kernel<__nv_bfloat16, true> : sample_kernel<__nv_bfloat16, false>)
                : (resident ? sample_kernel<float, true> : sample_kernel<float, false>);
}

// Sets the kernel's limits, once per device, and says whether the current device
// runs it in clusters of kSMaxCluster (more than every device has to).
cudaError_t prepare_sample(SampleKernel kernel, int which, bool *wide) {
    static std::atomic<uint64_t> limit_set[4] = {}, yes[4] = {}, no[4] = {};
    *wide = false;
    cudaError_t e = ensure_smem_limit(kernel, kHalfSm, limit_set[which]);
    int dev = 0;
    if (e == cudaSuccess) e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    const uint64_t bit = dev >= 0 && dev < 64 ? uint64_t{1} << dev : 0;
    if (!bit || (no[which].load(std::memory_order_acquire) & bit)) return cudaSuccess;
    if (!(yes[which].load(std::memory_order_acquire) & bit)) {
        cudaLaunchConfig_t cfg = {};
        cfg.gridDim = dim3(kSMaxCluster);
        cfg.blockDim = dim3(kSThreads);
        cfg.dynamicSmemBytes = kHalfSm;
        cudaLaunchAttribute a = {};
        a.id = cudaLaunchAttributeClusterDimension;
        a.val.clusterDim.x = kSMaxCluster;
        a.val.clusterDim.y = a.val.clusterDim.z = 1;
        cfg.attrs = &a;
        cfg.numAttrs = 1;
        int n = 0;
        if (cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess ||
            cudaOccupancyMaxActiveClusters(&n, kernel, &cfg) != cudaSuccess || n < 1) {
            cudaGetLastError();
            no[which].fetch_or(bit, std::memory_order_release);
            return cudaSuccess;
        }
        yes[which].fetch_or(bit, std::memory_order_release);
    }
    *wide = true;
    return cudaSuccess;
}

cudaError_t launch_sample(SampleParams p, int32_t n_rows, bool bf16, cudaStream_t st) {
    const int64_t slots = 2 * static_cast<int64_t>(device_sm_count());
    auto chunk_of = [&](int32_t c) { return ((p.vocab + c - 1) / c + 7) / 8 * 8; };
    auto fits = [&](int32_t c) { return sample_smem_bytes(chunk_of(c)) <= static_cast<size_t>(kHalfSm); };
    // As many CTAs a row as one round holds, 2048 logits each at least (1 row x
    // 152000: 16 CTAs 14.4 us, 8 17.4, 4 22.6; 8 rows 16.8, 20.8, 26.2; 64 x 32003: 4
    // CTAs 15.3, 8 23.0, 2 20.0; 20 x 5000: 4 CTAs 10.1, 2 11.0, 8 10.7), and parts
    // of at most 80 K logits: large batches in several rounds, whose passes then
    // overlap (256 x 152000: 115 us with 1 CTA a row, 105 with 2, 106 with 4, 141 with
    // 8).  Parts that fit into half an SM's shared memory stay there (1 x 152000: 14.4
    // us against 15.5 read again from L2; 32 x 128000 bf16 20.5 and 22.1).
    int32_t c = 1;
    while (c < kSMaxCluster &&
           ((2 * c * static_cast<int64_t>(n_rows) <= slots && chunk_of(c) > 2048) || chunk_of(c) > 80 * 1024))
        c *= 2;
    bool resident = fits(c), wide = false;
    cudaError_t e = prepare_sample(sample_kernel_of(bf16, resident), 2 * bf16 + resident, &wide);
    if (e == cudaSuccess && c > kPortableCluster && !wide) {
        c = kPortableCluster;
        resident = fits(c);
        e = prepare_sample(sample_kernel_of(bf16, resident), 2 * bf16 + resident, &wide);
    }
    if (e != cudaSuccess) return e;
    const SampleKernel kernel = sample_kernel_of(bf16, resident);
    p.chunk = chunk_of(c);
    const size_t smem = resident ? sample_smem_bytes(p.chunk) : sample_stream_smem_bytes(p.chunk, bf16);
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
