// Log probabilities of given tokens, the entropy of the next token, and its most
// likely alternatives, from a row of logits x with maximum M:
//   z_i = x_i - M,  S = sum exp(z_i),  T = sum z_i exp(z_i),
//   log p_i = z_i - ln S,  entropy = ln S - T / S,
// alternatives in the order of (x descending, index ascending).
//
// One pass over the row.  A thread sums 2^(x L - c), L = log2 e, against a whole
// number c of its own, raised when its logits outgrow it: a new c scales the
// sums by a power of two, exactly, and x L - c is rounded once.  (M need not be known,
// and a row is read from HBM once, by asynchronous copies into each thread's own
// places: no thread waits for another's.)  The n-th largest of the maxima of 64
// groups of threads is at most the n-th largest logit; what reaches it, a few times
// n of all logits, goes to a list, whose first n are found by comparing all pairs.
// That bound is raised as rounds of the pass double.  A cluster of CTAs shares a
// row where rows are few, and its first CTA joins what they found.
//
// Many rows are bound by HBM: 4096 x 128000 bf16 in 152.0 us, 6.9 TB/s, the copy's rate,
// with the issue slots 70 % busy (about 9 instructions a logit); 256 x 152000 with 20
// alternatives 27.8 us (5.6 TB/s, 26.5 without alternatives: one wave of CTAs that
// start and end together).  Few rows are a chain of copy, bound, list, ranks and two cluster
// barriers: 1 x 152000 7.4 us, 4.3 without alternatives.
//
// A CTA's part of a row that this does not suit is read again, a logit at a time, once for the
// sums and twice or more for the alternatives:
//  - where c has to follow a maximum (of a thread's 32 logits of a round) of 2^22 / L (2.9e6) and more in
//    size, or all logits of a warp are so: +inf, a finite mask between -6.9e29 and -2.9e6 that has all 32
//    of a thread's first ones (of half of a row's logits, at random, none has, of 99 % many), the
//    types' lowest values where they have all of a warp's (-inf never);
//  - where more logits reach the bound than a warp's list holds: all equal, or fewer
//    alternatives in front of the mask than are asked for.
// 256 x 152000 with 20 alternatives 426 us (99 % masked by -1e9, or +inf in every row; 27.8 by
// -inf), one row 20 to 33; 1024 x 128000 bf16 with 5 680.
#include <float.h>
#include <math.h>
#include <stddef.h>

#include <atomic>

#include "ppas_device.cuh"
#include "ppas_internal.h"

namespace ppas {
namespace {

constexpr int kLThreads = 256;  // of a CTA; where rows are many and short, 128 or 64
// 16-byte loads of a round, a thread (32 logits), rounds under way, and the CTAs that an SM
// then holds: of fp32 3 (bf16 4), and where there are fewer, kFew, 2 (3) with a round
// more under way.  (256 x 152000: 27.7 us, 29.0 with the shorter ring; 128: 19.0 and 20.7; 400
// 48.8 and 39.6; 32 x 128000 bf16 7.7 and 9.0, 1024 x 128000 48.2 and 43.7.  Rounds of 16
// logits of fp32: 1 x 152000 13 % longer; of 64 of bf16: 1024 x 128000 9 %.)
template <class T>
constexpr int kLLoads = sizeof(T) == 4 ? 8 : 4;
template <class T, bool kFew>
constexpr int kLStages = (sizeof(T) == 4 ? 2 : 3) + (kFew ? 1 : 0);
template <class T, bool kFew>
constexpr int kLAnSm = (sizeof(T) == 4 ? 3 : 4) - (kFew ? 1 : 0);
constexpr int kLGroups = 64;
// places of the lists, and of each of the N / 32 warps
template <int N>
constexpr int kLList = N == kLThreads ? 640 : 512;
template <int N>
constexpr int kLOfWarp = kLList<N> / (N / 32);
constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLLimit = 0x1p22f;  // |x L| from here on: the whole numbers c have no room left
constexpr float kLFloor = -1e30f;   // logits below count as this: 2^(x L - c) is 0, and 0 times x L - c too
constexpr float kLRaise = 8.f;      // c follows logits that are 2^8 past it
static_assert(kLMaxTop <= kLGroups, "each alternative has a group");

// The largest finite logit of type T, as which +inf counts.
template <class T>
constexpr float kLLargest = sizeof(T) == 4 ? FLT_MAX : 0x1.FEp127f;

template <class T>
__device__ __forceinline__ float value_of(T x) {
    if constexpr (sizeof(T) == 4) return x;
    else return __bfloat162float(x);
}
// a logit as it counts: a NaN as -inf, +inf as the largest finite one, -0 as 0
template <class T>
__device__ __forceinline__ float logit_of(T x) {
    return fminf(fmaxf(value_of(x), -INFINITY), kLLargest<T>) + 0.f;
}

// a logit as a whole number that ascends with it
__device__ __forceinline__ uint32_t ascending(float x) {
    const uint32_t b = __float_as_uint(x);
    return (b >> 31) ? ~b : b | 0x80000000u;
}
__device__ __forceinline__ float of_ascending(uint32_t key) {
    return __uint_as_float((key >> 31) ? key & 0x7FFFFFFFu : ~key);
}
// (x, index) as a whole number: larger logits first, of equal ones the lower index; never 0
__device__ __forceinline__ uint64_t place_of(float x, uint32_t index) {
    return (static_cast<uint64_t>(ascending(x)) << 32) | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ float place_logit(uint64_t place) {
    return of_ascending(static_cast<uint32_t>(place >> 32));
}
__device__ __forceinline__ int32_t place_index(uint64_t place) {
    return static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(place));
}

// the rounds that raise the bound: 0, 1, 3, 7, ... where as many are to come
__device__ __forceinline__ bool raises(int round, int rounds) {
    return ((round + 1) & round) == 0 && (round == 0 || rounds >= 2 * (round + 1));
}

// what a CTA found in its part of a row: the maximum, and the sums relative to it
struct LPart {
    float top, s, t;
};
template <int N>
struct LShared {
    static constexpr int kLWarps = N / 32;
    uint64_t list[kLList<N>];    // each warp's places at or above the bound
    uint32_t n_list[kLWarps];
    uint64_t best[kLMaxTop];  // this CTA's alternatives, in order; 0: none
    LPart parts[kLMaxCluster];
    union {
        alignas(16) uint32_t group[kLGroups];  // (read four at a time)
        uint64_t group_place[kLGroups];
    };
    uint64_t place[kLWarps];
    float s[kLWarps], t[kLWarps], top[kLWarps];
    uint32_t bad[kLWarps];
    float bound;
    uint64_t bound_place;
    uint32_t n_kept;
};

// Each thread's own logits under way; the memory has other uses once they are through.
template <class T, bool kFew, int N>
struct LRing {
    union {
        uint4 ring[kLStages<T, kFew>][kLLoads<T>][N];
        struct {
            uint64_t kept[kLList<N>];
            uint64_t all[kLMaxCluster * kLMaxTop];
        };
    };
};

template <int N>
__device__ __forceinline__ uint64_t block_max(LShared<N> &sh, uint64_t v) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int o = 16; o; o >>= 1) {
        const uint64_t u = __shfl_xor_sync(0xffffffffu, v, o);
        v = u > v ? u : v;
    }
    __syncthreads();
    if (lane == 0) sh.place[warp] = v;
    __syncthreads();
    for (int w = 0; w < N / 32; ++w) v = sh.place[w] > v ? sh.place[w] : v;
    return v;
}

__device__ __forceinline__ void cluster_arrive() {
    asm volatile("barrier.cluster.arrive.release.aligned;" ::: "memory");
}
__device__ __forceinline__ void st_cluster_u64(uint32_t a, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}

// The n-th largest of the groups' maxima (or a little less), given every thread's: a group's
// threads count how many are above it.
template <int N>
__device__ __forceinline__ float bound_of(LShared<N> &sh, float top, int n) {
    constexpr uint32_t kIndex = kLGroups - 1;  // a key's low bits tell equal maxima apart
    constexpr int kOf = N / kLGroups, kVecs = kLGroups / 4 / kOf;
    const int tid = threadIdx.x;
#pragma unroll
    for (int o = 1; o < kOf; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const uint32_t mine = (ascending(top) & ~kIndex) | static_cast<uint32_t>(tid / kOf);
    if (tid % kOf == 0) sh.group[tid / kOf] = mine;
    __syncthreads();
    const uint4 *g4 = reinterpret_cast<const uint4 *>(sh.group) + tid % kOf * kVecs;
    int above = 0;
#pragma unroll
    for (int j = 0; j < kVecs; ++j) {
        const uint4 g = g4[j];
        above += (g.x > mine) + (g.y > mine) + (g.z > mine) + (g.w > mine);
    }
#pragma unroll
    for (int o = 1; o < kOf; o <<= 1) above += __shfl_xor_sync(0xffffffffu, above, o);
    if (above == n - 1 && tid % kOf == 0)
        sh.bound = (mine & ~kIndex) <= ascending(-INFINITY) ? -INFINITY : of_ascending(mine & ~kIndex);
    __syncthreads();
    return sh.bound;
}

// emit(i, place) for the first n of the m places in `from` in their order, and emit(i, 0)
// for what they do not have: a place's rank is the number of larger ones, counted by several
// lanes.  By whichever thread: no barrier.
template <int N, class Emit>
__device__ __forceinline__ void rank_places(const uint64_t *from, int m, int n, Emit &&emit) {
    const int tid = threadIdx.x;
    if (tid >= m && tid < n) emit(tid, 0);
    int lanes = 32;
    while (lanes > 1 && m * lanes > N) lanes >>= 1;
    const int l = tid & (lanes - 1);
    for (int base = 0; base < m; base += N / lanes) {
        const int i = base + tid / lanes;
        const uint64_t mine = i < m ? from[i] : 0;
        int before = 0;
#pragma unroll 4
        for (int j = l; j < m; j += lanes) before += from[j] > mine;
        for (int o = lanes >> 1; o; o >>= 1) before += __shfl_xor_sync(0xffffffffu, before, o);
        if (l == 0 && i < m && before < n) emit(before, mine);
    }
}

// A part's alternatives where the list overflowed: by places instead of logits,
// which tells equal logits apart; and where even those are too many, one by one.
template <class T, int N>
__device__ __noinline__ void slow_top(LShared<N> &sh, const T *src, int n, int i0, int n_top) {
    const int tid = threadIdx.x;
    uint64_t best = 0;
    for (int i = tid; i < n; i += N) {
        const uint64_t v = place_of(logit_of(src[i]), static_cast<uint32_t>(i0 + i));
        best = v > best ? v : best;
    }
    for (int o = 1; o < N / kLGroups; o <<= 1) {
        const uint64_t other = __shfl_xor_sync(0xffffffffu, best, o);
        best = other > best ? other : best;
    }
    __syncthreads();
    if (tid % (N / kLGroups) == 0) sh.group_place[tid / (N / kLGroups)] = best;
    if (tid == 0) sh.n_kept = 0;
    __syncthreads();
    if (tid < kLGroups) {
        const uint64_t mine = sh.group_place[tid];
        int before = 0;
        for (int j = 0; j < kLGroups; ++j)
            before += sh.group_place[j] > mine || (sh.group_place[j] == mine && j < tid);  // (equal: 0, no logits)
        if (before == n_top - 1) sh.bound_place = mine;
    }
    __syncthreads();
    const uint64_t bound = sh.bound_place;
    for (int i = tid; i < n; i += N) {
        const uint64_t v = place_of(logit_of(src[i]), static_cast<uint32_t>(i0 + i));
        if (v >= bound && place_logit(v) > -INFINITY) {
            const uint32_t at = atomicAdd(&sh.n_kept, 1u);
            if (at < kLList<N>) sh.list[at] = v;
        }
    }
    __syncthreads();
    const uint32_t m = sh.n_kept;
    if (m <= kLList<N>) {
        rank_places<N>(sh.list, static_cast<int>(m), n_top, [&](int i, uint64_t v) { sh.best[i] = v; });
        __syncthreads();
        return;
    }
    uint64_t before = ~uint64_t{0};
    for (int j = 0; j < n_top; ++j) {
        best = 0;
        for (int i = tid; i < n; i += N) {
            const uint64_t v = place_of(logit_of(src[i]), static_cast<uint32_t>(i0 + i));
            if (v < before && v > best) best = v;
        }
        best = block_max(sh, best);
        before = best;
        if (tid == 0) sh.best[j] = best != 0 && place_logit(best) > -INFINITY ? best : 0;
    }
    __syncthreads();
}

// a part's sums, the maximum known
template <class T, int N>
__device__ __noinline__ float2 slow_sums(const T *src, int n, float top) {
    float s = 0.f, t = 0.f;
    // (32 at a time: fewer roundings lie behind one another)
    for (int a = threadIdx.x; a < n; a += 32 * N) {
        float s1 = 0.f, t1 = 0.f;
        for (int i = a; i < n && i < a + 32 * N; i += N) {
            const float z = logit_of(src[i]) - top, e = expf(z);
            s1 += e;
            t1 += e > 0.f ? z * e : 0.f;
        }
        s += s1;
        t += t1;
    }
    return make_float2(s, t);
}

// the values of 16 bytes, as they are and for the sums (none below kLFloor, no NaN), and their maximum with `top`
template <class T>
__device__ __forceinline__ void widen(uint4 q, float (&x)[16 / sizeof(T)]) {
    const uint32_t w[4] = {q.x, q.y, q.z, q.w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        if constexpr (sizeof(T) == 4) {
            x[k] = __uint_as_float(w[k]);
        } else {
            x[2 * k] = __uint_as_float(w[k] << 16);
            x[2 * k + 1] = __uint_as_float(w[k] & 0xFFFF0000u);
        }
    }
}
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
    uint32_t r;
    asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
    return r;
}
template <class T>
__device__ __forceinline__ uint4 floored(uint4 q) {
    if constexpr (sizeof(T) == 4) {
        auto f = [](uint32_t w) { return __float_as_uint(fmaxf(__uint_as_float(w), kLFloor)); };
        return make_uint4(f(q.x), f(q.y), f(q.z), f(q.w));
    } else {
        constexpr uint32_t kFloors = 0xF149F149u;  // twice -1e30 in bf16
        return make_uint4(max_bf16x2(q.x, kFloors), max_bf16x2(q.y, kFloors), max_bf16x2(q.z, kFloors),
                          max_bf16x2(q.w, kFloors));
    }
}
// the maximum of 16 bytes' values, NaNs passed over: of bf16 the two halves' each
template <class T>
__device__ __forceinline__ uint32_t max_bits(uint4 q) {
    if constexpr (sizeof(T) == 4)
        return __float_as_uint(fmaxf(max3(__uint_as_float(q.x), __uint_as_float(q.y), __uint_as_float(q.z)),
                                     __uint_as_float(q.w)));
    else return max_bf16x2(max_bf16x2(q.x, q.y), max_bf16x2(q.z, q.w));
}
template <class T>
__device__ __forceinline__ uint32_t max_bits(uint32_t a, uint32_t b) {
    if constexpr (sizeof(T) == 4) return __float_as_uint(fmaxf(__uint_as_float(a), __uint_as_float(b)));
    else return max_bf16x2(a, b);
}
template <class T>
__device__ __forceinline__ float max_value(uint32_t bits) {
    if constexpr (sizeof(T) == 4) return fmaxf(__uint_as_float(bits), -INFINITY);
    else return fmaxf(fmaxf(__uint_as_float(bits << 16), __uint_as_float(bits & 0xFFFF0000u)), -INFINITY);
}
// 16 bytes that are not all of the part, from its value `first` on: value by value, -inf where there is none
template <class T>
__device__ __noinline__ uint4 edge_vector(const T *src, int first, int n) {
    uint32_t w[4];
#pragma unroll
    for (int k = 0; k < 4; ++k) {
        auto bits = [&](int i) -> uint32_t {
            const bool in = i >= 0 && i < n;
            if constexpr (sizeof(T) == 4) return in ? __float_as_uint(src[i]) : 0xFF800000u;
            else return in ? __bfloat16_as_ushort(src[i]) : 0xFF80u;
        };
        if constexpr (sizeof(T) == 4) w[k] = bits(first + k);
        else w[k] = bits(first + 2 * k) | (bits(first + 2 * k + 1) << 16);
    }
    return make_uint4(w[0], w[1], w[2], w[3]);
}
__device__ __forceinline__ void copy16_async(uint32_t to, const void *from) {
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(to), "l"(from) : "memory");
}
__device__ __forceinline__ void copies_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int n>
__device__ __forceinline__ void copies_wait() {
    asm volatile("cp.async.wait_group %0;" ::"n"(n) : "memory");
}

}  // namespace

template <class T, bool kTop, bool kFew, int N>
__global__ void __launch_bounds__(N) token_logprobs_kernel(const __grid_constant__ LogprobParams p) {
    extern __shared__ __align__(16) uint8_t logprob_smem[];
    using Ring = LRing<T, kFew, N>;
    using Shared = LShared<N>;
    Ring &ring = *reinterpret_cast<Ring *>(logprob_smem);
    Shared &sh = *reinterpret_cast<Shared *>(logprob_smem + sizeof(Ring));
    constexpr int kLoads = kLLoads<T>, kStages = kLStages<T, kFew>;
    constexpr int kPer = 16 / sizeof(T);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t ctas = cluster_nctarank(), rank = ctas > 1 ? cluster_ctarank() : 0;
    const int64_t r = blockIdx.x / ctas;
    if (tid == 0) sh.n_kept = 0;
    grid_dep_launch();
    grid_dep_wait();
    const T *const row = static_cast<const T *>(p.logits) + r * p.row_stride;
    const bool joins = rank == 0 && tid == 0;

    // ---- this CTA's part of the row, from the 16-byte boundary at or before its first logit
    const int i0 = min(static_cast<int>(rank) * p.chunk, p.vocab), n = min(p.chunk, p.vocab - i0);
    const T *const src = row + i0;
    const int pad = static_cast<int>((reinterpret_cast<uintptr_t>(src) / sizeof(T)) % kPer);
    const int vecs = (pad + n + kPer - 1) / kPer;
    const int whole0 = pad ? 1 : 0, whole1 = (pad + n) / kPer;  // [whole0, whole1) have all their values
    const uint4 *const src4 = reinterpret_cast<const uint4 *>(src - pad);
    // A thread's copies go to its own places of the ring, from which it alone reads:
    // its own waits are all that it takes.
    constexpr int kRound = N * kLoads;
    const int rounds = (vecs + kRound - 1) / kRound;
    constexpr uint32_t kNone = sizeof(T) == 4 ? 0xFF800000u : 0xFF80FF80u;  // -inf, bf16 twice
    auto fetch = [&](int round, int stage) {
        const int v0 = round * kRound;
        if (v0 >= whole0 && v0 + kRound <= whole1) {
            const uint4 *from = src4 + v0 + tid;
            const uint32_t to = smem_u32(&ring.ring[stage][0][tid]);
#pragma unroll
            for (int k = 0; k < kLoads; ++k) copy16_async(to + k * N * 16, from + k * N);
        } else if (sizeof(T) == 4 && round < rounds) {
            // (a part's last round, all at once; of bf16 one 16 bytes after another, which the
            // kernel's other rounds lose least to: 3292 x 5323 fp32 takes 12 % longer so; 4096 x
            // 128000 bf16 11 % longer all at once)
#pragma unroll
            for (int k = 0; k < kLoads; ++k) {
                const int v = v0 + k * N + tid;
                if (v >= whole0 && v < whole1) copy16_async(smem_u32(&ring.ring[stage][k][tid]), src4 + v);
                else if (v >= vecs) ring.ring[stage][k][tid] = make_uint4(kNone, kNone, kNone, kNone);
            }
            // the part's first 16 bytes and its last, where they are not whole
            if (whole0 && v0 + tid == 0) ring.ring[stage][0][tid] = edge_vector(src, -pad, n);
            if (const int k = (whole1 - v0 - tid) / N;
                whole1 < vecs && whole1 >= max(v0, whole0) && k < kLoads && (whole1 - tid) % N == 0)
                ring.ring[stage][k][tid] = edge_vector(src, whole1 * kPer - pad, n);
        } else if (round < rounds) {
#pragma unroll 1
            for (int k = 0; k < kLoads; ++k) {
                const int v = v0 + k * N + tid;
                if (v >= whole0 && v < whole1) copy16_async(smem_u32(&ring.ring[stage][k][tid]), src4 + v);
                else if (v >= vecs) ring.ring[stage][k][tid] = make_uint4(kNone, kNone, kNone, kNone);
                else ring.ring[stage][k][tid] = edge_vector(src, v * kPer - pad, n);
            }
        }
        copies_commit();
    };
#pragma unroll
    for (int i = 0; i < kStages - 1; ++i) fetch(i, i);
    const int32_t given = joins && p.tokens ? __ldg(p.tokens + r) : -1;
    float top = -INFINITY, c = -1e30f, s = 0.f, t = 0.f, bound = INFINITY;
    bool bad = false;
    uint32_t n_list = 0;  // of this warp
    T x_given = {};
    for (int round = 0, stage = 0; round < rounds; ++round, stage = stage + 1 == kStages ? 0 : stage + 1) {
        fetch(round + kStages - 1, stage == 0 ? kStages - 1 : stage - 1);
        copies_wait<kStages - 1>();
        uint4 q[kLoads];
#pragma unroll
        for (int k = 0; k < kLoads; ++k) q[k] = ring.ring[stage][k][tid];
        // (by now the given token is known, and its logit has until the end to come)
        if (round == 0 && given >= 0 && given < p.vocab) x_given = row[given];
        uint32_t most[kLoads], all = 0;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            most[k] = max_bits<T>(q[k]);
            all = k ? max_bits<T>(all, most[k]) : most[k];
        }
        const float here = max_value<T>(all);
        top = fmaxf(top, here);
        if (kTop && raises(round, rounds)) bound = bound_of(sh, top, p.n_top);
        if (here * kLog2E - c > kLRaise) {  // (not where all are -inf)
            bad = bad || !(fabsf(here) * kLog2E < kLLimit);
            const float now = ceilf(here * kLog2E), d = now - c, f = ex2(-d);
            t = (t - d * s) * f;
            s *= f;
            c = now;
        }
        float2 s2 = make_float2(0.f, 0.f), t2 = s2;
#pragma unroll
        for (int k = 0; k < kLoads; ++k) {
            float x[kPer];
            widen<T>(floored<T>(q[k]), x);
#pragma unroll
            for (int e = 0; e < kPer; e += 2) {
                const float2 z = fma2(make_float2(x[e], x[e + 1]), make_float2(kLog2E, kLog2E), make_float2(-c, -c));
                const float2 w = make_float2(ex2(z.x), ex2(z.y));
                s2 = add2(s2, w);
                t2 = fma2(z, w, t2);
            }
        }
        s += s2.x + s2.y;
        t += t2.x + t2.y;
        if (kTop) {
            // the logits at or above the bound go to the list: the warp looks through the
            // values of one of its lanes after another (a lane by itself through its own, a
            // few of them at a time keeping the whole warp: 256 x 152000 12 % longer)
            uint32_t hits = __ballot_sync(0xffffffffu, here >= bound && here > -INFINITY);
            if (hits) {
                constexpr int kValues = kLoads * kPer;
                static_assert(kValues == 32, "a lane looks at one of them");
                const int k = lane / kPer, e = lane % kPer;
                __syncwarp();
                do {
                    const int from = (tid & ~31) + __ffs(hits) - 1;
                    hits &= hits - 1;
                    const float x = value_of(reinterpret_cast<const T *>(&ring.ring[stage][k][from])[e]);
                    const bool in = x >= bound && x > -INFINITY;
                    const uint32_t those = __ballot_sync(0xffffffffu, in);
                    const uint32_t at = n_list + __popc(those & ((1u << lane) - 1));
                    const int index = i0 + ((round * kLoads + k) * N + from) * kPer + e - pad;
                    if (in && at < kLOfWarp<N>) sh.list[warp * kLOfWarp<N> + at] = place_of(x + 0.f, static_cast<uint32_t>(index));
                    n_list += __popc(those);
                } while (hits);
                __syncwarp();
            }
        }
    }
    // ---- each warp's maximum and sums relative to it, behind one barrier (from which on
    // the ring's memory has other uses)
    {
        float most = top;
        for (int o = 16; o; o >>= 1) most = fmaxf(most, __shfl_xor_sync(0xffffffffu, most, o));
        const bool some = most > -INFINITY;
        if (some) {
            const float z = fmaf(most, kLog2E, -c), f = ex2(-z);  // (a thread without logits: z = 1e30, f = 0)
            t = kLn2 * (t - z * s) * f;
            s *= f;
        }
        for (int o = 16; o; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            t += __shfl_xor_sync(0xffffffffu, t, o);
        }
        bad = __any_sync(0xffffffffu, bad) || (some && !(fabsf(most) * kLog2E < kLLimit));
        if (lane == 0) {
            sh.top[warp] = most;
            sh.s[warp] = s;
            sh.t[warp] = t;
            sh.bad[warp] = bad;
            sh.n_list[warp] = n_list;
        }
    }
    __syncthreads();
    // the first CTA's ring may take the others' finds once every CTA is here (the other
    // half of this barrier is before the first store to it)
    if (ctas > 1) cluster_arrive();

    // ---- the part's, by every warp for itself
    const int w8 = lane % Shared::kLWarps;
    float part_top = sh.top[w8];
    for (int o = 1; o < Shared::kLWarps; o <<= 1) part_top = fmaxf(part_top, __shfl_xor_sync(0xffffffffu, part_top, o));
    part_top = fminf(part_top, kLLargest<T>);
    const bool any = part_top > -INFINITY;
    const bool part_bad = __any_sync(0xffffffffu, sh.bad[w8] != 0);
    const bool full = __any_sync(0xffffffffu, sh.n_list[w8] > kLOfWarp<N>);
    if (any && part_bad) {
        const float2 v = slow_sums<T, N>(src, n, part_top);
        s = v.x;
        t = v.y;
        for (int o = 16; o; o >>= 1) {
            s += __shfl_xor_sync(0xffffffffu, s, o);
            t += __shfl_xor_sync(0xffffffffu, t, o);
        }
        __syncthreads();
        if (lane == 0) {
            sh.s[warp] = s;
            sh.t[warp] = t;
        }
        __syncthreads();
        s = sh.s[w8];
        t = sh.t[w8];
    } else {
        const float d = sh.top[w8] - part_top, f = any ? expf(d) : 0.f;
        s = f > 0.f ? sh.s[w8] * f : 0.f;
        t = f > 0.f ? fmaf(d, sh.s[w8], sh.t[w8]) * f : 0.f;
    }
    for (int o = 1; o < Shared::kLWarps; o <<= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        t += __shfl_xor_sync(0xffffffffu, t, o);
    }
    // ---- its alternatives: in `kept`, or in their order in `best`
    const bool in_best = kTop && any && (part_bad || full);
    if (in_best) {
        slow_top(sh, src, n, i0, p.n_top);
    } else if (kTop) {
        // without those that only an earlier bound let in
        for (uint32_t j = 0; j < n_list; j += 32) {
            const uint32_t i = j + static_cast<uint32_t>(lane);
            const uint64_t v = i < n_list ? sh.list[warp * kLOfWarp<N> + i] : 0;
            const bool in = i < n_list && place_logit(v) >= bound;
            const uint32_t those = __ballot_sync(0xffffffffu, in);
            uint32_t at = 0;
            if (lane == 0) at = atomicAdd(&sh.n_kept, static_cast<uint32_t>(__popc(those)));
            at = __shfl_sync(0xffffffffu, at, 0) + __popc(those & ((1u << lane) - 1));
            if (in) ring.kept[at] = v;
        }
        __syncthreads();
    }
    float m = part_top;
    if (ctas > 1) {
        // ---- the first CTA joins the parts
        if (kTop && !in_best) {
            rank_places<N>(ring.kept, static_cast<int>(sh.n_kept), p.n_top, [&](int i, uint64_t v) { sh.best[i] = v; });
            __syncthreads();
        }
        cluster_wait();
        if (tid == 0) {
            const uint32_t to = dsmem_addr(smem_u32(&sh.parts[rank]), 0);
            dsmem_st_f32(to, part_top);
            dsmem_st_f32(to + 4, any ? s : 0.f);
            dsmem_st_f32(to + 8, any ? t : 0.f);
        }
        if (kTop && tid < p.n_top)
            st_cluster_u64(dsmem_addr(smem_u32(&ring.all[rank * p.n_top + tid]), 0), sh.best[tid]);
        cluster_sync_all();
        if (rank != 0) return;
        for (uint32_t i = 0; i < ctas; ++i) m = fmaxf(m, sh.parts[i].top);
        s = t = 0.f;
        if (m > -INFINITY)
            for (uint32_t i = 0; i < ctas; ++i) {
                const LPart part = sh.parts[i];
                const float d = part.top - m, f = expf(d);
                s = fmaf(part.s, f, s);
                t += f > 0.f ? f * fmaf(d, part.s, part.t) : 0.f;
            }
        if (kTop) {
            // the n-th largest of all is at least the least of every CTA's (n / CTAs)-th
            const int at = (p.n_top + static_cast<int>(ctas) - 1) / static_cast<int>(ctas) - 1;
            const uint32_t least = __reduce_min_sync(
                0xffffffffu, static_cast<uint32_t>(ring.all[min(lane, static_cast<int>(ctas) - 1) * p.n_top + at] >> 32));
            if (tid == 0) sh.n_kept = 0;
            __syncthreads();
            for (int i = tid; i < static_cast<int>(ctas) * p.n_top; i += N) {
                const uint64_t v = ring.all[i];
                if (v != 0 && static_cast<uint32_t>(v >> 32) >= least) ring.kept[atomicAdd(&sh.n_kept, 1u)] = v;
            }
            __syncthreads();
        }
    }
    const bool row_any = m > -INFINITY;
    s = fmaxf(s, 1.f);  // (the maximum's own, but for roundings)
    const float ln_s = logf(s);
    if (kTop) {
        auto put = [&](int i, uint64_t v) {
            p.top_tokens[r * p.n_top + i] = v ? place_index(v) : -1;
            p.top_logprobs[r * p.n_top + i] = v ? place_logit(v) - m - ln_s : -INFINITY;
        };
        if (in_best && ctas == 1) {
            if (tid < p.n_top) put(tid, sh.best[tid]);
        } else {
            rank_places<N>(ring.kept, static_cast<int>(sh.n_kept), p.n_top, put);
        }
    }
    if (tid == 0) {
        if (p.entropy) p.entropy[r] = row_any ? fmaxf(ln_s - t / s, 0.f) : 0.f;
        if (p.logprobs) {
            float lp = 0.f;
            if (given >= p.vocab) report_error(p.err, PPAS_DEVERR_BAD_INDEX);
            if (given >= 0) lp = row_any && given < p.vocab ? logit_of(x_given) - m - ln_s : -INFINITY;
            p.logprobs[r] = lp;
        }
    }
}

static_assert(kLMaxCluster * kLMaxTop <= kLList<kLThreads>, "the first CTA ranks them in `kept`");
template <class T, bool kFew, int N>
constexpr int kLSmem = static_cast<int>(sizeof(LRing<T, kFew, N>) + sizeof(LShared<N>));
template <class T, bool kFew>
constexpr bool kLFits = kLAnSm<T, kFew> * (kLSmem<T, kFew, kLThreads> + 1024) <= 233472;
static_assert(kLFits<float, false> && kLFits<float, true> && kLFits<__nv_bfloat16, false> && kLFits<__nv_bfloat16, true>,
              "shared memory of an SM");
static_assert(kLMaxTop <= 64, "an alternative a thread");
template <int N>
constexpr bool kLAligned = offsetof(LShared<N>, group) % 16 == 0 && sizeof(LRing<float, false, N>) % 16 == 0 &&
                           sizeof(LRing<__nv_bfloat16, false, N>) % 16 == 0;
static_assert(kLAligned<64> && kLAligned<128> && kLAligned<kLThreads>, "groups are read 16 bytes at a time");

// How many clusters of 2, 4, 8 and 16 CTAs (16 are more than the portable 8) of a kernel
// this device holds at a time; once per device.
template <class T, bool kTop, bool kFew>
cudaError_t prepare_logprobs(int32_t (&clusters)[5]) {
    static std::atomic<uint64_t> limit_set{0};
    static std::atomic<int32_t> known[64][5] = {};  // + 1; 0: not asked
    const auto kernel = token_logprobs_kernel<T, kTop, kFew, kLThreads>;
    cudaError_t e = ensure_smem_limit(kernel, kLSmem<T, kFew, kLThreads>, limit_set);
    int dev = 0;
    if (e == cudaSuccess) e = cudaGetDevice(&dev);
    if (e != cudaSuccess) return e;
    for (int i = 1; i < 5; ++i) {
        int32_t n = dev >= 0 && dev < 64 ? known[dev][i].load(std::memory_order_acquire) : 0;
        if (n == 0) {
            cudaLaunchConfig_t cfg = {};
            cfg.gridDim = dim3(1u << i);
            cfg.blockDim = dim3(kLThreads);
            cfg.dynamicSmemBytes = kLSmem<T, kFew, kLThreads>;
            cudaLaunchAttribute a = {};
            a.id = cudaLaunchAttributeClusterDimension;
            a.val.clusterDim.x = 1u << i;
            a.val.clusterDim.y = a.val.clusterDim.z = 1;
            cfg.attrs = &a;
            cfg.numAttrs = 1;
            int most = 0;
            if ((i == 4 && cudaFuncSetAttribute(kernel, cudaFuncAttributeNonPortableClusterSizeAllowed, 1) != cudaSuccess) ||
                cudaOccupancyMaxActiveClusters(&most, kernel, &cfg) != cudaSuccess) {
                cudaGetLastError();
                most = 0;  // (none: a row has fewer CTAs)
            }
            n = most + 1;
            if (dev >= 0 && dev < 64) known[dev][i].store(n, std::memory_order_release);
        }
        clusters[i] = n - 1;
    }
    return cudaSuccess;
}

template <class T, bool kTop, bool kFew>
cudaError_t launch_logprobs(LogprobParams p, int32_t n_rows, cudaStream_t st) {
    // As many CTAs a row as run at a time, 4096 logits each at least, 16 only where each
    // has an SM (1 x 152000: 16 CTAs 7.4 us, 8 8.0, 4 9.7; 12 x 128000 bf16: 8 CTAs 6.8, 16 7.5, 4 7.4;
    // 64 x 32003 bf16: 4 CTAs 6.7, 8, of fewer logits and in two rounds, 11.3, 2 8.0, 1 6.3; 64 x 152000:
    // 4 CTAs 14.4, 8, in two rounds, 20.2, 2 17.2).
    int32_t clusters[5] = {};
    const cudaError_t e = prepare_logprobs<T, kTop, kFew>(clusters);
    if (e != cudaSuccess) return e;
    int i = 16 * static_cast<int64_t>(n_rows) <= device_sm_count() ? 4 : 3;
    while (i > 0 && (n_rows > clusters[i] || p.vocab < 4096 << i)) --i;
    const int32_t c = 1 << i;
    p.chunk = ((p.vocab + c - 1) / c + 15) / 16 * 16;
    PdlLaunch l(dim3(static_cast<unsigned>(n_rows) * c), dim3(kLThreads), kLSmem<T, kFew, kLThreads>, st);
    cudaLaunchAttribute attrs[2] = {l.attr[0], {}};
    if (c > 1) {
        attrs[1].id = cudaLaunchAttributeClusterDimension;
        attrs[1].val.clusterDim.x = static_cast<unsigned>(c);
        attrs[1].val.clusterDim.y = 1;
        attrs[1].val.clusterDim.z = 1;
        l.cfg.attrs = attrs;
        l.cfg.numAttrs = 2;
    }
    return cudaLaunchKernelEx(&l.cfg, token_logprobs_kernel<T, kTop, kFew, kLThreads>, p);
}

template <class T, bool kTop, int N>
cudaError_t launch_narrow(LogprobParams p, int32_t n_rows, cudaStream_t st) {
    static std::atomic<uint64_t> limit_set{0};
    const auto kernel = token_logprobs_kernel<T, kTop, false, N>;
    constexpr int kSmem = kLSmem<T, false, N>;
    const cudaError_t e = ensure_smem_limit(kernel, kSmem, limit_set);
    if (e != cudaSuccess) return e;
    p.chunk = (p.vocab + 15) / 16 * 16;
    PdlLaunch l(dim3(static_cast<unsigned>(n_rows)), dim3(N), kSmem, st);
    return cudaLaunchKernelEx(&l.cfg, kernel, p);
}

template <class T, bool kTop>
cudaError_t launch_logprobs(const LogprobParams &p, int32_t n_rows, cudaStream_t st) {
    const int64_t sms = device_sm_count(), wide = kLAnSm<T, false> * sms;
    // A row's barriers, list and ranks hide behind other rows' loads, so where there are more
    // than CTAs of 256 threads hold at a time, and short ones, smaller CTAs take them (fp32, 3292 x
    // 5323, 1 alternative: 64 threads 20.3 us, 256 35.0; 4096 x 8000, 5: 27.6, 128 33.5, 256 42.8;
    // bf16 1024 x 16000, 20: 24.1, 128 15.4, 256 15.7; 2503 x 42728, 5: 128 44.3, 256 48.6; 300 x
    // 1000, 5: 64 4.1, 256 5.0; 700 x 64000, 20: 128 32.3, 256 26.7).
    if (n_rows > sms && (p.vocab <= 2048 || (n_rows > 2 * wide && p.vocab <= 8192)))
        return launch_narrow<T, kTop, 64>(p, n_rows, st);
    if (n_rows > wide && (p.vocab <= 16384 || (n_rows > 2 * wide && p.vocab <= 65536)))
        return launch_narrow<T, kTop, 128>(p, n_rows, st);
    return n_rows <= kLAnSm<T, true> * sms ? launch_logprobs<T, kTop, true>(p, n_rows, st)
                                           : launch_logprobs<T, kTop, false>(p, n_rows, st);
}

cudaError_t launch_token_logprobs(const LogprobParams &p, int32_t n_rows, bool bf16, cudaStream_t st) {
    if (p.n_top > 0)
        return bf16 ? launch_logprobs<__nv_bfloat16, true>(p, n_rows, st) : launch_logprobs<float, true>(p, n_rows, st);
    return bf16 ? launch_logprobs<__nv_bfloat16, false>(p, n_rows, st) : launch_logprobs<float, false>(p, n_rows, st);
}

}  // namespace ppas

using namespace ppas;

extern "C" ppas_status ppas_token_logprobs(const void *logits, int32_t logits_are_bf16, int64_t row_stride,
                                           int32_t n_rows, int32_t vocab, const int32_t *d_tokens, float *d_logprobs,
                                           float *d_entropy, int32_t n_top, int32_t *d_top_tokens,
                                           float *d_top_logprobs, int32_t *d_err_flag, void *stream) {
    if (n_rows < 0 || vocab < 1 || n_top < 0) return PPAS_ERR_INVALID_ARG;
    if (vocab > kSMaxVocab || n_top > kLMaxTop || n_rows > INT32_MAX / kLMaxCluster) return PPAS_ERR_UNSUPPORTED;
    if (n_rows == 0) return PPAS_OK;
    if (row_stride < vocab || !logits || !d_tokens != !d_logprobs ||
        (n_top > 0 && (!d_top_tokens || !d_top_logprobs)) || (n_top == 0 && !d_logprobs && !d_entropy))
        return PPAS_ERR_INVALID_ARG;
    auto on = [](const void *x, uintptr_t n) { return (reinterpret_cast<uintptr_t>(x) & (n - 1)) == 0; };
    if (!on(logits, logits_are_bf16 ? 2 : 4) || !on(d_tokens, 4) || !on(d_logprobs, 4) || !on(d_entropy, 4) ||
        !on(d_top_tokens, 4) || !on(d_top_logprobs, 4) || !on(d_err_flag, 4))
        return PPAS_ERR_INVALID_ARG;
    LogprobParams p = {};
    p.logits = logits;
    p.row_stride = row_stride;
    p.tokens = d_tokens;
    p.logprobs = d_logprobs;
    p.entropy = d_entropy;
    p.top_tokens = d_top_tokens;
    p.top_logprobs = d_top_logprobs;
    p.err = d_err_flag;
    p.vocab = vocab;
    p.n_top = n_top;
    return launch_token_logprobs(p, n_rows, logits_are_bf16 != 0, static_cast<cudaStream_t>(stream)) == cudaSuccess
               ? PPAS_OK
               : PPAS_ERR_CUDA;
}
