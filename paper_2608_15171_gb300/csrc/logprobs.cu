// Log probabilities of given tokens, the entropy of the next token, and its most
// likely alternatives, from a row of logits x with maximum M:
//   z_i = x_i - M,  S = sum exp(z_i),  T = sum z_i exp(z_i),
//   log p_i = z_i - ln S,  entropy = ln S - T / S,
// alternatives in the order of (x descending, index ascending).
//
// One pass over the row.  A thread sums 2^(x L - c), L = log2 e, against a whole
// number c of its own, raised when its logits outgrow it: a new c scales the
// sums by a power of two, exactly, and x L - c is rounded once.  (M need not be known,
// and a row is read from HBM once.)  The n-th largest of the maxima of 128
// groups of threads is at most the n-th largest logit; what reaches it, a few times
// n of all logits, goes to a list, whose first n are found by comparing all pairs.
// That bound is raised as rounds of the pass double.  A cluster of CTAs shares a
// row where rows are few, and its first CTA joins what they found.
//
// Rows that this does not suit (a maximum of 2^22 / L and more, infinite ones
// among them, or more logits at the bound than the list holds, as where all are equal)
// are read again, slowly and for sure.
#include <float.h>
#include <math.h>

#include "ppas_device.cuh"
#include "ppas_internal.h"

namespace ppas {
namespace {

constexpr int kLThreads = 256;
constexpr int kLWarps = kLThreads / 32;
constexpr int kLLoads = 4;       // 16-byte loads that a thread has under way
constexpr int kLGroups = kLThreads / 2;
constexpr int kLList = 1024;     // places of a list
constexpr float kLog2E = 1.4426950408889634f, kLn2 = 0.6931471805599453f;
constexpr float kLLimit = 0x1p22f;  // |x L| from here on: the whole numbers c have no room left
constexpr float kLFloor = -200.f;   // 2^-200 is 0, and so is its product with -200
constexpr float kLRaise = 8.f;      // c follows logits that are 2^8 past it
static_assert(kLMaxTop <= kLGroups, "each alternative has a group");

// The largest finite logit of type T, as which +inf counts.
template <class T>
constexpr float kLLargest = sizeof(T) == 4 ? FLT_MAX : 0x1.FEp127f;

// a logit as it counts: a NaN as -inf, +inf as the largest finite one, -0 as 0
template <class T>
__device__ __forceinline__ float logit_of(T x) {
    float v;
    if constexpr (sizeof(T) == 4) v = x;
    else v = __bfloat162float(x);
    return fminf(fmaxf(v, -INFINITY), kLLargest<T>) + 0.f;
}

// (x, index) as a whole number: larger logits first, of equal ones the lower index; never 0
__device__ __forceinline__ uint64_t place_of(float x, uint32_t index) {
    const uint32_t b = __float_as_uint(x);
    const uint32_t key = (b >> 31) ? ~b : b | 0x80000000u;  // ascending with x
    return (static_cast<uint64_t>(key) << 32) | (0xFFFFFFFFu - index);
}
__device__ __forceinline__ float place_logit(uint64_t place) {
    const uint32_t key = static_cast<uint32_t>(place >> 32);
    return __uint_as_float((key >> 31) ? key & 0x7FFFFFFFu : ~key);
}
__device__ __forceinline__ int32_t place_index(uint64_t place) {
    return static_cast<int32_t>(0xFFFFFFFFu - static_cast<uint32_t>(place));
}

// what a CTA found in its part of a row: the maximum, and the sums relative to it
struct LPart {
    float top, s, t;
};
struct LShared {
    uint64_t list[kLList];    // places at or above the bound
    uint64_t kept[kLList];    // of these the ones at or above the last bound
    uint64_t best[kLMaxTop];  // this CTA's alternatives, in order; 0: none
    uint64_t all[kLMaxCluster * kLMaxTop];  // first CTA: every CTA's
    LPart parts[kLMaxCluster];
    union {
        float group[kLGroups];
        uint64_t group_place[kLGroups];
    };
    uint64_t place[kLWarps];
    float s[kLWarps], t[kLWarps], top[kLWarps];
    float bound;
    uint64_t bound_place;
    uint32_t n_list, n_kept;
};

__device__ __forceinline__ uint64_t block_max(LShared &sh, uint64_t v) {
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    for (int o = 16; o; o >>= 1) {
        const uint64_t u = __shfl_xor_sync(0xffffffffu, v, o);
        v = u > v ? u : v;
    }
    __syncthreads();
    if (lane == 0) sh.place[warp] = v;
    __syncthreads();
    for (int w = 0; w < kLWarps; ++w) v = sh.place[w] > v ? sh.place[w] : v;
    return v;
}

__device__ __forceinline__ void st_cluster_u64(uint32_t a, uint64_t v) {
    asm volatile("st.shared::cluster.u64 [%0], %1;" ::"r"(a), "l"(v) : "memory");
}

// The n-th largest of the groups' maxima, given every thread's.
__device__ __forceinline__ float bound_of(LShared &sh, float top, int n) {
    const int tid = threadIdx.x;
    top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, 1));
    if ((tid & 1) == 0) sh.group[tid >> 1] = top;
    __syncthreads();
    if (tid < kLGroups) {
        const float mine = sh.group[tid];
        const float4 *g4 = reinterpret_cast<const float4 *>(sh.group);
        int before = 0;
#pragma unroll 8
        for (int j = 0; j < kLGroups / 4; ++j) {
            const float4 g = g4[j];
            before += g.x > mine || (g.x == mine && 4 * j < tid);
            before += g.y > mine || (g.y == mine && 4 * j + 1 < tid);
            before += g.z > mine || (g.z == mine && 4 * j + 2 < tid);
            before += g.w > mine || (g.w == mine && 4 * j + 3 < tid);
        }
        if (before == n - 1) sh.bound = mine;
    }
    __syncthreads();
    return sh.bound;
}

// best[0 .. n) of the m places in `from` (a 0 is none), in order (0 where there are fewer)
__device__ __forceinline__ void rank_places(const uint64_t *from, int m, uint64_t *best, int n) {
    for (int i = threadIdx.x; i < n; i += kLThreads) best[i] = 0;
    __syncthreads();
    for (int i = threadIdx.x; i < m; i += kLThreads) {
        const uint64_t mine = from[i];
        int before = 0;
#pragma unroll 4
        for (int j = 0; j < m; ++j) before += from[j] > mine;
        if (before < n && mine != 0) best[before] = mine;
    }
    __syncthreads();
}

// A part's alternatives where the list overflowed: by places instead of logits,
// which tells equal logits apart; and where even those are too many, one by one.
template <class T>
__device__ __noinline__ void slow_top(LShared &sh, const T *src, int n, int i0, int n_top) {
    const int tid = threadIdx.x;
    uint64_t best = 0;
    for (int i = tid; i < n; i += kLThreads) {
        const uint64_t v = place_of(logit_of(src[i]), static_cast<uint32_t>(i0 + i));
        best = v > best ? v : best;
    }
    const uint64_t other = __shfl_xor_sync(0xffffffffu, best, 1);
    best = other > best ? other : best;
    __syncthreads();
    if ((tid & 1) == 0) sh.group_place[tid >> 1] = best;
    if (tid == 0) sh.n_list = 0;
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
    for (int i = tid; i < n; i += kLThreads) {
        const uint64_t v = place_of(logit_of(src[i]), static_cast<uint32_t>(i0 + i));
        if (v >= bound && place_logit(v) > -INFINITY) {
            const uint32_t at = atomicAdd(&sh.n_list, 1u);
            if (at < kLList) sh.list[at] = v;
        }
    }
    __syncthreads();
    const uint32_t m = sh.n_list;
    if (m <= kLList) {
        rank_places(sh.list, static_cast<int>(m), sh.best, n_top);
        return;
    }
    uint64_t before = ~uint64_t{0};
    for (int j = 0; j < n_top; ++j) {
        best = 0;
        for (int i = tid; i < n; i += kLThreads) {
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
template <class T>
__device__ __noinline__ float2 slow_sums(const T *src, int n, float top) {
    float s = 0.f, t = 0.f;
    // (32 at a time: fewer roundings lie behind one another)
    for (int a = threadIdx.x; a < n; a += 32 * kLThreads) {
        float s1 = 0.f, t1 = 0.f;
        for (int i = a; i < n && i < a + 32 * kLThreads; i += kLThreads) {
            const float z = logit_of(src[i]) - top, e = expf(z);
            s1 += e;
            t1 += e > 0.f ? z * e : 0.f;
        }
        s += s1;
        t += t1;
    }
    return make_float2(s, t);
}

// the values of 16 bytes
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

}  // namespace

template <class T, bool kTop>
__global__ void __launch_bounds__(kLThreads) token_logprobs_kernel(const __grid_constant__ LogprobParams p) {
    __shared__ __align__(16) LShared sh;
    constexpr int kPer = 16 / sizeof(T);
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const uint32_t ctas = cluster_nctarank(), rank = ctas > 1 ? cluster_ctarank() : 0;
    const int64_t r = blockIdx.x / ctas;
    // (the other half of this barrier is before the first store to another CTA)
    cluster_arrive_relaxed();
    if (tid == 0) sh.n_list = sh.n_kept = 0;
    grid_dep_launch();
    grid_dep_wait();
    const T *const row = static_cast<const T *>(p.logits) + r * p.row_stride;
    const bool joins = rank == 0 && tid == 0;
    const int32_t given = joins && p.tokens ? __ldg(p.tokens + r) : -1;
    const float x_given = given >= 0 && given < p.vocab ? logit_of(row[given]) : 0.f;

    // ---- this CTA's part of the row, from the 16-byte boundary at or before its first logit
    const int i0 = min(static_cast<int>(rank) * p.chunk, p.vocab), n = min(p.chunk, p.vocab - i0);
    const T *const src = row + i0;
    const int pad = static_cast<int>((reinterpret_cast<uintptr_t>(src) / sizeof(T)) % kPer);
    const int vecs = (pad + n + kPer - 1) / kPer;
    const int whole0 = pad ? 1 : 0, whole1 = (pad + n) / kPer;  // [whole0, whole1) have all their values
    const uint4 *const src4 = reinterpret_cast<const uint4 *>(src - pad);
    auto load = [&](int v) {
        if (v >= whole0 && v < whole1) return __ldg(src4 + v);
        uint32_t w[4];  // the first and the last ones: value by value (and past them -inf)
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            auto bits = [&](int e) -> uint32_t {
                const int i = v * kPer + e - pad;
                const bool in = i >= 0 && i < n;
                if constexpr (sizeof(T) == 4) return in ? __float_as_uint(src[i]) : 0xFF800000u;
                else return in ? __bfloat16_as_ushort(src[i]) : 0xFF80u;
            };
            if constexpr (sizeof(T) == 4) w[k] = bits(k);
            else w[k] = bits(2 * k) | (bits(2 * k + 1) << 16);
        }
        return make_uint4(w[0], w[1], w[2], w[3]);
    };
    float top = -INFINITY, c = -1e30f, s = 0.f, t = 0.f, bound = INFINITY;
    bool bad = false;
    int rounds = 0;
    for (int base = 0; base < vecs; base += kLThreads * kLLoads, ++rounds) {
        uint4 q[kLLoads];
#pragma unroll
        for (int k = 0; k < kLLoads; ++k) q[k] = load(base + k * kLThreads + tid);
        float here = -INFINITY;  // (a maximum passes over NaNs)
#pragma unroll
        for (int k = 0; k < kLLoads; ++k) {
            float x[kPer];
            widen<T>(q[k], x);
#pragma unroll
            for (int e = 0; e < kPer; e += 2) here = max3(here, x[e], x[e + 1]);
        }
        top = fmaxf(top, here);
        if (kTop && (rounds & (rounds + 1)) == 0) bound = bound_of(sh, top, p.n_top);
        if (here * kLog2E - c > kLRaise) {  // (not where all are -inf)
            bad = bad || !(fabsf(here) * kLog2E < kLLimit);
            const float now = ceilf(here * kLog2E), d = now - c, f = ex2(-d);
            t = (t - d * s) * f;
            s *= f;
            c = now;
        }
        float2 s2 = make_float2(0.f, 0.f), t2 = s2;
#pragma unroll
        for (int k = 0; k < kLLoads; ++k) {
            float x[kPer];
            widen<T>(q[k], x);
#pragma unroll
            for (int e = 0; e < kPer; e += 2) {
                float2 z = fma2(make_float2(x[e], x[e + 1]), make_float2(kLog2E, kLog2E), make_float2(-c, -c));
                z.x = fmaxf(z.x, kLFloor);
                z.y = fmaxf(z.y, kLFloor);
                const float2 w = make_float2(ex2(z.x), ex2(z.y));
                s2 = add2(s2, w);
                t2 = fma2(z, w, t2);
            }
        }
        s += s2.x + s2.y;
        t += t2.x + t2.y;
        if (kTop && here >= bound && here > -INFINITY) {
#pragma unroll
            for (int k = 0; k < kLLoads; ++k) {
                float x[kPer];
                widen<T>(q[k], x);
#pragma unroll
                for (int e = 0; e < kPer; ++e)
                    if (x[e] >= bound && x[e] > -INFINITY) {
                        const uint32_t at = atomicAdd(&sh.n_list, 1u);
                        if (at < kLList)
                            sh.list[at] = place_of(x[e] + 0.f, static_cast<uint32_t>(
                                                                  i0 + (base + k * kLThreads + tid) * kPer + e - pad));
                    }
            }
        }
    }

    // ---- the part's maximum and sums
    float part_top = top;
    for (int o = 16; o; o >>= 1) part_top = fmaxf(part_top, __shfl_xor_sync(0xffffffffu, part_top, o));
    if (lane == 0) sh.top[warp] = part_top;
    __syncthreads();
    for (int w = 0; w < kLWarps; ++w) part_top = fmaxf(part_top, sh.top[w]);
    part_top = fminf(part_top, kLLargest<T>);
    const bool any = part_top > -INFINITY;
    const bool part_bad = __syncthreads_or(bad || (any && !(fabsf(part_top) * kLog2E < kLLimit))) != 0;
    if (any && part_bad) {
        const float2 v = slow_sums(src, n, part_top);
        s = v.x;
        t = v.y;
    } else if (any) {
        const float z = fmaf(part_top, kLog2E, -c), f = ex2(-z);  // (a thread without logits: z = 1e30, f = 0)
        t = kLn2 * (t - z * s) * f;
        s *= f;
    }
    for (int o = 16; o; o >>= 1) {
        s += __shfl_xor_sync(0xffffffffu, s, o);
        t += __shfl_xor_sync(0xffffffffu, t, o);
    }
    if (lane == 0) {
        sh.s[warp] = s;
        sh.t[warp] = t;
    }
    // ---- its alternatives
    if (kTop) {
        const uint32_t m = sh.n_list;
        if (!any) {
            if (tid < p.n_top) sh.best[tid] = 0;
        } else if (m > kLList || part_bad) {
            slow_top(sh, src, n, i0, p.n_top);
        } else {
            const float last = (rounds & (rounds - 1)) == 0 ? bound : bound_of(sh, top, p.n_top);
            for (uint32_t i = tid; i < m; i += kLThreads) {
                const uint64_t v = sh.list[i];
                if (place_logit(v) >= last) sh.kept[atomicAdd(&sh.n_kept, 1u)] = v;
            }
            __syncthreads();
            rank_places(sh.kept, static_cast<int>(sh.n_kept), sh.best, p.n_top);
        }
    }
    __syncthreads();
    // ---- the first CTA joins the parts
    cluster_wait();  // every CTA of the cluster has started
    if (tid == 0) {
        s = t = 0.f;
        for (int w = 0; w < kLWarps; ++w) {
            s += sh.s[w];
            t += sh.t[w];
        }
        const uint32_t to = dsmem_addr(smem_u32(&sh.parts[rank]), 0);
        dsmem_st_f32(to, part_top);
        dsmem_st_f32(to + 4, any ? s : 0.f);
        dsmem_st_f32(to + 8, any ? t : 0.f);
    }
    if (kTop && ctas > 1 && tid < p.n_top)
        st_cluster_u64(dsmem_addr(smem_u32(&sh.all[rank * p.n_top + tid]), 0), sh.best[tid]);
    if (ctas > 1) cluster_sync_all();
    else __syncthreads();
    if (rank != 0) return;
    float m = -INFINITY;
    for (uint32_t i = 0; i < ctas; ++i) m = fmaxf(m, sh.parts[i].top);
    s = t = 0.f;
    const bool row_any = m > -INFINITY;
    if (row_any)
        for (uint32_t i = 0; i < ctas; ++i) {
            const LPart part = sh.parts[i];
            const float d = part.top - m, f = expf(d);
            s = fmaf(part.s, f, s);
            t += f > 0.f ? f * fmaf(d, part.s, part.t) : 0.f;
        }
    s = fmaxf(s, 1.f);  // (the maximum's own, but for roundings)
    const float ln_s = logf(s);
    if (kTop) {
        const uint64_t *found = sh.best;
        if (ctas > 1) {
            rank_places(sh.all, static_cast<int>(ctas) * p.n_top, sh.kept, p.n_top);
            found = sh.kept;
        }
        if (tid < p.n_top) {
            const uint64_t v = found[tid];
            p.top_tokens[r * p.n_top + tid] = v ? place_index(v) : -1;
            p.top_logprobs[r * p.n_top + tid] = v ? place_logit(v) - m - ln_s : -INFINITY;
        }
    }
    if (tid == 0) {
        if (p.entropy) p.entropy[r] = row_any ? fmaxf(ln_s - t / s, 0.f) : 0.f;
        if (p.logprobs) {
            float lp = 0.f;
            if (given >= p.vocab) report_error(p.err, PPAS_DEVERR_BAD_INDEX);
            if (given >= 0) lp = row_any && given < p.vocab ? x_given - m - ln_s : -INFINITY;
            p.logprobs[r] = lp;
        }
    }
}

template <class T>
cudaError_t launch_logprobs(LogprobParams p, int32_t n_rows, cudaStream_t st) {
    // as many CTAs a row as the SMs hold at a time, 4096 logits each at least
    const int64_t slots = 4 * static_cast<int64_t>(device_sm_count());
    int32_t c = 1;
    while (c < kPortableLCluster && 2 * c * static_cast<int64_t>(n_rows) <= slots && p.vocab >= 2 * c * 4096) c *= 2;
    p.chunk = ((p.vocab + c - 1) / c + 15) / 16 * 16;
    PdlLaunch l(dim3(static_cast<unsigned>(n_rows) * c), dim3(kLThreads), 0, st);
    cudaLaunchAttribute attrs[2] = {l.attr[0], {}};
    if (c > 1) {
        attrs[1].id = cudaLaunchAttributeClusterDimension;
        attrs[1].val.clusterDim.x = static_cast<unsigned>(c);
        attrs[1].val.clusterDim.y = 1;
        attrs[1].val.clusterDim.z = 1;
        l.cfg.attrs = attrs;
        l.cfg.numAttrs = 2;
    }
    return p.n_top > 0 ? cudaLaunchKernelEx(&l.cfg, token_logprobs_kernel<T, true>, p)
                       : cudaLaunchKernelEx(&l.cfg, token_logprobs_kernel<T, false>, p);
}

cudaError_t launch_token_logprobs(const LogprobParams &p, int32_t n_rows, bool bf16, cudaStream_t st) {
    return bf16 ? launch_logprobs<__nv_bfloat16>(p, n_rows, st) : launch_logprobs<float>(p, n_rows, st);
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
