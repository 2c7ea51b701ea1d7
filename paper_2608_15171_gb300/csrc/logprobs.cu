// Log probabilities of given tokens, the entropy of the next token, and its most
// likely alternatives, from a row of logits x with maximum M:
//   z_i = x_i - M,  S = sum exp(z_i),  T = sum z_i exp(z_i),
//   log p_i = z_i - ln S,  entropy = ln S - T / S,
// alternatives in the order of (x descending, index ascending).
//
// The simplest form: a CTA has a row and reads it once for M, once for the sums and
// once for each alternative.
#include <float.h>
#include <math.h>

#include "ppas_device.cuh"
#include "ppas_internal.h"

namespace ppas {
namespace {

constexpr int kLThreads = 256;
constexpr int kLWarps = kLThreads / 32;

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

// (x, index) as a whole number: larger logits first, of equal ones the lower index
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

struct LShared {
    uint64_t place[kLWarps];
    float s[kLWarps], t[kLWarps];
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

}  // namespace

template <class T>
__global__ void __launch_bounds__(kLThreads) token_logprobs_kernel(const __grid_constant__ LogprobParams p) {
    __shared__ LShared sh;
    const int tid = threadIdx.x, lane = tid & 31, warp = tid >> 5;
    const int64_t r = blockIdx.x;
    grid_dep_launch();
    grid_dep_wait();
    const T *const x = static_cast<const T *>(p.logits) + r * p.row_stride;
    const int32_t given = p.tokens ? __ldg(p.tokens + r) : -1;
    uint64_t best = 0, before = ~uint64_t{0};
    float top = 0.f, ln_s = 0.f, entropy = 0.f;
    bool any = false;
    // the largest place below the one before, again and again
    for (int j = 0; j < (p.n_top > 1 ? p.n_top : 1); ++j) {
        best = 0;
        for (int32_t i = tid; i < p.vocab; i += kLThreads) {
            const uint64_t v = place_of(logit_of(x[i]), static_cast<uint32_t>(i));
            if (v < before && v > best) best = v;
        }
        best = block_max(sh, best);
        before = best;
        const float z_at = place_logit(best);
        if (j == 0) {
            top = z_at;
            any = top > -INFINITY;
            float s = 0.f, t = 0.f;
            // (32 at a time: fewer roundings lie behind one another)
            for (int32_t i0 = tid; any && i0 < p.vocab; i0 += 32 * kLThreads) {
                float s1 = 0.f, t1 = 0.f;
                for (int32_t i = i0; i < p.vocab && i < i0 + 32 * kLThreads; i += kLThreads) {
                    const float z = logit_of(x[i]) - top, e = expf(z);
                    s1 += e;
                    t1 += e > 0.f ? z * e : 0.f;
                }
                s += s1;
                t += t1;
            }
            for (int o = 16; o; o >>= 1) {
                s += __shfl_xor_sync(0xffffffffu, s, o);
                t += __shfl_xor_sync(0xffffffffu, t, o);
            }
            if (lane == 0) {
                sh.s[warp] = s;
                sh.t[warp] = t;
            }
            __syncthreads();
            s = t = 0.f;
            for (int w = 0; w < kLWarps; ++w) {
                s += sh.s[w];
                t += sh.t[w];
            }
            s = fmaxf(s, 1.f);
            ln_s = logf(s);
            entropy = any ? fmaxf(ln_s - t / s, 0.f) : 0.f;
        }
        if (tid == 0 && p.n_top > 0) {
            const bool there = any && best != 0 && z_at > -INFINITY;
            p.top_tokens[r * p.n_top + j] = there ? place_index(best) : -1;
            p.top_logprobs[r * p.n_top + j] = there ? z_at - top - ln_s : -INFINITY;
        }
    }
    if (tid == 0) {
        if (p.entropy) p.entropy[r] = entropy;
        if (p.logprobs) {
            float lp = 0.f;
            if (given >= p.vocab) {
                report_error(p.err, PPAS_DEVERR_BAD_INDEX);
                lp = -INFINITY;
            } else if (given >= 0) {
                lp = any ? logit_of(x[given]) - top - ln_s : -INFINITY;
            }
            p.logprobs[r] = lp;
        }
    }
}

cudaError_t launch_token_logprobs(const LogprobParams &p, int32_t n_rows, bool bf16, cudaStream_t st) {
    PdlLaunch l(dim3(static_cast<unsigned>(n_rows)), dim3(kLThreads), 0, st);
    return bf16 ? cudaLaunchKernelEx(&l.cfg, token_logprobs_kernel<__nv_bfloat16>, p)
                : cudaLaunchKernelEx(&l.cfg, token_logprobs_kernel<float>, p);
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
