// Rotary positions and KV append in one pass: the new tokens' queries and keys
// are rotated by their positions, the keys and values go into their 16-token
// pages.  With pair (a, b) of a head, position t and inverse frequency f:
//   phi = t f,  a' = a c - b s,  b' = b c + a s,  c = factor cos phi, s = factor sin phi;
// a pair is (x[i], x[i + r/2]) in the half layout, (x[2i], x[2i + 1]) in the
// interleaved one, i < r/2; dims from r on pass through.
//
// The phase is kept as a fraction of a turn in 64-bit fixed point: f / 2 pi in
// units of 2^-64 turn comes from f's 24-bit significand and the digits of 1 / 2 pi,
// its product with the position wraps modulo one turn (2^-31 turn off at the
// most, for |t| <= 2^31), and the top 32 bits go to sincospif().
// So the angle of any 32-bit position and any finite f is good to 2^-25 turn,
// where t * f in fp32 is off by up to 0.004 rad at 131072.  (No 64-bit floating
// point: its rate is low here.)
//
// Pure data movement but for that: 4 bytes a value, bound by HBM in large
// calls and by launch and one memory round trip in small ones.  A warp takes
// one token's angles (computed once, 32 at a time, into shared memory) and some
// of its head rows; a lane has 2 x 16 bytes of a row, both members of its 8
// pairs, so rotation needs no exchange and may run in place.  16384 tokens of 32/8
// heads in 64.7 us (403 MB: 6.2 TB/s, 0.92 of a plain copy's rate); 2056 tokens of
// 16/2 heads take 5.6 us and one token 4.6, what a call costs the host.
#include <math.h>

#include "ppas_device.cuh"
#include "ppas_internal.h"

namespace ppas {
namespace {

constexpr int kRopeWarps = 8;
constexpr int kRopeMaxIter = 4;      // 32-lane passes over head rows a warp makes, loads of all in flight
constexpr int kRopeMaxDim = 512;     // head_dim: 16 values a lane
// a unit's 8 (cos, sin) pairs, two pairs of padding after them: the 16-byte
// reads of 8 neighbouring lanes then hit all banks once
constexpr int kUnitPitch = 10;

// 2^192 / (2 pi), rounded down
constexpr uint64_t kInv2 = 0x28BE60DB9391054Aull, kInv1 = 0x7F09D5F47D4D3770ull, kInv0 = 0x36D8A5664F10E410ull;

// f / (2 pi) modulo 1 as a 64-bit fraction of a turn, to 2^-63 turn, of f = m 2^-shift.
// The digits of 1 / (2 pi) that matter are those which f's exponent moves to the 64
// places behind the point (Payne and Hanek's reduction): 192 for the largest fp32
// numbers.  For f of 2 and more, which are rare: as a call it leaves the kernel's time
// as it is without it (2056 tokens 5.64 us, 5.93 inline).
__device__ __noinline__ uint64_t turns_of_large(uint64_t m, int shift) {
    // the product p3 p2 p1 p0 of m and the digits, the point in front of p2
    const uint64_t c0 = __umul64hi(m, kInv0), p1 = m * kInv1 + c0;
    const uint64_t c1 = __umul64hi(m, kInv1) + (p1 < c0 ? 1 : 0), p2 = m * kInv2 + c1;
    const uint64_t p3 = __umul64hi(m, kInv2) + (p2 < c1 ? 1 : 0);
    if (shift > 0) return (p2 >> shift) | (p3 << (64 - shift));
    if (shift == 0) return p2;
    if (shift > -64) return (p2 << -shift) | (p1 >> (64 + shift));
    if (shift == -64) return p1;
    return (p1 << (-shift - 64)) | (m * kInv0 >> (128 + shift));
}

// the same of any finite f; below 2 the first 64 digits do
__device__ __forceinline__ uint64_t turns_per_position(float f) {
    const uint32_t b = __float_as_uint(f);
    const int e = static_cast<int>((b >> 23) & 0xFF);
    const uint64_t m = e ? ((b & 0x7FFFFFu) | 0x800000u) : (b & 0x7FFFFFu);
    const int shift = 150 - (e ? e : 1);  // f = m 2^-shift
    const uint64_t lo = m * kInv2, hi = __umul64hi(m, kInv2);
    uint64_t t;
    if (shift < 23) t = turns_of_large(m, shift);
    else if (shift < 64) t = (lo >> shift) | (hi << (64 - shift));
    else t = shift < 128 ? hi >> (shift - 64) : 0;
    return (b >> 31) ? 0 - t : t;
}

// (factor cos, factor sin) of position times frequency
__device__ __forceinline__ float2 rope_angle(int32_t position, float inv_freq, float factor) {
    const uint64_t phase = turns_per_position(inv_freq) * static_cast<uint64_t>(static_cast<int64_t>(position));
    const float half_turns = static_cast<float>(static_cast<int32_t>(phase >> 32)) * 0x1p-31f;
    float s, c;
    sincospif(half_turns, &s, &c);
    return make_float2(c * factor, s * factor);
}

__device__ __forceinline__ float2 unpack_bf16x2(uint32_t v) {
    return make_float2(__uint_as_float(v << 16), __uint_as_float(v & 0xFFFF0000u));
}

// where a token's keys and values go; -1: nowhere
__device__ __forceinline__ int32_t checked_slot(const RopeParams &p, int32_t token, bool reports) {
    const int32_t slot = __ldg(p.slots + token);
    if (slot < 0) return -1;
    if (slot / kPage >= p.num_blocks) {
        if (reports) report_error(p.err, PPAS_DEVERR_BAD_INDEX);
        return -1;
    }
    return slot;
}

// head row `row` of a token: queries, then keys, then values
struct RopeRow {
    const __nv_bfloat16 *src;
    __nv_bfloat16 *dst;  // NULL: not written
    bool turns;
};
__device__ __forceinline__ RopeRow rope_row(const RopeParams &p, int32_t token, int32_t slot, int32_t row) {
    RopeRow r;
    const int64_t t = token;
    if (row < p.n_q_heads) {
        r.src = p.q + t * p.q_stride + row * p.head_dim;
        r.dst = p.q_out + (t * p.n_q_heads + row) * p.head_dim;
        r.turns = true;
        return r;
    }
    row -= p.n_q_heads;
    r.turns = row < p.n_kv_heads;
    const int32_t h = r.turns ? row : row - p.n_kv_heads;
    r.src = r.turns ? p.k + t * p.k_stride + h * p.head_dim : p.v + t * p.v_stride + h * p.head_dim;
    __nv_bfloat16 *const cache = r.turns ? p.k_cache : p.v_cache;
    // cache layout [block][kv_head][16][head_dim]
    r.dst = slot < 0 ? nullptr
                     : cache + ((static_cast<int64_t>(slot / kPage) * p.n_kv_heads + h) * kPage + slot % kPage) *
                                   p.head_dim;
    return r;
}

}  // namespace

// 16-byte accesses: rotary_dim a multiple of 16, every row 16-byte aligned.
template <bool kInterleaved>
__global__ void __launch_bounds__(kRopeWarps * 32) rope_append_kernel(const __grid_constant__ RopeParams p) {
    // the launch that follows may start its set-up now
    grid_dep_launch();
    extern __shared__ float4 rope_smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int32_t task = blockIdx.x * kRopeWarps + warp;
    if (task >= p.n_tasks) return;
    const int32_t token = task / p.tasks_per_token;
    const int32_t part = task - token * p.tasks_per_token;
    const int units = (p.head_dim + 15) / 16, half = p.rotary_dim / 2;
    const int rows_at_once = 32 / units;
    const int u = lane % units, sub = lane / units;
    const int rot_units = half / 8;
    float2 *const table = reinterpret_cast<float2 *>(rope_smem) + warp * rot_units * kUnitPitch;
    grid_dep_wait();

    // this lane's rows of the task: every load goes out before the angles are needed
    const int32_t n_rows = p.n_q_heads + 2 * p.n_kv_heads;
    const int32_t row0 = part * p.iters * rows_at_once + sub;
    const int32_t slot = checked_slot(p, token, lane == 0 && part == 0);
    const int chunks = p.head_dim / 8;
    uint4 a[kRopeMaxIter], b[kRopeMaxIter];
    RopeRow r[kRopeMaxIter];
    const bool turned = u < rot_units;  // this lane's chunks are rotated (in a row that turns)
    // the two 16-byte chunks of the lane's unit
    const int ca = kInterleaved || !turned ? 2 * u : u, cb = kInterleaved || !turned ? 2 * u + 1 : u + rot_units;
#pragma unroll
    for (int i = 0; i < kRopeMaxIter; ++i) {
        const int32_t row = row0 + i * rows_at_once;
        r[i].dst = nullptr;
        if (i < p.iters && sub < rows_at_once && row < n_rows) r[i] = rope_row(p, token, slot, row);
        if (r[i].dst) {
            const uint4 *src = reinterpret_cast<const uint4 *>(r[i].src);
            a[i] = src[ca];
            if (cb < chunks) b[i] = src[cb];
        }
    }
    const int32_t position = __ldg(p.positions + token);
    for (int f = lane; f < half; f += 32)
        table[(f >> 3) * kUnitPitch + (f & 7)] = rope_angle(position, __ldg(p.inv_freq + f), p.factor);
    __syncwarp();
    float2 cs[8];
    if (turned) {
        const float4 *t4 = reinterpret_cast<const float4 *>(table + u * kUnitPitch);
#pragma unroll
        for (int k = 0; k < 4; ++k) {
            const float4 v = t4[k];
            cs[2 * k] = make_float2(v.x, v.y);
            cs[2 * k + 1] = make_float2(v.z, v.w);
        }
    }
#pragma unroll
    for (int i = 0; i < kRopeMaxIter; ++i) {
        if (!r[i].dst) continue;
        if (turned && r[i].turns) {
            uint32_t x[4] = {a[i].x, a[i].y, a[i].z, a[i].w}, y[4] = {b[i].x, b[i].y, b[i].z, b[i].w};
#pragma unroll
            for (int k = 0; k < 4; ++k) {
                if constexpr (kInterleaved) {
                    const float2 v = unpack_bf16x2(x[k]), w = unpack_bf16x2(y[k]);
                    const float2 c = cs[k], d = cs[k + 4];
                    x[k] = pack_bf16x2(v.x * c.x - v.y * c.y, v.y * c.x + v.x * c.y);
                    y[k] = pack_bf16x2(w.x * d.x - w.y * d.y, w.y * d.x + w.x * d.y);
                } else {
                    const float2 v = unpack_bf16x2(x[k]), w = unpack_bf16x2(y[k]);
                    const float2 c = cs[2 * k], d = cs[2 * k + 1];
                    x[k] = pack_bf16x2(v.x * c.x - w.x * c.y, v.y * d.x - w.y * d.y);
                    y[k] = pack_bf16x2(w.x * c.x + v.x * c.y, w.y * d.x + v.y * d.y);
                }
            }
            a[i] = make_uint4(x[0], x[1], x[2], x[3]);
            b[i] = make_uint4(y[0], y[1], y[2], y[3]);
        }
        // a row of values (or one past rotary_dim) keeps its chunks' places
        uint4 *dst = reinterpret_cast<uint4 *>(r[i].dst);
        dst[ca] = a[i];
        if (cb < chunks) dst[cb] = b[i];
    }
}

// Any alignment, strides and even rotary_dim: a thread moves one pair (or one
// value past rotary_dim) of one head row.
__global__ void __launch_bounds__(256) rope_append_any_kernel(const __grid_constant__ RopeParams p) {
    grid_dep_launch();
    grid_dep_wait();
    const int half = p.rotary_dim / 2;
    const int32_t per_row = p.head_dim - half, n_rows = p.n_q_heads + 2 * p.n_kv_heads;
    const int64_t total = static_cast<int64_t>(p.n_tokens) * n_rows * per_row;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * blockDim.x + threadIdx.x; i < total;
         i += static_cast<int64_t>(gridDim.x) * blockDim.x) {
        const int64_t row_of = i / per_row;
        const int32_t e = static_cast<int32_t>(i - row_of * per_row);
        const int32_t token = static_cast<int32_t>(row_of / n_rows), row = static_cast<int32_t>(row_of % n_rows);
        const RopeRow r = rope_row(p, token, checked_slot(p, token, e == 0), row);
        if (!r.dst) continue;
        if (e >= half) {
            r.dst[e + half] = r.src[e + half];
            continue;
        }
        const int x = p.interleaved ? 2 * e : e, y = p.interleaved ? 2 * e + 1 : e + half;
        __nv_bfloat16 u = r.src[x], w = r.src[y];
        if (r.turns) {
            const float2 cs = rope_angle(__ldg(p.positions + token), __ldg(p.inv_freq + e), p.factor);
            const float fu = __bfloat162float(u), fw = __bfloat162float(w);
            u = __float2bfloat16_rn(fu * cs.x - fw * cs.y);
            w = __float2bfloat16_rn(fw * cs.x + fu * cs.y);
        }
        r.dst[x] = u;
        r.dst[y] = w;
    }
}

cudaError_t launch_rope_append(RopeParams p, cudaStream_t st) {
    auto on16 = [](const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
    const bool wide = p.rotary_dim % 16 == 0 && p.q_stride % 8 == 0 && p.k_stride % 8 == 0 && p.v_stride % 8 == 0 &&
                      on16(p.q) && on16(p.k) && on16(p.v) && on16(p.q_out);
    const int64_t sms = device_sm_count();
    const int32_t n_rows = p.n_q_heads + 2 * p.n_kv_heads;
    const int32_t passes = (n_rows + 32 / ((p.head_dim + 15) / 16) - 1) / (32 / ((p.head_dim + 15) / 16));
    // A warp makes up to 4 passes over a token's rows, for its angles; one pass
    // each while that leaves warps idle
    const int32_t parts = (passes + kRopeMaxIter - 1) / kRopeMaxIter;
    p.iters = static_cast<int64_t>(p.n_tokens) * passes <= sms * kRopeWarps * 4 ? 1 : (passes + parts - 1) / parts;
    p.tasks_per_token = (passes + p.iters - 1) / p.iters;
    const int64_t tasks = static_cast<int64_t>(p.n_tokens) * p.tasks_per_token;
    if (wide && tasks <= INT32_MAX - kRopeWarps) {
        p.n_tasks = static_cast<int32_t>(tasks);
        const size_t smem = static_cast<size_t>(kRopeWarps) * (p.rotary_dim / 16) * kUnitPitch * sizeof(float2);
        PdlLaunch l(dim3(static_cast<unsigned>((tasks + kRopeWarps - 1) / kRopeWarps)), dim3(kRopeWarps * 32), smem,
                    st);
        return p.interleaved ? cudaLaunchKernelEx(&l.cfg, rope_append_kernel<true>, p)
                             : cudaLaunchKernelEx(&l.cfg, rope_append_kernel<false>, p);
    }
    const int64_t total = static_cast<int64_t>(p.n_tokens) * n_rows * (p.head_dim - p.rotary_dim / 2);
    const int64_t blocks = (total + 255) / 256;
    PdlLaunch l(dim3(static_cast<unsigned>(blocks < sms * 16 ? blocks : sms * 16)), dim3(256), 0, st);
    return cudaLaunchKernelEx(&l.cfg, rope_append_any_kernel, p);
}

}  // namespace ppas

using namespace ppas;

extern "C" ppas_status ppas_rope_frequencies(int32_t kind, int32_t rotary_dim, double base, double scale,
                                             int32_t original_len, double low, double high, float *h_inv_freq,
                                             float *h_factor) {
    if (rotary_dim < 2 || rotary_dim % 2 || !(base > 1.0) || !std::isfinite(base) || !h_inv_freq || !h_factor)
        return PPAS_ERR_INVALID_ARG;
    if (kind < PPAS_ROPE_PLAIN || kind > PPAS_ROPE_RAMP) return PPAS_ERR_INVALID_ARG;
    if (kind != PPAS_ROPE_PLAIN && (!(scale >= 1.0) || !std::isfinite(scale))) return PPAS_ERR_INVALID_ARG;
    const bool windowed = kind == PPAS_ROPE_BANDS || kind == PPAS_ROPE_RAMP;
    if (windowed && (original_len < 1 || !(low > 0.0) || !(high > low) || !std::isfinite(high)))
        return PPAS_ERR_INVALID_ARG;
    if (kind == PPAS_ROPE_BASE && rotary_dim < 4) return PPAS_ERR_INVALID_ARG;
    constexpr double kTwoPi = 6.283185307179586476925286766559;
    const int32_t half = rotary_dim / 2;
    const double b = kind == PPAS_ROPE_BASE ? base * std::pow(scale, rotary_dim / (rotary_dim - 2.0)) : base;
    double first = 0.0, last = 1.0;  // RAMP: the indices between which frequencies go over to f / scale
    if (kind == PPAS_ROPE_RAMP) {
        auto index_of = [&](double turns) { return half * std::log(original_len / (turns * kTwoPi)) / std::log(base); };
        first = std::fmax(std::floor(index_of(high)), 0.0);
        last = std::fmin(std::ceil(index_of(low)), rotary_dim - 1.0);
        if (!(last > first)) last = first + 0.001;
    }
    for (int32_t i = 0; i < half; ++i) {
        const double f = std::pow(b, -static_cast<double>(i) / half);
        double keep = 1.0;  // share of f itself, the rest is of f / scale
        if (kind == PPAS_ROPE_LINEAR) keep = 0.0;
        if (kind == PPAS_ROPE_BANDS)
            keep = std::fmin(1.0, std::fmax(0.0, (original_len * f / kTwoPi - low) / (high - low)));
        if (kind == PPAS_ROPE_RAMP) keep = 1.0 - std::fmin(1.0, std::fmax(0.0, (i - first) / (last - first)));
        h_inv_freq[i] = static_cast<float>(keep == 1.0 ? f : f * keep + f / scale * (1.0 - keep));
    }
    *h_factor = kind == PPAS_ROPE_RAMP ? static_cast<float>(0.1 * std::log(scale) + 1.0) : 1.0f;
    return PPAS_OK;
}

extern "C" ppas_status ppas_rope_append(const void *q, const void *k, const void *v, int64_t q_stride,
                                        int64_t k_stride, int64_t v_stride, const int32_t *d_positions,
                                        const int32_t *d_slot_mapping, int32_t n_tokens, const float *d_inv_freq,
                                        int32_t rotary_dim, int32_t interleaved, float factor, void *q_out,
                                        void *k_cache, void *v_cache, int32_t num_blocks, int32_t n_q_heads,
                                        int32_t n_kv_heads, int32_t head_dim, int32_t *d_err_flag, void *stream) {
    if (n_tokens < 0 || n_q_heads < 0 || n_kv_heads < 1 || head_dim < 8 || head_dim % 8 != 0 || num_blocks < 1)
        return PPAS_ERR_INVALID_ARG;
    if (rotary_dim < 0 || rotary_dim % 2 || rotary_dim > head_dim || !std::isfinite(factor))
        return PPAS_ERR_INVALID_ARG;
    if (head_dim > kRopeMaxDim || n_q_heads > 65536 || n_kv_heads > 65536) return PPAS_ERR_UNSUPPORTED;
    if (static_cast<int64_t>(num_blocks) * kPage > INT32_MAX) return PPAS_ERR_UNSUPPORTED;
    if (n_tokens == 0) return PPAS_OK;
    const int64_t q_row = static_cast<int64_t>(n_q_heads) * head_dim, kv_row = static_cast<int64_t>(n_kv_heads) * head_dim;
    if (k_stride < kv_row || v_stride < kv_row || (n_q_heads > 0 && q_stride < q_row)) return PPAS_ERR_INVALID_ARG;
    if (!k || !v || !d_positions || !d_slot_mapping || !k_cache || !v_cache || (rotary_dim > 0 && !d_inv_freq) ||
        (n_q_heads > 0 && (!q || !q_out)))
        return PPAS_ERR_INVALID_ARG;
    auto on = [](const void *x, uintptr_t n) { return (reinterpret_cast<uintptr_t>(x) & (n - 1)) == 0; };
    if (!on(q, 2) || !on(k, 2) || !on(v, 2) || !on(q_out, 2) || !on(k_cache, 16) || !on(v_cache, 16) ||
        !on(d_positions, 4) || !on(d_slot_mapping, 4) || !on(d_inv_freq, 4) || !on(d_err_flag, 4))
        return PPAS_ERR_INVALID_ARG;
    if (n_q_heads > 0 && q_out == q && q_stride != q_row) return PPAS_ERR_INVALID_ARG;  // in place: contiguous rows
    RopeParams p = {};
    if (n_q_heads > 0) {
        p.q = static_cast<const __nv_bfloat16 *>(q);
        p.q_out = static_cast<__nv_bfloat16 *>(q_out);
        p.q_stride = q_stride;
    }
    p.k = static_cast<const __nv_bfloat16 *>(k);
    p.v = static_cast<const __nv_bfloat16 *>(v);
    p.k_stride = k_stride;
    p.v_stride = v_stride;
    p.positions = d_positions;
    p.slots = d_slot_mapping;
    p.inv_freq = d_inv_freq;
    p.k_cache = static_cast<__nv_bfloat16 *>(k_cache);
    p.v_cache = static_cast<__nv_bfloat16 *>(v_cache);
    p.err = d_err_flag;
    p.factor = factor;
    p.n_tokens = n_tokens;
    p.num_blocks = num_blocks;
    p.n_q_heads = n_q_heads;
    p.n_kv_heads = n_kv_heads;
    p.head_dim = head_dim;
    p.rotary_dim = rotary_dim;
    p.interleaved = interleaved ? 1 : 0;
    return launch_rope_append(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? PPAS_OK : PPAS_ERR_CUDA;
}
