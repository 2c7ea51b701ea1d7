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
//
// With norms (kNorm) each query and key head x becomes x r w first, w a weight a
// dim, r = 1 / sqrt(mean x^2 + eps), all in fp32 and rounded once behind the
// rotation.  A row is in the registers of one warp, so its sum of squares takes a
// few shuffles and no memory: the bytes are those of the rotation alone.  16384 tokens
// of 32/8 heads in 68.6 us (5.9 TB/s), 2056 of 16/2 in 7.2.
#include <float.h>
#include <math.h>

#include "ppas_device.cuh"
#include "ppas_internal.h"

namespace ppas {
namespace {

constexpr int kRopeWarps = 8;
// CTAs an SM holds of the kernel with norms for heads of 128 (of 80 registers; 16384 tokens of
// 32/8 heads: 68.6 us, with 4 of 64 73.2, with 2 74.5)
constexpr int kNormCtas = 3;
constexpr int kRopeMaxIter = 4;      // 32-lane passes over head rows a warp makes, loads of all in flight
constexpr int kRopeMaxDim = 512;     // head_dim: 16 values a lane
// a unit's 8 (cos, sin) pairs, two pairs of padding after them: the 16-byte
// reads of 8 neighbouring lanes then hit all banks once
constexpr int kUnitPitch = 10;

// the same of a unit's 16 weights, and of 8 cosines, sines and negative sines
constexpr int kWeightPitch = 20, kAnglePitch = 28;
constexpr size_t norm_rope_smem(int head_dim, int rotary_dim) {
    return (2 * ((head_dim + 15) / 16) * static_cast<size_t>(kWeightPitch) +
            static_cast<size_t>(kRopeWarps) * (rotary_dim / 16) * kAnglePitch) * sizeof(float);
}
static_assert(norm_rope_smem(kRopeMaxDim, kRopeMaxDim) <= 48 * 1024, "shared memory without a raised limit");

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

__device__ __forceinline__ float2 mul2(float2 a, float2 b) { return fma2(a, b, make_float2(-0.f, -0.f)); }

// Heads whose squares leave the fp32 range are summed again times a power of two, eps
// with them: by kSquareDown where they pass it (the largest bf16 numbers then stay below 2^59,
// 512 squares of them in range), and by kSquareUp where they are lost below it and
// eps is as small (below 2^-110 all values are less than 2^-55; the least bf16 number's square is then
// 2^-126, the least eps 2^-9).  Elsewhere what a sum has lost, 512 2^-150 at the most, is less than 2^-31 of it,
// or than 2^-40 of eps.
constexpr float kSquareDown = 0x1p-70f, kSquareUp = 0x1p70f;
constexpr float kEpsSmall = 0x1p-100f, kEpsLarge = 0x1p100f;  // eps that is lost itself, or passes the range with a sum
constexpr float kSumSmall = 0x1p-110f;

__device__ __forceinline__ bool in_range(const RopeParams &p, float sum) {
    return sum >= p.sum_least && sum <= p.sum_most;  // (not NaN)
}
// what a sum that is not in range is taken again with, of the values times this
__device__ __forceinline__ float square_scale(float sum) { return sum < 1.f ? kSquareUp : kSquareDown; }
// 1 / sqrt(mean + eps) of a head's sum of squares, or of the one of the values times `scale`
__device__ __forceinline__ float norm_factor(const RopeParams &p, float sum) {
    return rsqrtf(fmaf(sum, p.inv_dim, p.eps));
}
__device__ __forceinline__ float norm_factor(const RopeParams &p, float sum, float scale) {
    return rsqrtf(fmaf(sum, p.inv_dim, p.eps * scale * scale)) * scale;
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
    bool turns;  // (and has a norm)
    bool is_q;
};
__device__ __forceinline__ RopeRow rope_row(const RopeParams &p, int32_t token, int32_t slot, int32_t row) {
    RopeRow r;
    const int64_t t = token;
    if (row < p.n_q_heads) {
        r.src = p.q + t * p.q_stride + row * p.head_dim;
        r.dst = p.q_out + (t * p.n_q_heads + row) * p.head_dim;
        r.turns = r.is_q = true;
        return r;
    }
    row -= p.n_q_heads;
    r.is_q = false;
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

// The same with norms.  A warp takes a run of tasks, and a token's angles with its
// first one; angles and weights lie in shared memory in the order of the lanes that
// read them (in registers they left room for two CTAs an SM: 16384 tokens of 32/8 heads
// 103 us).  What bounds it next is the number of instructions: heads of 128 have a
// kernel of their own (kDim; 0: any), products run on two values at once.
template <bool kInterleaved, int kDim>
__global__ void __launch_bounds__(kRopeWarps * 32, kDim ? kNormCtas : 2)
    norm_rope_append_kernel(const __grid_constant__ RopeParams p) {
    grid_dep_launch();
    extern __shared__ float4 rope_smem[];
    const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
    const int dim = kDim ? kDim : p.head_dim;
    const int units = (dim + 15) / 16, half = p.rotary_dim / 2, rot_units = half / 8;
    const int rows_at_once = 32 / units, chunks = dim / 8;
    const int u = lane % units, sub = lane / units;
    const bool turned = u < rot_units;
    auto first_chunk = [&](int unit) { return kInterleaved || unit >= rot_units ? 2 * unit : unit; };
    auto second_chunk = [&](int unit) { return kInterleaved || unit >= rot_units ? 2 * unit + 1 : unit + rot_units; };
    const int ca = first_chunk(u), cb = second_chunk(u);
    const bool has_row = kDim == 128 || sub < rows_at_once, has_b = kDim == 128 || cb < chunks;
    constexpr int kPitch = kWeightPitch, kTurnPitch = kAnglePitch;
    // [queries, keys][unit][16 weights]; then each warp's angles [unit][8 cosines, 8 sines, the sines' negatives]
    float *const weights = reinterpret_cast<float *>(rope_smem);
    float *const table = weights + 2 * units * kPitch + warp * rot_units * kTurnPitch;
    const int32_t n_turned = p.n_q_heads + p.n_kv_heads, n_rows = n_turned + p.n_kv_heads;
    // this warp's tasks
    const int64_t w = static_cast<int64_t>(blockIdx.x) * kRopeWarps + warp;
    const int64_t n_warps = static_cast<int64_t>(gridDim.x) * kRopeWarps;
    int32_t task = static_cast<int32_t>(p.n_tasks * w / n_warps);
    const int32_t task_end = static_cast<int32_t>(p.n_tasks * (w + 1) / n_warps);
    grid_dep_wait();
    for (int i = threadIdx.x; i < 2 * units * 16; i += kRopeWarps * 32) {
        const int which = i / (units * 16), unit = i / 16 % units, e = i % 16;
        const int d = (e < 8 ? first_chunk(unit) : second_chunk(unit)) * 8 + e % 8;
        const float *const from = which ? p.k_weight : p.q_weight;
        weights[(which * units + unit) * kPitch + e] = from && d < dim ? __ldg(from + d) : 1.f;
    }
    __syncthreads();
    int32_t token = task / p.tasks_per_token, part = task - token * p.tasks_per_token;
    bool angles = false;  // the token's are in the table
    for (; task < task_end; ++task) {
        const int32_t slot = checked_slot(p, token, lane == 0 && part == 0);
        const __nv_bfloat16 *const q = p.q + token * p.q_stride, *const k = p.k + token * p.k_stride;
        const __nv_bfloat16 *const v = p.v + token * p.v_stride;
        const int32_t row0 = part * p.iters * rows_at_once + sub;
        uint4 a[kRopeMaxIter], b[kRopeMaxIter];
#pragma unroll
        for (int i = 0; i < kRopeMaxIter; ++i) {
            const int32_t row = row0 + i * rows_at_once;
            a[i] = b[i] = make_uint4(0, 0, 0, 0);
            if (i < p.iters && has_row && row < n_rows) {
                const __nv_bfloat16 *src = row < p.n_q_heads ? q + row * dim
                                           : row < n_turned  ? k + (row - p.n_q_heads) * dim
                                                             : v + (row - n_turned) * dim;
                const uint4 *from = reinterpret_cast<const uint4 *>(src);
                a[i] = from[ca];
                if (has_b) b[i] = from[cb];
            }
        }
        if (!angles) {
            const int32_t position = __ldg(p.positions + token);
            for (int f = lane; f < half; f += 32) {
                const float2 cs = rope_angle(position, __ldg(p.inv_freq + f), p.factor);
                float *const to = table + (f >> 3) * kTurnPitch + (f & 7);
                to[0] = cs.x;
                to[8] = cs.y;
                to[16] = -cs.y;
            }
            angles = true;
            __syncwarp();
        }
        __nv_bfloat16 *const q_to = p.q_out + static_cast<int64_t>(token) * p.n_q_heads * dim;
        const int64_t in_page =
            (static_cast<int64_t>(slot / kPage) * p.n_kv_heads * kPage + slot % kPage) * dim;
        __nv_bfloat16 *const k_to = p.k_cache + in_page, *const v_to = p.v_cache + in_page;
#pragma unroll
        for (int i = 0; i < kRopeMaxIter; ++i) {
            if (i >= p.iters) break;
            const int32_t row = row0 + i * rows_at_once;
            float2 x[8];  // 8 values of each chunk
            {
                const uint32_t xa[4] = {a[i].x, a[i].y, a[i].z, a[i].w}, xb[4] = {b[i].x, b[i].y, b[i].z, b[i].w};
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    x[e] = unpack_bf16x2(xa[e]);
                    x[4 + e] = unpack_bf16x2(xb[e]);
                }
            }
            // (every lane of the warp: a row's lanes are its units; what a lane did not load is 0)
            auto over_row = [&](float s) {
                if (kDim == 128) {
                    s += __shfl_xor_sync(0xffffffffu, s, 1);
                    s += __shfl_xor_sync(0xffffffffu, s, 2);
                    return s + __shfl_xor_sync(0xffffffffu, s, 4);
                }
                if ((units & (units - 1)) == 0) {
                    for (int o = 1; o < units; o <<= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
                    return s;
                }
                float all = 0.f;
                for (int j = 0; j < units; ++j) all += __shfl_sync(0xffffffffu, s, (sub * units + j) & 31);
                return all;
            };
            float2 s2 = mul2(x[0], x[0]);
#pragma unroll
            for (int e = 1; e < 8; ++e) s2 = fma2(x[e], x[e], s2);
            const float sum = over_row(s2.x + s2.y);
            const bool in = in_range(p, sum);
            float again = 0.f;
            if (__any_sync(0xffffffffu, !in)) {
                const float scale = square_scale(sum);
                float s = 0.f;
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float y0 = x[e].x * scale, y1 = x[e].y * scale;
                    s = fmaf(y0, y0, fmaf(y1, y1, s));
                }
                again = norm_factor(p, over_row(s), scale);
            }
            if (!has_row || row >= n_rows || (row >= p.n_q_heads && slot < 0)) continue;
            if (row < n_turned) {
                const float f = in ? norm_factor(p, sum) : again;
                const float4 *const w4 =
                    reinterpret_cast<const float4 *>(weights + ((row < p.n_q_heads ? 0 : units) + u) * kPitch);
                const float2 ff = make_float2(f, f);
#pragma unroll
                for (int e = 0; e < 4; ++e) {
                    const float4 wt = w4[e];
                    x[2 * e] = mul2(mul2(x[2 * e], ff), make_float2(wt.x, wt.y));
                    x[2 * e + 1] = mul2(mul2(x[2 * e + 1], ff), make_float2(wt.z, wt.w));
                }
                if (turned) {
                    const float *const at = table + u * kTurnPitch;
                    if constexpr (kInterleaved) {  // pair e is (x[e].x, x[e].y)
#pragma unroll
                        for (int e = 0; e < 8; ++e) {
                            const float c = at[e], s = at[8 + e], m = x[e].x;
                            x[e].x = m * c - x[e].y * s;
                            x[e].y = x[e].y * c + m * s;
                        }
                    } else {  // pairs 2 e and 2 e + 1 are (x[e].x, x[4 + e].x) and (x[e].y, x[4 + e].y)
#pragma unroll
                        for (int h = 0; h < 2; ++h) {
                            const float4 c = reinterpret_cast<const float4 *>(at)[h];
                            const float4 s = reinterpret_cast<const float4 *>(at)[2 + h];
                            const float4 z = reinterpret_cast<const float4 *>(at)[4 + h];
                            auto turn = [](float2 &m, float2 &n, float2 c_, float2 s_, float2 z_) {
                                const float2 m0 = m;
                                m = fma2(n, z_, mul2(m, c_));
                                n = fma2(m0, s_, mul2(n, c_));
                            };
                            turn(x[2 * h], x[4 + 2 * h], make_float2(c.x, c.y), make_float2(s.x, s.y),
                                 make_float2(z.x, z.y));
                            turn(x[2 * h + 1], x[4 + 2 * h + 1], make_float2(c.z, c.w), make_float2(s.z, s.w),
                                 make_float2(z.z, z.w));
                        }
                    }
                }
                a[i] = make_uint4(pack_bf16x2(x[0].x, x[0].y), pack_bf16x2(x[1].x, x[1].y), pack_bf16x2(x[2].x, x[2].y),
                                  pack_bf16x2(x[3].x, x[3].y));
                b[i] = make_uint4(pack_bf16x2(x[4].x, x[4].y), pack_bf16x2(x[5].x, x[5].y), pack_bf16x2(x[6].x, x[6].y),
                                  pack_bf16x2(x[7].x, x[7].y));
            }
            uint4 *const to = reinterpret_cast<uint4 *>(
                row < p.n_q_heads ? q_to + row * dim
                                  : (row < n_turned ? k_to + (row - p.n_q_heads) * kPage * dim
                                                    : v_to + (row - n_turned) * kPage * dim));
            to[ca] = a[i];
            if (has_b) to[cb] = b[i];
        }
        __syncwarp();  // the angles have been read
        if (++part == p.tasks_per_token) {
            part = 0;
            ++token;
            angles = false;
        }
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

// The same with norms: a warp has a head row.
__global__ void __launch_bounds__(256) norm_rope_append_any_kernel(const __grid_constant__ RopeParams p) {
    grid_dep_launch();
    grid_dep_wait();
    const int lane = threadIdx.x & 31, half = p.rotary_dim / 2;
    const int32_t n_rows = p.n_q_heads + 2 * p.n_kv_heads;
    const int64_t total = static_cast<int64_t>(p.n_tokens) * n_rows;
    for (int64_t i = static_cast<int64_t>(blockIdx.x) * 8 + (threadIdx.x >> 5); i < total;
         i += static_cast<int64_t>(gridDim.x) * 8) {
        const int32_t token = static_cast<int32_t>(i / n_rows), row = static_cast<int32_t>(i % n_rows);
        const RopeRow r = rope_row(p, token, checked_slot(p, token, lane == 0), row);
        if (!r.dst) continue;  // (the whole warp)
        if (!r.turns) {
            for (int e = lane; e < p.head_dim; e += 32) r.dst[e] = r.src[e];
            continue;
        }
        auto row_sum = [&](float scale) {
            float s = 0.f;
            for (int e = lane; e < p.head_dim; e += 32) {
                const float x = __bfloat162float(r.src[e]) * scale;
                s = fmaf(x, x, s);
            }
            for (int o = 16; o; o >>= 1) s += __shfl_xor_sync(0xffffffffu, s, o);
            return s;
        };
        const float sum = row_sum(1.f);
        const float scale = square_scale(sum);
        const float f = in_range(p, sum) ? norm_factor(p, sum) : norm_factor(p, row_sum(scale), scale);
        const float *const weight = r.is_q ? p.q_weight : p.k_weight;
        const int32_t position = __ldg(p.positions + token);
        auto normed = [&](int e) { return __bfloat162float(r.src[e]) * f * (weight ? __ldg(weight + e) : 1.f); };
        __syncwarp();  // in place: every lane has read the row
        for (int e = lane; e < half; e += 32) {
            const int x = p.interleaved ? 2 * e : e, y = p.interleaved ? 2 * e + 1 : e + half;
            const float2 cs = rope_angle(position, __ldg(p.inv_freq + e), p.factor);
            const float fu = normed(x), fw = normed(y);
            r.dst[x] = __float2bfloat16_rn(fu * cs.x - fw * cs.y);
            r.dst[y] = __float2bfloat16_rn(fw * cs.x + fu * cs.y);
        }
        for (int e = 2 * half + lane; e < p.head_dim; e += 32) r.dst[e] = __float2bfloat16_rn(normed(e));
    }
}

cudaError_t launch_rope_append(RopeParams p, cudaStream_t st) {
    auto on16 = [](const void *x) { return (reinterpret_cast<uintptr_t>(x) & 15u) == 0; };
    const bool wide = p.rotary_dim % 16 == 0 && p.q_stride % 8 == 0 && p.k_stride % 8 == 0 && p.v_stride % 8 == 0 &&
                      on16(p.q) && on16(p.k) && on16(p.v) && on16(p.q_out) && on16(p.q_weight) && on16(p.k_weight);
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
        if (p.norm) {
            // (angles once a token: as many CTAs as the SMs hold at a time of the kernel for heads of 128;
            // of the one for other sizes, of 103 and 110 registers, they hold 2, and a third start behind those)
            l.cfg.dynamicSmemBytes = norm_rope_smem(p.head_dim, p.rotary_dim);
            const unsigned most = static_cast<unsigned>(sms) * kNormCtas;
            if (l.cfg.gridDim.x > most) l.cfg.gridDim.x = most;
            const bool d128 = p.head_dim == 128;
            const auto kernel = p.interleaved ? (d128 ? norm_rope_append_kernel<true, 128> : norm_rope_append_kernel<true, 0>)
                                              : (d128 ? norm_rope_append_kernel<false, 128> : norm_rope_append_kernel<false, 0>);
            return cudaLaunchKernelEx(&l.cfg, kernel, p);
        }
        return p.interleaved ? cudaLaunchKernelEx(&l.cfg, rope_append_kernel<true>, p)
                             : cudaLaunchKernelEx(&l.cfg, rope_append_kernel<false>, p);
    }
    if (p.norm) {
        const int64_t warps = (static_cast<int64_t>(p.n_tokens) * n_rows + 7) / 8;
        PdlLaunch l(dim3(static_cast<unsigned>(warps < sms * 16 ? warps : sms * 16)), dim3(256), 0, st);
        return cudaLaunchKernelEx(&l.cfg, norm_rope_append_any_kernel, p);
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

namespace {

// the checks and the launch of both entry points; norm: with q_weight, k_weight (or NULL) and eps
ppas_status rope_call(const void *q, const void *k, const void *v, int64_t q_stride, int64_t k_stride,
                      int64_t v_stride, const int32_t *d_positions, const int32_t *d_slot_mapping, int32_t n_tokens,
                      const float *d_inv_freq, int32_t rotary_dim, int32_t interleaved, float factor, void *q_out,
                      void *k_cache, void *v_cache, int32_t num_blocks, int32_t n_q_heads, int32_t n_kv_heads,
                      int32_t head_dim, int32_t *d_err_flag, void *stream, bool norm, const float *d_q_weight,
                      const float *d_k_weight, float eps) {
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
    if (!on(d_q_weight, 4) || !on(d_k_weight, 4)) return PPAS_ERR_INVALID_ARG;
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
    p.norm = norm ? 1 : 0;
    p.q_weight = d_q_weight;
    p.k_weight = d_k_weight;
    p.eps = eps;
    p.inv_dim = 1.f / static_cast<float>(head_dim);
    p.sum_least = eps < kEpsSmall ? kSumSmall : 0.f;
    p.sum_most = eps > kEpsLarge ? kEpsLarge : FLT_MAX;  // (eps plus a mean that large is rounded to eps)
    return launch_rope_append(p, static_cast<cudaStream_t>(stream)) == cudaSuccess ? PPAS_OK : PPAS_ERR_CUDA;
}

}  // namespace

extern "C" ppas_status ppas_rope_append(const void *q, const void *k, const void *v, int64_t q_stride,
                                        int64_t k_stride, int64_t v_stride, const int32_t *d_positions,
                                        const int32_t *d_slot_mapping, int32_t n_tokens, const float *d_inv_freq,
                                        int32_t rotary_dim, int32_t interleaved, float factor, void *q_out,
                                        void *k_cache, void *v_cache, int32_t num_blocks, int32_t n_q_heads,
                                        int32_t n_kv_heads, int32_t head_dim, int32_t *d_err_flag, void *stream) {
    return rope_call(q, k, v, q_stride, k_stride, v_stride, d_positions, d_slot_mapping, n_tokens, d_inv_freq,
                     rotary_dim, interleaved, factor, q_out, k_cache, v_cache, num_blocks, n_q_heads, n_kv_heads,
                     head_dim, d_err_flag, stream, false, nullptr, nullptr, 0.f);
}

extern "C" ppas_status ppas_norm_rope_append(const void *q, const void *k, const void *v, int64_t q_stride,
                                             int64_t k_stride, int64_t v_stride, const float *d_q_weight,
                                             const float *d_k_weight, float eps, const int32_t *d_positions,
                                             const int32_t *d_slot_mapping, int32_t n_tokens, const float *d_inv_freq,
                                             int32_t rotary_dim, int32_t interleaved, float factor, void *q_out,
                                             void *k_cache, void *v_cache, int32_t num_blocks, int32_t n_q_heads,
                                             int32_t n_kv_heads, int32_t head_dim, int32_t *d_err_flag, void *stream) {
    if (!(eps > 0.f) || !std::isfinite(eps)) return PPAS_ERR_INVALID_ARG;
    return rope_call(q, k, v, q_stride, k_stride, v_stride, d_positions, d_slot_mapping, n_tokens, d_inv_freq,
                     rotary_dim, interleaved, factor, q_out, k_cache, v_cache, num_blocks, n_q_heads, n_kv_heads,
                     head_dim, d_err_flag, stream, true, d_q_weight, d_k_weight, eps);
}
