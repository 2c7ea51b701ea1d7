// Attention of single-token rows in groups that share a prefix.
//
// With the keys of a row split into the prefix P that its group shares and its
// own O, softmax over both is two partial results joined:
//   m_X = max s_j, l_X = sum 2^(s_j - m_X), o_X = sum 2^(s_j - m_X) v_j  (j in X, s in log2 units)
//   out = (2^(m_P - M) o_P + 2^(m_O - M) o_O) / (2^(m_P - M) l_P + 2^(m_O - M) l_O).
// The prefix's part is the same keys for every row of the group and every
// q-head of a kv-head's group: one matrix of queries against one K, so its K and
// V are read once and the products go to the tensor cores, 128 (row, head) pairs
// to a tile, two tiles to a CTA that share every K/V tile.  One CTA takes one
// piece of a prefix's KV tiles; the roles of its warps are those of the prefill
// kernel (attn_prefill.cu): TMA producers, a Q K^T and a P V issuer, and a softmax
// warpgroup for each Q tile whose threads own a query row each.
// The own keys are read by one row only: they stream through rings of single
// warps, each an equal run of their pages, products by mma.sync with the q-heads
// as 8 columns, on the CTAs after those of the pieces.
// Every partial goes to the workspace in fp32 and a second launch joins them.
//
// Bound by HBM where prefixes and own keys are long (64 rows of up to 1000 own keys after
// 30k shared, 32/8 heads: 53.5 us for 264 MB, 49 of them this launch), by the start
// and end of two launches where they are short (32 rows after 25k, 16/2 heads: 17.7
// us, of which the tiles take 4 and the join 4), and by the tensor cores of the SMs
// that have a piece in large groups (512 rows after 25k: 88.7 us, 1195 TFLOP/s; 128
// pieces of 49 tiles on 152 SMs).
#include <math.h>

#include "attn_decode_body.cuh"
#include "attn_shared.cuh"
#include "ppas_device.cuh"

namespace ppas {
namespace {

constexpr int kKT = kPrefillKT;
constexpr int kPagesPerTile = kKT / kPage;
constexpr int kNK = 3;                      // K ring depth
constexpr int kNV = 2;                      // V ring depth
constexpr uint32_t kBox = 2048;             // one TMA box: 16 rows x 128 B
constexpr uint32_t kHalf = 16384;           // 128 rows x 128 B (64 columns)
constexpr uint32_t kTileBytes = 2 * kHalf;  // a Q, K or V tile: 128 rows x 256 B

constexpr uint32_t kOffQ = 0;
constexpr uint32_t kOffK = kOffQ + 2 * kTileBytes;
constexpr uint32_t kOffV = kOffK + kNK * kTileBytes;
constexpr uint32_t kOffBar = kOffV + kNV * kTileBytes;
enum : int {
    B_Q = 0,                 // [tile]
    B_KFULL = B_Q + 2,
    B_KEMPTY = B_KFULL + kNK,
    B_VFULL = B_KEMPTY + kNK,
    B_VEMPTY = B_VFULL + kNV,
    B_SFULL = B_VEMPTY + kNV,  // [tile]
    B_SFREE = B_SFULL + 2,     // the S columns have been read out
    B_PFULL = B_SFREE + 1,     // [tile]
    B_ODONE = B_PFULL + 2,     // [tile]
    B_QKI = B_ODONE + 2,       // [4]: Q K^T batch n, issued (n mod 4)
    B_DRAIN = B_QKI + 4,
    B_COUNT = B_DRAIN + 1
};
constexpr uint32_t kOffTmem = kOffBar + B_COUNT * 8;
constexpr uint32_t kOffAbort = kOffTmem + 4;
static_assert(kOffAbort + 4 <= kOffBar + 256, "barrier area");
constexpr uint32_t kSmemBytes = kOffBar + 256 + 1024;  // + alignment slack
static_assert(kSmemBytes <= 232448, "shared memory per CTA");
constexpr uint32_t kTmemCols = 512;
constexpr uint32_t kColS = 0;    // one S (128 columns) that the two tiles use in turn
constexpr uint32_t kColP = 128;  // P of tile t at kColP + 64 t
constexpr uint32_t kColO = 256;  // O of tile t at kColO + 128 t
constexpr float kRescaleThreshold = 8.0f;  // log2 units
constexpr int kThreads = 512;
constexpr int kMmaWarp = 4;
constexpr int kQWarp = 6;
constexpr int kSoftmaxWarp0 = 8;
// register split: 8 warps x 56 + 8 warps x 200 = 512 threads x 128 at launch
constexpr int kRegsSmall = 56;
constexpr int kRegsLarge = 200;
static_assert(8 * 32 * kRegsSmall + 8 * 32 * kRegsLarge <= kThreads * 128, "register split");

constexpr uint32_t kIdescQK = idesc_bf16_f32(128, kKT, false, false);  // B = K rows (K-major)
constexpr uint32_t kIdescPV = idesc_bf16_f32(128, 128, false, true);   // B = V rows (MN-major)

// rings of own keys: one a warp
constexpr int kOwnStages = 3;
constexpr uint32_t kOwnStageBytes = 4 * kBox;  // K lo, K hi, V lo, V hi
constexpr uint32_t kOwnQBytes = 8 * kRowBytes;  // q-heads of a kv-head; a warp has two of them, pair by pair
constexpr uint32_t kOwnOffQ = kSharedWarps * kOwnStages * kOwnStageBytes;
constexpr uint32_t kOwnOffBar = kOwnOffQ + kSharedWarps * 2 * kOwnQBytes;
static_assert(kOwnOffBar + kSharedWarps * kOwnStages * 8 + 1024 <= kSmemBytes, "own rings");

__device__ __forceinline__ void bulk_load(uint32_t dst, const void *src, uint32_t bytes, uint32_t bar) {
    asm volatile("cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];" ::"r"(dst),
                 "l"(src), "r"(bytes), "r"(bar)
                 : "memory");
}

// One piece of a prefix (all 512 threads).
template <class P>
__device__ __forceinline__ void prefix_cta(const CUtensorMap &tm_q, const CUtensorMap &tm_k, const CUtensorMap &tm_v,
                                           const P &p, int piece) {
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_s = smem_u32(smem_raw);
    const uint32_t sb = (raw_s + 1023u) & ~1023u;  // 1024-aligned for the 128-byte swizzle
    uint8_t *const sg = smem_raw + (sb - raw_s);
    const int tid = threadIdx.x, lane = tid & 31;
    const int warp = __shfl_sync(0xffffffffu, tid >> 5, 0);  // (uniform)

    const SharedPiece pc = p.pieces[piece];
    const SharedGroup grp = p.groups[pc.group];
    const int n_kt = pc.kt1 - pc.kt0;
    // query rows (row, head of the group) of this piece's tiles that exist
    const int rows_valid = grp.n_rows * p.group - pc.mu * p.tiles * kTileQ;
    const int nt = p.tiles == 2 && rows_valid > kTileQ ? 2 : 1;

    auto bar = [&](int i) { return sb + kOffBar + 8u * static_cast<uint32_t>(i); };
    volatile int *abort_flag = reinterpret_cast<volatile int *>(sg + kOffAbort);
    // pages of KV tile j that are part of the prefix
    auto pages_in = [&](int j) { return min(kPagesPerTile, grp.prefix / kPage - j * kPagesPerTile); };

    if (warp == kMmaWarp) {
        tmem_alloc(sb + kOffTmem, kTmemCols);
        tmem_relinquish();
    }
    if (tid == 0) {
        for (int t = 0; t < 2; ++t) mbar_init(bar(B_Q + t), 1);
        for (int s = 0; s < kNK; ++s) {
            mbar_init(bar(B_KFULL + s), 2);  // two producer warps per tile
            mbar_init(bar(B_KEMPTY + s), 1);
        }
        for (int s = 0; s < kNV; ++s) {
            mbar_init(bar(B_VFULL + s), 2);
            mbar_init(bar(B_VEMPTY + s), 1);
        }
        for (int t = 0; t < 2; ++t) {
            mbar_init(bar(B_SFULL + t), 1);
            mbar_init(bar(B_PFULL + t), 4);
            mbar_init(bar(B_ODONE + t), 1);
        }
        mbar_init(bar(B_SFREE), 4);
        for (int i = 0; i < 4; ++i) mbar_init(bar(B_QKI + i), 1);
        mbar_init(bar(B_DRAIN), 2);
        *abort_flag = 0;
        fence_mbar_init();
        prefetch_tmap(&tm_q);
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
    }
    tc_fence_before();
    __syncthreads();
    tc_fence_after();
    const uint32_t tmem = __shfl_sync(0xffffffffu, *reinterpret_cast<volatile uint32_t *>(sg + kOffTmem), 0);
    // the set-up above overlaps the kernel before this one on the stream;
    // global memory only after it
    grid_dep_wait();
    int issued = 0;  // KV tiles (Q tiles) whose copies this warp has issued

    if (warp < 4) {
        // ------------------------------------------------------------ K/V producers
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsSmall));
        const bool is_v = warp >= 2;
        const int pg_lo = (warp & 1) * (kPagesPerTile / 2);  // this warp's pages of each tile
        const int ns = is_v ? kNV : kNK;
        const CUtensorMap *tm = is_v ? &tm_v : &tm_k;
        const uint32_t ring = sb + (is_v ? kOffV : kOffK);
        const int full0 = is_v ? B_VFULL : B_KFULL, empty0 = is_v ? B_VEMPTY : B_KEMPTY;
        const int32_t *table = p.block_tables + static_cast<int64_t>(grp.row0) * p.table_stride;
        const int pg = pg_lo + (lane & 3);  // lane i (mod 4) looks after page pg_lo + i
        int id = 0;
        auto load_id = [&](int j) { id = pg < pages_in(j) ? __ldg(table + j * kPagesPerTile + pg) : 0; };
        load_id(pc.kt0);
        for (int g = 0; g < n_kt; ++g) {
            const int s = g % ns;
            const int np = max(0, min(kPagesPerTile / 2, pages_in(pc.kt0 + g) - pg_lo));
            if (pg - pg_lo < np && (id < 0 || id >= p.num_blocks)) {
                if (lane < 4) report_error(p.err, PPAS_DEVERR_BAD_INDEX);
                id = 0;  // keep the barrier's byte count consistent
            }
            const int row = (id * p.n_kv_heads + pc.kvh) * kPage;
            if (g + 1 < n_kt) load_id(pc.kt0 + g + 1);
            if (g >= ns && !mbar_wait_warp(bar(empty0 + s), ((g / ns) & 1) ^ 1, p.err)) {
                *abort_flag = 1;
                break;
            }
            int rows[kPagesPerTile / 2];
#pragma unroll
            for (int i = 0; i < kPagesPerTile / 2; ++i) rows[i] = __shfl_sync(0xffffffffu, row, i);
            if (elect_one()) {
                const uint32_t b = bar(full0 + s);
                mbar_expect_tx(b, static_cast<uint32_t>(np) * 2 * kBox);
                const uint32_t dst = ring + s * kTileBytes + pg_lo * kBox;
#pragma unroll
                for (int i = 0; i < kPagesPerTile / 2; ++i)
                    if (i < np) {
                        tma_load_2d(dst + i * kBox, tm, 0, rows[i], b);
                        tma_load_2d(dst + kHalf + i * kBox, tm, 64, rows[i], b);
                    }
            }
            __syncwarp();
            ++issued;
        }
    } else if (warp < kSoftmaxWarp0) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsSmall));
        if (warp == kMmaWarp) {
            // -------------------------------------------------------- Q K^T issuer
            const uint64_t dq0 = smem_desc_sw128(sb + kOffQ, 16, 1024);
            const uint64_t dk0 = smem_desc_sw128(sb + kOffK, 16, 1024);
            bool ok = true;
            int n = 0;  // S tiles so far
            for (int g = 0; ok && g < n_kt; ++g) {
                const int sk = g % kNK;
                if (!mbar_wait_warp(bar(B_KFULL + sk), (g / kNK) & 1, p.err)) { ok = false; break; }
                const uint64_t dk = dk0 + ((sk * kTileBytes) >> 4);
                for (int t = 0; t < nt; ++t, ++n) {
                    if (g == 0 && !mbar_wait_warp(bar(B_Q + t), 0, p.err)) { ok = false; break; }
                    // the S columns, once the softmax before has read them out
                    if (n >= 1 && !mbar_wait_warp(bar(B_SFREE), (n - 1) & 1, p.err)) { ok = false; break; }
                    tc_fence_after();
                    const uint64_t dq = dq0 + ((t * kTileBytes) >> 4);
                    if (elect_one()) {
#pragma unroll
                        for (int kk = 0; kk < 8; ++kk) {
                            const uint32_t o = (kk >> 2) * kHalf + (kk & 3) * 32;
                            umma_bf16(tmem + kColS, dq + (o >> 4), dk + (o >> 4), kIdescQK, kk > 0 ? 1u : 0u);
                        }
                        umma_commit(bar(B_SFULL + t));
                        mbar_arrive(bar(B_QKI + (n & 3)));  // P V (n - nt) may follow
                        if (t == nt - 1) umma_commit(bar(B_KEMPTY + sk));
                    }
                    __syncwarp();
                }
            }
            if (!ok) *abort_flag = 1;
            // every MMA issued so far completes before TMEM is released
            if (elect_one()) umma_commit(bar(B_DRAIN));
            __syncwarp();
            mbar_wait(bar(B_DRAIN), 0, p.err);
        } else if (warp == kMmaWarp + 1) {
            // -------------------------------------------------------- P V issuer
            const uint64_t dv0 = smem_desc_sw128(sb + kOffV, kHalf, 1024);
            bool ok = true;
            for (int g = 0; ok && g < n_kt; ++g) {
                const int sv = g % kNV;
                if (!mbar_wait_warp(bar(B_VFULL + sv), (g / kNV) & 1, p.err)) { ok = false; break; }
                const uint64_t dv = dv0 + ((sv * kTileBytes) >> 4);
                const int chunks = pages_in(pc.kt0 + g);
                for (int t = 0; t < nt; ++t) {
                    if (!mbar_wait_warp(bar(B_PFULL + t), g & 1, p.err)) { ok = false; break; }
                    // behind the Q K^T batch after the next one, as in the prefill kernel
                    if (g + 1 < n_kt) {
                        const int gate = (g + 1) * nt + t;
                        if (!mbar_wait_warp(bar(B_QKI + (gate & 3)), (gate >> 2) & 1, p.err)) { ok = false; break; }
                    }
                    tc_fence_after();
                    // O_t += P_t V(j), P_t from TMEM; the first tile overwrites O_t
                    const uint32_t d_p = tmem + kColP + t * 64, d_o = tmem + kColO + t * 128;
                    if (elect_one()) {
                        for (int kk = 0; kk < chunks; ++kk)
                            umma_bf16_ts(d_o, d_p + kk * 8, dv + ((kk * 2048) >> 4), kIdescPV,
                                         (g > 0 || kk > 0) ? 1u : 0u);
                        umma_commit(bar(B_ODONE + t));
                        if (t == nt - 1) umma_commit(bar(B_VEMPTY + sv));
                    }
                    __syncwarp();
                }
            }
            if (!ok) *abort_flag = 1;
            if (elect_one()) umma_commit(bar(B_DRAIN));
            __syncwarp();
            mbar_wait(bar(B_DRAIN), 0, p.err);
        } else if (warp == kQWarp) {
            // -------------------------------------------------------- Q loader
            // a box holds the group's heads of 128 / group rows: 128 query rows
            const int per = kTileQ / p.group;
            for (int t = 0; t < nt; ++t) {
                const int row = grp.row0 + (pc.mu * p.tiles + t) * per;
                if (elect_one()) {
                    mbar_expect_tx(bar(B_Q + t), kTileBytes);
                    tma_load_3d(sb + kOffQ + t * kTileBytes, &tm_q, 0, pc.kvh * p.group, row, bar(B_Q + t));
                    tma_load_3d(sb + kOffQ + t * kTileBytes + kHalf, &tm_q, 64, pc.kvh * p.group, row, bar(B_Q + t));
                }
                __syncwarp();
                ++issued;
            }
        }
    } else {
        // ------------------------------------------------------------ softmax warpgroups
        asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsLarge));
        const int t = (warp - kSoftmaxWarp0) / 4;
        if (t < nt) {
            const int wq = warp & 3;
            const int r = wq * 32 + lane;  // query row == TMEM lane
            // a warp whose rows are all past the group's takes part in the
            // barriers alone (its lanes of P and O hold anything)
            const bool live = t * kTileQ + wq * 32 < rows_valid;
            const uint32_t t_lane = tmem + (static_cast<uint32_t>(wq * 32) << 16);
            const uint32_t t_s = t_lane + kColS, t_p = t_lane + kColP + t * 64, t_o = t_lane + kColO + t * 128;
            const float sl2 = p.scale_log2;
            bool ok = true;
            float m_used = -INFINITY, l_run = 0.f;
            for (int g = 0; ok && g < n_kt; ++g) {
                ok = mbar_wait_warp(bar(B_SFULL + t), g & 1, p.err);
                if (!ok) break;
                tc_fence_after();
                if (!live) {
                    tc_fence_before();
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(B_SFREE));
                    if (g >= 1) ok = mbar_wait_warp(bar(B_ODONE + t), (g - 1) & 1, p.err);
                    if (!ok) break;
                    __syncwarp();
                    if (lane == 0) mbar_arrive(bar(B_PFULL + t));
                    continue;
                }
                float s[kKT];
                tmem_ld128_sync(t_s, s);
                // S is in registers: the other tile's Q K^T may overwrite it
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B_SFREE));
                const int keys = grp.prefix - (pc.kt0 + g) * kKT;  // of this tile and those after it
                if (keys < kKT) {
                    // pages past the prefix were not loaded: a multiple of 16 keys is left
#pragma unroll
                    for (int i = 0; i < kKT; ++i)
                        if (i >= keys) s[i] = -INFINITY;
                }
                float mx0 = fmaxf(s[0], s[4]), mx1 = fmaxf(s[1], s[5]);
                float mx2 = fmaxf(s[2], s[6]), mx3 = fmaxf(s[3], s[7]);
#pragma unroll
                for (int i = 8; i < kKT; i += 8) {
                    mx0 = max3(mx0, s[i], s[i + 4]);
                    mx1 = max3(mx1, s[i + 1], s[i + 5]);
                    mx2 = max3(mx2, s[i + 2], s[i + 6]);
                    mx3 = max3(mx3, s[i + 3], s[i + 7]);
                }
                const float m_cand = max3(fmaxf(mx0, mx1), mx2, mx3) * sl2;
                // the maximum is only raised, and O rescaled, when it grows by 2^8
                const bool need = m_cand > m_used + kRescaleThreshold;
                float alpha = 1.f;
                if (need) {
                    alpha = ex2(m_used - m_cand);
                    m_used = m_cand;
                }
                const float neg_m = m_used == -INFINITY ? 0.f : -m_used;
                const float2 sl2x2 = make_float2(sl2, sl2), negx2 = make_float2(neg_m, neg_m);
                float2 ra = make_float2(0.f, 0.f), rb = make_float2(0.f, 0.f);
                // P is rounded to bf16 for the tensor core (its sum l is not): 2^-9 of
                // a weight, averaged over the keys, under the output's own rounding
                uint32_t pk[4][16];
#pragma unroll
                for (int q = 0; q < 4; ++q) {
#pragma unroll
                    for (int i = 0; i < 32; i += 4) {
                        const float *v = s + 32 * q + i;
                        const float2 xa = fma2(make_float2(v[0], v[1]), sl2x2, negx2);
                        const float2 xb = fma2(make_float2(v[2], v[3]), sl2x2, negx2);
                        const float2 ea = make_float2(ex2(xa.x), ex2(xa.y)), eb = make_float2(ex2(xb.x), ex2(xb.y));
                        ra = add2(ra, ea);
                        rb = add2(rb, eb);
                        pk[q][i / 2] = pack_bf16x2(ea.x, ea.y);
                        pk[q][i / 2 + 1] = pack_bf16x2(eb.x, eb.y);
                    }
                }
                // P V (g-1) has read the P before and O is stable
                if (g >= 1) {
                    ok = mbar_wait_warp(bar(B_ODONE + t), (g - 1) & 1, p.err);
                    if (!ok) break;
                    tc_fence_after();
                }
#pragma unroll
                for (int q = 0; q < 4; ++q) tmem_st16(t_p + 16 * q, pk[q]);
                l_run = l_run * alpha + ((ra.x + ra.y) + (rb.x + rb.y));
                if (g >= 1 && __any_sync(0xffffffffu, need)) {
#pragma unroll 1
                    for (int c4 = 0; c4 < 4; ++c4) {
                        float v[32];
                        tmem_ld32_sync(t_o + c4 * 32, v);
#pragma unroll
                        for (int i = 0; i < 32; ++i) v[i] *= alpha;
                        tmem_st32_f(t_o + c4 * 32, v);
                    }
                }
                tmem_wait_st();
                tc_fence_before();
                __syncwarp();
                if (lane == 0) mbar_arrive(bar(B_PFULL + t));
            }
            // ---- the piece's partial: O as 32 chunks of [128 rows][4 floats], so
            // that a store instruction of a warp writes 512 contiguous bytes
            if (ok) ok = __all_sync(0xffffffffu, mbar_wait(bar(B_ODONE + t), (n_kt - 1) & 1, p.err));
            if (ok && live) {
                tc_fence_after();
                const int64_t b = static_cast<int64_t>(piece) * p.tiles + t;
                float4 *dst = reinterpret_cast<float4 *>(p.pre_o) + b * (kHeadDim / 4) * kTileQ + r;
#pragma unroll 1
                for (int c4 = 0; c4 < 4; ++c4) {
                    float v[32];
                    tmem_ld32_sync(t_o + c4 * 32, v);
#pragma unroll
                    for (int i = 0; i < 8; ++i)
                        __stcg(dst + (c4 * 8 + i) * kTileQ, make_float4(v[4 * i], v[4 * i + 1], v[4 * i + 2], v[4 * i + 3]));
                }
                __stcg(p.pre_ml + (b * kTileQ + r) * 2, m_used);
                __stcg(p.pre_ml + (b * kTileQ + r) * 2 + 1, l_run);
            }
            if (!ok) *abort_flag = 1;
        }
    }

    tc_fence_before();
    __syncthreads();
    if (warp == kMmaWarp) {
        tc_fence_after();
        tmem_dealloc(tmem, kTmemCols);
    }
    // a wait ran out: the copies in flight land before the CTA leaves
    if (*abort_flag && issued > 0) {
        const bool q = warp == kQWarp, v = warp >= 2;
        ring_land(bar(q ? B_Q : v ? B_VFULL : B_KFULL), issued, q ? nt : v ? kNV : kNK, lane);
    }
}

// A place in the line of own pages: page `page` of (row, kv-head), one of `pages`.
struct OwnAt {
    int32_t row, kvh, page, pages;
};

// the first place at or after the one given that exists (rows without own keys are left out)
template <class P>
__device__ __forceinline__ void own_settle(const P &p, OwnAt &a) {
    while (a.page >= a.pages) {
        a.page = 0;
        if (a.pages == 0 || ++a.kvh == p.n_kv_heads) {
            a.kvh = 0;
            if (++a.row >= p.n_rows) {
                a.pages = 1;  // past the end (nobody reads there)
                return;
            }
            a.pages = (p.rows[a.row].own + kPage - 1) / kPage;
        }
    }
}
// n places on, within the pair or just past its end
template <class P>
__device__ __forceinline__ OwnAt own_after(const P &p, const OwnAt &a, int32_t n) {
    OwnAt b = a;
    b.page += n;
    own_settle(p, b);
    return b;
}

// place `at` of the line
template <class P>
__device__ __forceinline__ OwnAt own_place(const P &p, int32_t at) {
    int lo = 0, hi = p.n_rows - 1;  // the last row that begins at or before it
    while (lo < hi) {
        const int mid = (lo + hi + 1) >> 1;
        if (p.rows[mid].page0 <= at) lo = mid; else hi = mid - 1;
    }
    OwnAt a;
    a.row = lo;
    a.pages = (p.rows[lo].own + kPage - 1) / kPage;
    const int32_t local = at - p.rows[lo].page0;
    a.kvh = a.pages ? local / a.pages : 0;
    a.page = local - a.kvh * a.pages;
    return a;
}

// Block ids of 32 own pages of a row, a lane each.  A row of up to 32 pages has
// one such window for all of its kv-heads.
struct OwnIds {
    int32_t row, page0, id;
};
template <class P>
__device__ __forceinline__ OwnIds own_ids(const P &p, const OwnAt &a, int lane) {
    OwnIds w = {a.row, a.page & ~31, 0};
    if (a.row < p.n_rows && w.page0 + lane < a.pages) {
        w.id = __ldg(p.block_tables + static_cast<int64_t>(a.row) * p.table_stride + p.rows[a.row].table + w.page0 + lane);
        if (w.id < 0 || w.id >= p.num_blocks) {
            report_error(p.err, PPAS_DEVERR_BAD_INDEX);
            w.id = 0;
        }
    }
    return w;
}
// the first place after a's window
template <class P>
__device__ __forceinline__ OwnAt own_past_window(const P &p, const OwnAt &a) {
    OwnAt b = a;
    if (a.pages <= 32) {
        b.kvh = p.n_kv_heads - 1;
        b.page = a.pages;
    } else {
        b.page = (a.page & ~31) + 32;
    }
    own_settle(p, b);
    return b;
}

// Warp `w` of those that work on own keys: pages [w, w + 1) * p.warp_pages of the line.
template <class P>
__device__ __forceinline__ void own_warp(const CUtensorMap &tm_k, const CUtensorMap &tm_v, const P &p, int w) {
    using namespace decode_detail;
    extern __shared__ uint8_t smem_raw[];
    const uint32_t raw_s = smem_u32(smem_raw);
    const uint32_t sb = (raw_s + 1023u) & ~1023u;
    uint8_t *const sg = smem_raw + (sb - raw_s);
    const int lane = threadIdx.x & 31;
    const int warp = __shfl_sync(0xffffffffu, static_cast<int>(threadIdx.x >> 5), 0);
    const uint32_t ring = sb + warp * kOwnStages * kOwnStageBytes;
    const uint32_t q_slots = kOwnOffQ + warp * 2 * kOwnQBytes;  // from sb
    auto bar = [&](int st) { return sb + kOwnOffBar + (warp * kOwnStages + st) * 8u; };
    if (lane == 0) {
        for (int st = 0; st < kOwnStages; ++st) mbar_init(bar(st), 1);
        fence_mbar_init();
        prefetch_tmap(&tm_k);
        prefetch_tmap(&tm_v);
    }
    const int32_t first = w * p.warp_pages;
    const int32_t count = max(0, min(p.warp_pages, p.own_pages - first));
    OwnAt at = {p.n_rows, 0, 0, 1};  // past the end: no ids to load
    if (count > 0) at = own_place(p, first);
    __syncwarp();
    grid_dep_wait();

    const int hr = lane >> 2, c = lane & 3, g = p.group;
    const int mi = lane >> 3, ri = lane & 7;
    const float sl2 = p.scale_log2;
    // pages are issued up to kOwnStages ahead of use, their ids loaded a window
    // ahead; a pair's queries come with its first page, into one of two slots
    int issued = 0, consumed = 0, pairs = 0, pairs_done = 0;
    OwnAt ahead = at;
    OwnIds ids = own_ids(p, at, lane), next_ids = own_ids(p, own_past_window(p, at), lane);
    auto top_up = [&]() {
        while (issued - consumed < kOwnStages && issued < count) {
            const bool opens = issued == 0 || ahead.page == 0;
            if (opens && pairs - pairs_done == 2) break;
            if (ahead.row != ids.row || (ahead.page & ~31) != ids.page0) {
                ids = next_ids;
                next_ids = own_ids(p, own_past_window(p, ahead), lane);
            }
            const int blk = __shfl_sync(0xffffffffu, ids.id, ahead.page & 31);
            const int r = __shfl_sync(0xffffffffu, (blk * p.n_kv_heads + ahead.kvh) * kPage, 0);
            const int st = issued % kOwnStages;
            if (elect_one()) {
                const uint32_t dst = ring + st * kOwnStageBytes, b = bar(st);
                mbar_expect_tx(b, kOwnStageBytes + (opens ? g * kRowBytes : 0));
                tma_load_2d(dst, &tm_k, 0, r, b);
                tma_load_2d(dst + kBox, &tm_k, 64, r, b);
                tma_load_2d(dst + 2 * kBox, &tm_v, 0, r, b);
                tma_load_2d(dst + 3 * kBox, &tm_v, 64, r, b);
                if (opens)
                    bulk_load(sb + q_slots + (pairs & 1) * kOwnQBytes,
                              p.q + (static_cast<int64_t>(ahead.row) * p.n_q_heads + ahead.kvh * g) * kHeadDim,
                              g * kRowBytes, b);
            }
            __syncwarp();
            ++issued;
            pairs += opens;
            ahead = own_after(p, ahead, 1);
        }
    };
    if (count > 0) top_up();
    bool ok = true;
    while (consumed < count) {
        const int here = min(at.pages - at.page, count - consumed);  // pages of the (row, kv-head) at hand
        const int last = (p.rows[at.row].own + kPage - 1) % kPage + 1;  // keys of the pair's last page
        // this lane: tokens hr, hr + 8 of a page's S, head dims 16 n + hr (+ 8) of
        // O, heads 2c, 2c + 1 of both
        float m0 = -INFINITY, m1 = -INFINITY, l0 = 0.f, l1 = 0.f;
        float o[8][4];
#pragma unroll
        for (int n = 0; n < 8; ++n) o[n][0] = o[n][1] = o[n][2] = o[n][3] = 0.f;
        uint32_t qb[8][2];  // Q as the B operand: n = the group's heads, k = head dims
        for (int i = 0; i < here; ++i) {
            const int st = consumed % kOwnStages;
            ok = mbar_wait_warp(bar(st), (consumed / kOwnStages) & 1, p.err);
            if (!ok) break;
            if (i == 0) {
                const uint32_t *qrow =
                    reinterpret_cast<const uint32_t *>(sg + q_slots + (pairs_done & 1) * kOwnQBytes + hr * kRowBytes);
#pragma unroll
                for (int kk = 0; kk < 8; ++kk) {
                    qb[kk][0] = hr < g ? qrow[kk * 8 + c] : 0u;
                    qb[kk][1] = hr < g ? qrow[kk * 8 + 4 + c] : 0u;
                }
            }
            const int valid = at.page + i + 1 < at.pages ? kPage : last;
            const uint32_t kb = ring + st * kOwnStageBytes, vb = kb + 2 * kBox;
            if (valid < kPage) {
                // tokens past the context: zero their V rows so that 0 * V stays 0
                uint8_t *vg = sg + (vb - sb);
                const int n = (kPage - valid) * 8;
                for (int x = lane; x < 2 * n; x += 32) {
                    const int half = x / n, rr = valid + (x % n) / 8, ch = x % 8;
                    *reinterpret_cast<uint4 *>(vg + half * kBox + rr * 128 + ch * 16) = make_uint4(0, 0, 0, 0);
                }
                fence_proxy_async_smem();
                __syncwarp();
            }
            // S^T = K Q^T: 16 tokens x 8 heads
            float sa[4] = {0.f, 0.f, 0.f, 0.f}, sc[4] = {0.f, 0.f, 0.f, 0.f};
#pragma unroll
            for (int kk = 0; kk < 8; kk += 2) {
                uint32_t a[4];
                ldsm_x4(kb + swz((mi & 1) * 8 + ri, kk * 2 + (mi >> 1)), a[0], a[1], a[2], a[3]);
                mma_bf16_16816(sa, a, qb[kk][0], qb[kk][1]);
                ldsm_x4(kb + swz((mi & 1) * 8 + ri, kk * 2 + 2 + (mi >> 1)), a[0], a[1], a[2], a[3]);
                mma_bf16_16816(sc, a, qb[kk + 1][0], qb[kk + 1][1]);
            }
            const float x0 = hr < valid ? (sa[0] + sc[0]) * sl2 : -INFINITY;  // (token hr, head 2c)
            const float x1 = hr < valid ? (sa[1] + sc[1]) * sl2 : -INFINITY;
            const float x2 = hr + 8 < valid ? (sa[2] + sc[2]) * sl2 : -INFINITY;  // (token hr + 8, head 2c)
            const float x3 = hr + 8 < valid ? (sa[3] + sc[3]) * sl2 : -INFINITY;
            float mx0 = fmaxf(x0, x2), mx1 = fmaxf(x1, x3);
#pragma unroll
            for (int o_ = 4; o_ <= 16; o_ <<= 1) {
                mx0 = fmaxf(mx0, __shfl_xor_sync(0xffffffffu, mx0, o_));
                mx1 = fmaxf(mx1, __shfl_xor_sync(0xffffffffu, mx1, o_));
            }
            mx0 = fmaxf(m0, mx0);
            mx1 = fmaxf(m1, mx1);
            // (while every score so far is -inf, all weights are 0 and not 2^(-inf + inf))
            const float s0 = mx0 == -INFINITY ? 0.f : mx0, s1 = mx1 == -INFINITY ? 0.f : mx1;
            const float al0 = ex2(m0 - s0), al1 = ex2(m1 - s1);
            m0 = mx0;
            m1 = mx1;
            const float e0 = ex2(x0 - s0), e1 = ex2(x1 - s1), e2 = ex2(x2 - s0), e3 = ex2(x3 - s1);
            l0 = l0 * al0 + (e0 + e2);
            l1 = l1 * al1 + (e1 + e3);
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                o[n][0] *= al0;
                o[n][1] *= al1;
                o[n][2] *= al0;
                o[n][3] *= al1;
            }
            // O^T += V^T P^T: 16 head dims x 8 heads at a time, k over the tokens
            const uint32_t p0 = movmatrix_t(pack_bf16x2(e0, e1)), p1 = movmatrix_t(pack_bf16x2(e2, e3));
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                uint32_t a[4];
                ldsm_x4_t(vb + swz((mi >> 1) * 8 + ri, n * 2 + (mi & 1)), a[0], a[1], a[2], a[3]);
                mma_bf16_16816(o[n], a, p0, p1);
            }
            __syncwarp();
            ++consumed;
            top_up();
        }
        if (!ok) break;
        // ---- the pair's partial
#pragma unroll
        for (int o_ = 4; o_ <= 16; o_ <<= 1) {
            l0 += __shfl_xor_sync(0xffffffffu, l0, o_);
            l1 += __shfl_xor_sync(0xffffffffu, l1, o_);
        }
        const int64_t slot = static_cast<int64_t>(at.row) * p.n_kv_heads + at.kvh + w;
        float *const po = p.own_o + slot * g * kHeadDim;
        float2 *const pml = reinterpret_cast<float2 *>(p.own_ml) + slot * g;
#pragma unroll
        for (int x = 0; x < 2; ++x) {
            const int hh = 2 * c + x;
            if (hh >= g) continue;
            if (hr == 0) __stcg(pml + hh, x ? make_float2(m1, l1) : make_float2(m0, l0));
            float *dst = po + hh * kHeadDim + hr;
#pragma unroll
            for (int n = 0; n < 8; ++n) {
                __stcg(dst + 16 * n, o[n][x]);
                __stcg(dst + 16 * n + 8, o[n][2 + x]);
            }
        }
        at = own_after(p, at, here);
        ++pairs_done;
        __syncwarp();
        top_up();
    }
    // copies still in flight (only after a wait ran out)
    if (lane == 0)
        for (int i = consumed; i < issued; ++i) mbar_wait(bar(i % kOwnStages), (i / kOwnStages) & 1, nullptr);
}

}  // namespace

template <class P>
__global__ void __launch_bounds__(kThreads, 1)
    shared_attn_kernel(const __grid_constant__ CUtensorMap tm_q, const __grid_constant__ CUtensorMap tm_k,
                       const __grid_constant__ CUtensorMap tm_v, const __grid_constant__ P p) {
    if (static_cast<int>(blockIdx.x) < p.n_pieces) {
        prefix_cta(tm_q, tm_k, tm_v, p, blockIdx.x);
        return;
    }
    const int warp = threadIdx.x >> 5;
    if (warp >= kSharedWarps) {
        asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" ::"n"(kRegsSmall));
        return;
    }
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" ::"n"(kRegsLarge));
    own_warp(tm_k, tm_v, p, (static_cast<int>(blockIdx.x) - p.n_pieces) * kSharedWarps + warp);
}

// Joins the partials of 32 query rows (a lane a row) of a tile: CTA of units x
// tiles x 4 quarters x 2 ways.  A warp takes 8 columns, so a load of a prefix
// partial is 512 contiguous bytes; `ways` of the warps share the partials of
// their rows, in turn, and add up in shared memory.  (Joined by the CTAs of the
// launch before instead, behind a barrier of all of them in a cooperative launch:
// 24.6 us for 32 rows x 25k against 18.9, for such a launch does not overlap the
// one before it, and 137 CTAs take the 256 tasks in two rounds.  Nor does an early
// start pay: the CTAs then crowd on the SMs that are free first, 21.0 us.)
template <class P>
__global__ void __launch_bounds__(256) shared_join_kernel(const __grid_constant__ P p) {
    __shared__ float2 s_ml[8 * 32];       // [warp][lane]
    __shared__ float4 s_acc[8 * 2 * 32];  // [warp][2][lane]
    const int warp = threadIdx.x >> 5, lane = threadIdx.x & 31;
    const int sub = warp / p.ways, part = warp % p.ways;  // the warp's columns, its share of the partials
    const int cols_of_cta = 8 / p.ways, ctas = 16 / cols_of_cta;  // of 16 column groups
    const int col = (blockIdx.x % ctas) * cols_of_cta + sub;
    int rest = blockIdx.x / ctas;
    const int quarter = rest % 4;
    rest /= 4;
    const int t = rest % p.tiles;
    const SharedUnit u = p.units[rest / p.tiles];
    const int r = quarter * 32 + lane;                // of the tile
    const int q = (u.mu * p.tiles + t) * kTileQ + r;  // query row of the (group, kv-head)
    if (q - lane >= u.n_rows * p.group) return;     // none of the task's rows exists
    const bool valid = q < u.n_rows * p.group;
    const int row = u.row0 + (valid ? q / p.group : 0), h = q % p.group;
    const SharedRow sr = p.rows[row];
    // the pair's own pages, the first and the last warp that had some of them
    const int pages = (sr.own + kPage - 1) / kPage;
    const int page0 = sr.page0 + u.kvh * pages;
    const int w0 = page0 / p.warp_pages, n_own = pages ? (page0 + pages - 1) / p.warp_pages - w0 + 1 : 0;
    const int n = valid ? u.n_pieces + n_own : 0;
    const int n_max = __reduce_max_sync(0xffffffffu, n);
    const int64_t slot0 = static_cast<int64_t>(row) * p.n_kv_heads + u.kvh + w0 - u.n_pieces;
    grid_dep_wait();  // the partials come from the launch before this one

    float M = -INFINITY, L = 0.f;
    float4 acc[2] = {make_float4(0.f, 0.f, 0.f, 0.f), make_float4(0.f, 0.f, 0.f, 0.f)};
    constexpr int kBatch = 6;
    for (int k0 = part; k0 < n_max; k0 += kBatch * p.ways) {
        float2 ml[kBatch];
        float4 o[kBatch][2];
        float mn = M;
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const int k = k0 + b * p.ways;
            ml[b] = make_float2(-INFINITY, 0.f);
            o[b][0] = o[b][1] = make_float4(0.f, 0.f, 0.f, 0.f);
            if (k >= n) continue;
            if (k < u.n_pieces) {
                const int64_t at = static_cast<int64_t>(u.piece0 + k) * p.tiles + t;
                ml[b] = __ldcg(reinterpret_cast<const float2 *>(p.pre_ml) + at * kTileQ + r);
                const float4 *src = reinterpret_cast<const float4 *>(p.pre_o) + (at * (kHeadDim / 4) + 2 * col) * kTileQ + r;
                o[b][0] = __ldcg(src);
                o[b][1] = __ldcg(src + kTileQ);
            } else {
                const int64_t at = (slot0 + k) * p.group + h;
                ml[b] = __ldcg(reinterpret_cast<const float2 *>(p.own_ml) + at);
                const float4 *src = reinterpret_cast<const float4 *>(p.own_o) + at * (kHeadDim / 4) + 2 * col;
                o[b][0] = __ldcg(src);
                o[b][1] = __ldcg(src + 1);
            }
        }
#pragma unroll
        for (int b = 0; b < kBatch; ++b) mn = fmaxf(mn, ml[b].x);
        if (mn == -INFINITY) continue;
        const float sc = M == -INFINITY ? 0.f : ex2(M - mn);
        L *= sc;
#pragma unroll
        for (int c = 0; c < 2; ++c) acc[c] = make_float4(acc[c].x * sc, acc[c].y * sc, acc[c].z * sc, acc[c].w * sc);
#pragma unroll
        for (int b = 0; b < kBatch; ++b) {
            const float f = ml[b].x == -INFINITY ? 0.f : ex2(ml[b].x - mn);
            L += f * ml[b].y;
#pragma unroll
            for (int c = 0; c < 2; ++c)
                acc[c] = make_float4(acc[c].x + f * o[b][c].x, acc[c].y + f * o[b][c].y, acc[c].z + f * o[b][c].z,
                                     acc[c].w + f * o[b][c].w);
        }
        M = mn;
    }
    if (p.ways > 1) {
        s_ml[warp * 32 + lane] = make_float2(M, L);
        s_acc[warp * 64 + lane] = acc[0];
        s_acc[warp * 64 + 32 + lane] = acc[1];
        __syncthreads();
        if (part != 0) return;
        float top = M;
        for (int w = 1; w < p.ways; ++w) top = fmaxf(top, s_ml[(warp + w) * 32 + lane].x);
        const float f0 = M == -INFINITY ? 0.f : ex2(M - top);
        L *= f0;
#pragma unroll
        for (int c = 0; c < 2; ++c)
            acc[c] = make_float4(acc[c].x * f0, acc[c].y * f0, acc[c].z * f0, acc[c].w * f0);
        for (int w = 1; w < p.ways; ++w) {
            const float2 ml = s_ml[(warp + w) * 32 + lane];
            const float f = ml.x == -INFINITY ? 0.f : ex2(ml.x - top);
            L += f * ml.y;
#pragma unroll
            for (int c = 0; c < 2; ++c) {
                const float4 a = s_acc[(warp + w) * 64 + c * 32 + lane];
                acc[c] = make_float4(acc[c].x + f * a.x, acc[c].y + f * a.y, acc[c].z + f * a.z, acc[c].w + f * a.w);
            }
        }
    }
    if (!valid) return;
    const float inv = 1.f / L;
    __nv_bfloat16 *dst = p.out + (static_cast<int64_t>(row) * p.n_q_heads + u.kvh * p.group + h) * kHeadDim + 8 * col;
    *reinterpret_cast<uint4 *>(dst) =
        make_uint4(pack_bf16x2(acc[0].x * inv, acc[0].y * inv), pack_bf16x2(acc[0].z * inv, acc[0].w * inv),
                   pack_bf16x2(acc[1].x * inv, acc[1].y * inv), pack_bf16x2(acc[1].z * inv, acc[1].w * inv));
}
template <class P>
cudaError_t launch_shared(const CUtensorMap &tm_q, const CUtensorMap &tm_k, const CUtensorMap &tm_v, const P &p,
                          int32_t n_ctas, cudaStream_t st) {
    static std::atomic<uint64_t> smem_set{0};
    const cudaError_t e = ensure_smem_limit(shared_attn_kernel<P>, static_cast<int>(kSmemBytes), smem_set);
    if (e != cudaSuccess) return e;
    if (n_ctas <= 0) return cudaSuccess;
    PdlLaunch l(dim3(n_ctas), dim3(kThreads), kSmemBytes, st);
    return cudaLaunchKernelEx(&l.cfg, shared_attn_kernel<P>, tm_q, tm_k, tm_v, p);
}

template <class P>
cudaError_t launch_shared_join(const P &p, cudaStream_t st) {
    if (p.n_units <= 0) return cudaSuccess;
    PdlLaunch l(dim3(p.n_units * p.tiles * 4 * 2 * p.ways), dim3(256), 0, st);
    return cudaLaunchKernelEx(&l.cfg, shared_join_kernel<P>, p);
}

#define PPAS_LAUNCH_SHARED(P)                                                                                    \
    template cudaError_t launch_shared(const CUtensorMap &, const CUtensorMap &, const CUtensorMap &, const P &, \
                                       int32_t, cudaStream_t)
PPAS_LAUNCH_SHARED(SharedParamsSmall);
PPAS_LAUNCH_SHARED(SharedParamsMid);
PPAS_LAUNCH_SHARED(SharedParamsBig);
template cudaError_t launch_shared_join(const SharedParamsSmall &, cudaStream_t);
template cudaError_t launch_shared_join(const SharedParamsMid &, cudaStream_t);
template cudaError_t launch_shared_join(const SharedJoinBig &, cudaStream_t);

}  // namespace ppas
