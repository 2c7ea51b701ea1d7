// Host side of the attention over shared prefixes: the plan of its launches,
// argument checks and the C entry points.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <exception>
#include <iterator>
#include <stdexcept>

#include "attn_shared.cuh"

namespace ppas {

namespace {

size_t align256(size_t x) { return (x + 255) & ~static_cast<size_t>(255); }

// Times behind the split of the SMs, in us, fitted on GB300 to the best of splits
// from 6 to 120 SMs for the own keys, 15 batches.  A piece takes 5.5 (ids, first K
// tile, last softmax, writing O) and 1.2 a KV tile, 1.5 with two Q tiles; a warp's
// run of own pages 4.2 and 1.1 a page.  (Alone, a tile takes 0.8 or 1.0 and a page
// 0.75: side by side all of them wait for memory.)
constexpr double kPieceUs = 5.5, kTileUs[2] = {1.2, 1.5}, kRunUs = 4.2, kPageUs = 1.1;

// a single row's prefix of up to this many pages is cheaper as its own keys; a longer
// one would leave the join too many partials
constexpr int32_t kOwnPrefixPages = 256;

// pieces of a prefix at the longest
int32_t least_pieces(int32_t prefix) {
    return (prefix + kSharedMaxPiece * kPrefillKT - 1) / (kSharedMaxPiece * kPrefillKT);
}

}  // namespace

SharedPlan plan_shared(int32_t n_groups, const int32_t *group_rows, const int32_t *prefix_lens,
                       const int32_t *ctx_lens, int32_t n_q_heads, int32_t n_kv_heads, int32_t num_sms) {
    SharedPlan plan;
    const int32_t g = n_q_heads / n_kv_heads;
    struct Part {
        int32_t row0, n_rows, prefix;
    };
    // units of a part, and its pieces at the longest, with `tiles` Q tiles a piece
    auto units_of = [&](const Part &pt, int32_t tiles) {
        return n_kv_heads * ((pt.n_rows * g + kTileQ * tiles - 1) / (kTileQ * tiles));
    };
    auto pieces_of = [&](const Part &pt, int32_t tiles) {
        return units_of(pt, tiles) * least_pieces(pt.prefix);
    };
    // A group of more rows than a launch's tables hold is several parts.  Rows read
    // a short prefix as their own keys, where that takes less of the SMs' time than
    // a piece's fixed latency: 100 groups of 2 rows x 512 (16/2 heads) 25.5 us, in
    // pieces 157.6; 60 of 2 x 320 (8/8) 34.6 and 278.5; the other way, 4 rows x 2048
    // 9.4 us in pieces and 11.0 as own keys, 1 x 8000 9.1 and 11.5, 1 x 25k 11.2 and
    // 17.6, 4 groups of 1 x 25k 23.4 and 26.2.
    auto as_own = [](int32_t n, int32_t prefix) {
        const double pages = prefix / kPage;
        return n == 1 ? pages <= kOwnPrefixPages
                      : n * pages * kPageUs / kSharedWarps < kPieceUs + pages * kTileUs[0] / (kPrefillKT / kPage);
    };
    std::vector<Part> parts;
    for (int32_t i = 0, row = 0; i < n_groups; row += group_rows[i++]) {
        const int32_t tables = kSharedMaxPieces / (n_kv_heads * std::max(1, least_pieces(prefix_lens[i])));
        const int32_t most = std::min<int64_t>(kSharedMaxRows, static_cast<int64_t>(tables) * 2 * kTileQ / g);
        for (int32_t r = 0; r < group_rows[i]; r += most) {
            const int32_t n = std::min(most, group_rows[i] - r);
            parts.push_back({row + r, n, as_own(n, prefix_lens[i]) ? 0 : prefix_lens[i]});
        }
    }
    for (size_t i0 = 0; i0 < parts.size();) {
        SharedLaunch l;
        l.row0 = parts[i0].row0;
        size_t i1 = i0;
        int32_t most = 0, units[2] = {0, 0}, pieces[2] = {0, 0};  // with 1, 2 tiles a piece
        for (; i1 < parts.size(); ++i1) {
            const Part &pt = parts[i1];
            if (i1 > i0 && (l.n_rows + pt.n_rows > kSharedMaxRows || i1 - i0 == kSharedMaxGroups ||
                            units[1] + units_of(pt, 2) > kSharedMaxUnits ||
                            pieces[1] + pieces_of(pt, 2) > kSharedMaxPieces))
                break;
            for (int32_t t = 1; t <= 2; ++t) {
                units[t - 1] += units_of(pt, t);
                pieces[t - 1] += pieces_of(pt, t);
            }
            if (pt.prefix > 0) most = std::max(most, pt.n_rows * g);
            l.n_rows += pt.n_rows;
        }
        // two Q tiles a piece where a group fills more than one (or the tables ask for it)
        l.tiles = most > kTileQ || units[0] > kSharedMaxUnits || pieces[0] > kSharedMaxPieces ? 2 : 1;
        const int32_t per = kTileQ * l.tiles;
        int64_t own_pages = 0, most_pages = 0, tiles = 0;
        for (size_t i = i0; i < i1; ++i) {
            const Part &pt = parts[i];
            for (int32_t r = pt.row0; r < pt.row0 + pt.n_rows; ++r) {
                const int64_t pages = (ctx_lens[r] - pt.prefix + kPage - 1) / kPage;
                own_pages += pages * n_kv_heads;
                most_pages = std::max(most_pages, pages);
            }
            tiles += pt.prefix;
        }
        if (own_pages > (int64_t{1} << 30)) throw std::length_error("own keys");
        // The prefixes' pieces have one length, the shortest that sms SMs hold in
        // one round; the own pages are cut into runs of at least 2 (below that a
        // run's fixed latency is all there is), and at most 128 to a (row, kv-head)
        // (one row's 25k tokens in 521 runs: 18.9 us, most of it the join).
        auto piece_len = [&](int32_t sms) {
            int32_t len = 1, hi = kSharedMaxPiece;
            while (len < hi) {
                const int32_t mid = (len + hi) / 2;
                int64_t k = 0;
                for (size_t i = i0; i < i1; ++i)
                    k += static_cast<int64_t>(((parts[i].prefix + kPrefillKT - 1) / kPrefillKT + mid - 1) / mid) *
                         units_of(parts[i], l.tiles);
                if (k <= sms) hi = mid;
                else len = mid + 1;
            }
            return len;
        };
        auto run_len = [&](int32_t sms) {
            const int64_t warps = sms * static_cast<int64_t>(kSharedWarps);
            return std::max({int64_t{2}, (own_pages + warps - 1) / warps, (most_pages + 127) / 128});
        };
        // the SMs for the own keys with which the slower of the two kinds ends first
        int32_t own_sms = own_pages == 0 ? 0 : num_sms;
        if (own_pages > 0 && tiles > 0 && num_sms > 1) {
            double best = INFINITY;
            for (int32_t k = 1; k < num_sms; k += k < 32 ? 1 : 2) {
                const double t = std::max(kPieceUs + kTileUs[l.tiles - 1] * piece_len(num_sms - k),
                                          kRunUs + kPageUs * static_cast<double>(run_len(k)));
                if (t < best) {
                    best = t;
                    own_sms = k;
                }
            }
        }
        l.own_pages = static_cast<int32_t>(own_pages);
        l.warp_pages = static_cast<int32_t>(run_len(std::max(1, own_sms)));
        l.own_ctas = static_cast<int32_t>((own_pages + static_cast<int64_t>(l.warp_pages) * kSharedWarps - 1) /
                                          (static_cast<int64_t>(l.warp_pages) * kSharedWarps));
        const int32_t len = piece_len(std::max(1, num_sms - own_sms));
        int32_t page0 = 0, most_own = 0, most_pieces = 0;
        for (size_t i = i0; i < i1; ++i) {
            const Part &pt = parts[i];
            const uint16_t gi = static_cast<uint16_t>(i - i0);
            l.groups.push_back({pt.row0 - l.row0, pt.n_rows, pt.prefix});
            for (int32_t r = pt.row0; r < pt.row0 + pt.n_rows; ++r) {
                const int32_t own = ctx_lens[r] - pt.prefix, pages = (own + kPage - 1) / kPage;
                l.rows.push_back({own, page0, pt.prefix / kPage});
                page0 += pages * n_kv_heads;
                most_own = std::max(most_own, pages / l.warp_pages + 2);
            }
            const int32_t kt = (pt.prefix + kPrefillKT - 1) / kPrefillKT, np = (kt + len - 1) / len;
            for (int32_t mu = 0; mu < (pt.n_rows * g + per - 1) / per; ++mu)
                for (int32_t h = 0; h < n_kv_heads; ++h) {
                    l.units.push_back({pt.row0 - l.row0, static_cast<uint16_t>(pt.n_rows), static_cast<uint16_t>(h),
                                       static_cast<uint16_t>(mu),
                                       static_cast<uint16_t>(l.pieces.size()), static_cast<uint16_t>(np), 0});
                    for (int32_t k = 0; k < np; ++k)
                        l.pieces.push_back({gi, static_cast<uint16_t>(h), static_cast<uint16_t>(mu),
                                            static_cast<uint16_t>(static_cast<int64_t>(kt) * k / np),
                                            static_cast<uint16_t>(static_cast<int64_t>(kt) * (k + 1) / np), 0});
                    most_pieces = std::max(most_pieces, np);
                }
        }
        l.n_groups = static_cast<int32_t>(i1 - i0);
        const int32_t partials = most_pieces + most_own;
        l.ways = partials > 32 ? 8 : partials > 16 ? 4 : partials > 8 ? 2 : 1;
        const size_t slots = own_pages == 0 ? 0 : static_cast<size_t>(l.n_rows) * n_kv_heads + l.own_ctas * kSharedWarps;
        l.pre_o_bytes = align256(l.pieces.size() * l.tiles * kTileQ * kHeadDim * sizeof(float));
        l.pre_ml_bytes = align256(l.pieces.size() * l.tiles * kTileQ * 2 * sizeof(float));
        l.own_o_bytes = align256(slots * g * kHeadDim * sizeof(float));
        l.own_ml_bytes = align256(slots * g * 2 * sizeof(float));
        plan.bytes = std::max(plan.bytes, l.total_bytes());
        plan.launches.push_back(std::move(l));
        i0 = i1;
    }
    return plan;
}

namespace {

// The last few plans made on this thread (every layer of an iteration has the
// same lengths), keyed by all that a plan depends on.
struct CachedShared {
    int32_t hq = 0, hk = 0, sms = 0;
    std::vector<int32_t> rows, prefixes, ctx;
    std::shared_ptr<const SharedPlan> plan;
};
constexpr int kCached = 4;
thread_local CachedShared t_shared[kCached];
thread_local int t_shared_next = 0;

std::shared_ptr<const SharedPlan> plan_cached(int32_t n_groups, const int32_t *rows, const int32_t *prefixes,
                                              const int32_t *ctx, int32_t n_rows, int32_t hq, int32_t hk) {
    const int32_t sms = plan_sms();
    for (const CachedShared &e : t_shared)
        if (e.plan && e.hq == hq && e.hk == hk && e.sms == sms &&
            e.rows.size() == static_cast<size_t>(n_groups) && e.ctx.size() == static_cast<size_t>(n_rows) &&
            std::equal(rows, rows + n_groups, e.rows.begin()) &&
            std::equal(prefixes, prefixes + n_groups, e.prefixes.begin()) && std::equal(ctx, ctx + n_rows, e.ctx.begin()))
            return e.plan;
    auto made = std::make_shared<const SharedPlan>(plan_shared(n_groups, rows, prefixes, ctx, hq, hk, sms));
    CachedShared &e = t_shared[t_shared_next];
    t_shared_next = (t_shared_next + 1) % kCached;
    e.plan = nullptr;
    e.hq = hq;
    e.hk = hk;
    e.sms = sms;
    e.rows.assign(rows, rows + n_groups);
    e.prefixes.assign(prefixes, prefixes + n_groups);
    e.ctx.assign(ctx, ctx + n_rows);
    e.plan = made;
    return made;
}

// the lengths alone: PPAS_OK and the number of rows
ppas_status check_lengths(int32_t n_groups, const int32_t *rows, const int32_t *prefixes, const int32_t *ctx,
                          int32_t hq, int32_t hk, int32_t *n_rows) {
    if (n_groups < 0 || hq < 1 || hk < 1 || (n_groups > 0 && (!rows || !prefixes || !ctx))) return PPAS_ERR_INVALID_ARG;
    if (hq % hk != 0) return PPAS_ERR_INVALID_ARG;
    const int32_t g = hq / hk;
    if (g != 1 && g != 2 && g != 4 && g != 8) return PPAS_ERR_UNSUPPORTED;
    if (hq / (g >= 2 ? 2 : 1) > 256) return PPAS_ERR_UNSUPPORTED;
    // every group first: the number of contexts follows from all of them, and a
    // context is read only where that many are there
    int64_t n = 0;
    for (int32_t i = 0; i < n_groups; ++i) {
        if (rows[i] < 1 || prefixes[i] < 0 || prefixes[i] % kPage != 0) return PPAS_ERR_INVALID_ARG;
        n += rows[i];
    }
    if (n > INT32_MAX / 1024) return PPAS_ERR_UNSUPPORTED;
    for (int32_t i = 0, r = 0; i < n_groups; ++i) {
        // a launch's table of pieces
        if (static_cast<int64_t>(hk) * least_pieces(std::min(prefixes[i], 65535 * kPrefillKT)) > kSharedMaxPieces)
            return PPAS_ERR_UNSUPPORTED;
        for (const int32_t end = r + rows[i]; r < end; ++r) {
            if (ctx[r] < 1 || ctx[r] < prefixes[i]) return PPAS_ERR_INVALID_ARG;
            if (ctx[r] > 65535 * kPrefillKT) return PPAS_ERR_UNSUPPORTED;  // 16-bit KV tiles
        }
    }
    *n_rows = static_cast<int32_t>(n);
    return PPAS_OK;
}

bool on16(const void *p) { return (reinterpret_cast<uintptr_t>(p) & 15u) == 0; }

ppas_status run(const void *q, const void *k_cache, const void *v_cache, int32_t num_blocks,
                const int32_t *d_block_tables, int32_t max_blocks_per_seq, const SharedPlan &plan, int32_t n_rows,
                int32_t hq, int32_t hk, float scale, void *out, void *workspace, int32_t *err, cudaStream_t st) {
    CUtensorMap tm_q, tm_k, tm_v;
    const int32_t g = hq / hk;
    if (!encode_kv_map(&tm_k, k_cache, num_blocks, hk) || !encode_kv_map(&tm_v, v_cache, num_blocks, hk))
        return PPAS_ERR_CUDA;
    static thread_local SharedParamsSmall small;
    static thread_local SharedParamsMid mid;  // (these are kept off the stack: up to 24 KB each)
    static thread_local SharedParamsBig big;
    static thread_local SharedJoinBig big_join;
    for (const SharedLaunch &l : plan.launches) {
        const __nv_bfloat16 *const q0 = static_cast<const __nv_bfloat16 *>(q) + static_cast<int64_t>(l.row0) * hq * kHeadDim;
        if (!encode_q_group_map(&tm_q, q0, std::min(l.n_rows, n_rows - l.row0), hq, g)) return PPAS_ERR_CUDA;
        uint8_t *const ws = static_cast<uint8_t *>(workspace);
        auto fill = [&](auto &p) {
            p.q = q0;
            p.out = static_cast<__nv_bfloat16 *>(out) + static_cast<int64_t>(l.row0) * hq * kHeadDim;
            p.block_tables = d_block_tables + static_cast<int64_t>(l.row0) * max_blocks_per_seq;
            p.table_stride = max_blocks_per_seq;
            p.num_blocks = num_blocks;
            p.n_q_heads = hq;
            p.n_kv_heads = hk;
            p.group = g;
            p.tiles = l.tiles;
            p.n_rows = l.n_rows;
            p.n_pieces = static_cast<int32_t>(l.pieces.size());
            p.n_units = static_cast<int32_t>(l.units.size());
            p.own_pages = l.own_pages;
            p.warp_pages = l.warp_pages;
            p.ways = l.ways;
            p.scale_log2 = scale * 1.4426950408889634f;
            p.err = err;
            p.pre_o = reinterpret_cast<float *>(ws);
            p.pre_ml = p.pre_o + l.pre_o_bytes / sizeof(float);
            p.own_o = p.pre_ml + l.pre_ml_bytes / sizeof(float);
            p.own_ml = p.own_o + l.own_o_bytes / sizeof(float);
            if (l.groups.size() <= std::size(p.groups)) std::copy(l.groups.begin(), l.groups.end(), p.groups);
            std::copy(l.rows.begin(), l.rows.end(), p.rows);
            if (l.pieces.size() <= std::size(p.pieces)) std::copy(l.pieces.begin(), l.pieces.end(), p.pieces);
            if (l.units.size() <= std::size(p.units)) std::copy(l.units.begin(), l.units.end(), p.units);
        };
        auto fits = [&](const auto &p) {
            return l.rows.size() <= std::size(p.rows) && l.groups.size() <= std::size(p.groups) &&
                   l.pieces.size() <= std::size(p.pieces) && l.units.size() <= std::size(p.units);
        };
        auto launch = [&](auto &p, auto &join) {
            const cudaError_t e = launch_shared(tm_q, tm_k, tm_v, p, l.n_ctas(), st);
            return e == cudaSuccess ? launch_shared_join(join, st) : e;
        };
        cudaError_t e;
        if (fits(small)) {
            fill(small);
            e = launch(small, small);
        } else if (fits(mid)) {
            fill(mid);
            e = launch(mid, mid);
        } else {
            fill(big);
            fill(big_join);
            e = launch(big, big_join);
        }
        if (e != cudaSuccess) return PPAS_ERR_CUDA;
    }
    return PPAS_OK;
}

}  // namespace

}  // namespace ppas

using namespace ppas;

extern "C" size_t ppas_shared_attention_workspace_size(int32_t n_groups, const int32_t *h_group_rows,
                                                       const int32_t *h_prefix_lens, const int32_t *h_ctx_lens,
                                                       int32_t n_q_heads, int32_t n_kv_heads) {
    int32_t n_rows = 0;
    if (check_lengths(n_groups, h_group_rows, h_prefix_lens, h_ctx_lens, n_q_heads, n_kv_heads, &n_rows) != PPAS_OK ||
        n_groups == 0)
        return 0;
    try {
        return plan_cached(n_groups, h_group_rows, h_prefix_lens, h_ctx_lens, n_rows, n_q_heads, n_kv_heads)->bytes;
    } catch (const std::exception &) {
        return 0;
    }
}

extern "C" ppas_status ppas_shared_attention_step(const void *q, const void *k_cache, const void *v_cache,
                                                  int32_t num_blocks, const int32_t *d_block_tables,
                                                  int32_t max_blocks_per_seq, int32_t n_groups,
                                                  const int32_t *h_group_rows, const int32_t *h_prefix_lens,
                                                  const int32_t *h_ctx_lens, int32_t n_q_heads, int32_t n_kv_heads,
                                                  int32_t head_dim, float scale, void *out, void *workspace,
                                                  size_t workspace_bytes, int32_t *d_err_flag, void *stream) {
    int32_t n_rows = 0;
    if (head_dim < 1) return PPAS_ERR_INVALID_ARG;
    if (head_dim != kHeadDim) return PPAS_ERR_UNSUPPORTED;
    const ppas_status st =
        check_lengths(n_groups, h_group_rows, h_prefix_lens, h_ctx_lens, n_q_heads, n_kv_heads, &n_rows);
    if (st != PPAS_OK || n_groups == 0) return st;
    if (!q || !k_cache || !v_cache || !d_block_tables || !out || num_blocks < 1 || max_blocks_per_seq < 1)
        return PPAS_ERR_INVALID_ARG;
    if (!on16(q) || !on16(k_cache) || !on16(v_cache) || !on16(out) || !(scale > 0.f) || !std::isfinite(scale))
        return PPAS_ERR_INVALID_ARG;
    for (int32_t r = 0; r < n_rows; ++r)
        if (h_ctx_lens[r] > static_cast<int64_t>(max_blocks_per_seq) * kPage) return PPAS_ERR_INVALID_ARG;
    if (static_cast<int64_t>(n_rows) * n_q_heads > INT32_MAX ||
        static_cast<int64_t>(num_blocks) * n_kv_heads * kPage > INT32_MAX)
        return PPAS_ERR_UNSUPPORTED;
    try {
        const auto plan = plan_cached(n_groups, h_group_rows, h_prefix_lens, h_ctx_lens, n_rows, n_q_heads, n_kv_heads);
        if (plan->bytes > 0 && (!workspace || workspace_bytes < plan->bytes)) return PPAS_ERR_CAPACITY;
        if ((reinterpret_cast<uintptr_t>(workspace) & 255u) != 0) return PPAS_ERR_INVALID_ARG;
        return run(q, k_cache, v_cache, num_blocks, d_block_tables, max_blocks_per_seq, *plan, n_rows, n_q_heads,
                   n_kv_heads, scale, out, workspace, d_err_flag, static_cast<cudaStream_t>(stream));
    } catch (const std::exception &) {
        return PPAS_ERR_CAPACITY;  // host memory
    }
}
