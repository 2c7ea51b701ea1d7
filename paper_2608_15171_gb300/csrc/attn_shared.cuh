// Structures of the attention over shared prefixes: its plan, the parameters of
// its two launches, and what host code needs of them.
#pragma once

#include <memory>
#include <vector>

#include "ppas_internal.h"

namespace ppas {

constexpr int kSharedMaxRows = 512;     // rows of a launch
constexpr int kSharedMaxGroups = 128;
constexpr int kSharedMaxUnits = 1024;   // (group, kv-head, 128 or 256 query rows) of a launch
constexpr int kSharedMaxPieces = 1280;  // pieces of units: at most units + CTAs
constexpr int kSharedWarps = 8;         // warps of a CTA that work on own keys
constexpr int kSharedMaxPiece = 512;    // KV tiles: see kPrefillMaxPiece

// The pages of own keys lie end to end, row by row, a row's kv-heads one after
// the other, and each warp takes the same number of them.  What it has of one
// (row, kv-head) is a partial; the slot of pair (row, kv-head) and warp is
// row * n_kv_heads + kv-head + warp: along the line one of them grows from partial
// to partial, so slots differ, and those of a pair are consecutive.
struct SharedGroup {
    int32_t row0, n_rows;  // packed rows (the launch's first row is 0)
    int32_t prefix;        // keys of the prefix, a multiple of 16
};
struct SharedRow {
    int32_t own;     // keys past the prefix
    int32_t page0;   // pages of own keys before this row's, over all kv-heads
    int32_t table;   // entry of its block-table row that holds its first own page
};
// one CTA's work on a prefix: query rows [128 tiles mu, ...) of (group, kv-head)
// over KV tiles [kt0, kt1)
struct SharedPiece {
    uint16_t group, kvh, mu, kt0, kt1, pad;
};
// the join's view: query rows [128 tiles mu, ...) of n_rows rows from row0 on
struct SharedUnit {
    int32_t row0;
    uint16_t n_rows, kvh, mu, piece0, n_pieces, pad;
};

// The tables come in three sizes: a launch's parameters are copied by the host and
// read by the device (4 rows: 13.5 us a call with 24 KB of them, 11.5 with 3).
template <int kRows, int kGroups, int kPieces, int kUnits>
struct SharedParamsT {
    static constexpr int kMaxRows = kRows, kMaxGroups = kGroups, kMaxPieces = kPieces, kMaxUnits = kUnits;
    const __nv_bfloat16 *q;        // the launch's first row
    __nv_bfloat16 *out;            // likewise
    const int32_t *block_tables;   // likewise
    int32_t table_stride, num_blocks;
    int32_t n_q_heads, n_kv_heads, group;  // group: q-heads of a kv-head
    int32_t tiles;                 // Q tiles of 128 query rows a piece has room for: 1 or 2
    int32_t n_rows, n_pieces, n_units;
    int32_t own_pages, warp_pages;  // in all, and a warp's
    int32_t ways;                  // warps that share a row's partials in the join: 1, 2, 4 or 8
    float scale_log2;
    int32_t *err;
    float *pre_o;   // [n_pieces, tiles, 32 chunks, 128 rows, 4]
    float *pre_ml;  // [n_pieces, tiles, 128 rows, 2]
    float *own_o;   // [slots, group, 128]
    float *own_ml;  // [slots, group, 2]
    SharedGroup groups[kGroups];
    SharedRow rows[kRows];
    SharedPiece pieces[kPieces];
    SharedUnit units[kUnits];
};
using SharedParamsSmall = SharedParamsT<64, 8, 160, 64>;
using SharedParamsMid = SharedParamsT<256, 32, 256, 256>;
// (no room for the units beside the pieces: the join of these has its own tables)
using SharedParamsBig = SharedParamsT<kSharedMaxRows, kSharedMaxGroups, kSharedMaxPieces, 1>;
using SharedJoinBig = SharedParamsT<kSharedMaxRows, 1, 1, kSharedMaxUnits>;
static_assert(sizeof(SharedParamsBig) + 3 * 128 <= 32764 && sizeof(SharedJoinBig) <= 32764, "kernel parameter space");

// one launch of each kernel
struct SharedLaunch {
    int32_t row0 = 0, n_rows = 0, n_groups = 0;
    int32_t tiles = 1, own_pages = 0, warp_pages = 1, own_ctas = 0, ways = 1;
    std::vector<SharedGroup> groups;
    std::vector<SharedRow> rows;
    std::vector<SharedPiece> pieces;
    std::vector<SharedUnit> units;
    size_t pre_o_bytes = 0, pre_ml_bytes = 0, own_o_bytes = 0, own_ml_bytes = 0;
    size_t total_bytes() const { return pre_o_bytes + pre_ml_bytes + own_o_bytes + own_ml_bytes; }
    int32_t n_ctas() const { return static_cast<int32_t>(pieces.size()) + own_ctas; }
};
struct SharedPlan {
    std::vector<SharedLaunch> launches;
    size_t bytes = 0;  // the largest launch's partials (the launches follow one another)
};
SharedPlan plan_shared(int32_t n_groups, const int32_t *group_rows, const int32_t *prefix_lens,
                       const int32_t *ctx_lens, int32_t n_q_heads, int32_t n_kv_heads, int32_t num_sms);

template <class P>
cudaError_t launch_shared(const CUtensorMap &tm_q, const CUtensorMap &tm_k, const CUtensorMap &tm_v, const P &p,
                          int32_t n_ctas, cudaStream_t st);
template <class P>
cudaError_t launch_shared_join(const P &p, cudaStream_t st);

}  // namespace ppas
