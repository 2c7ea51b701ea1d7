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
constexpr int kSharedMaxItemPages = 32; // pages of an item of own keys: one id a lane
constexpr int kSharedWarps = 8;         // warps of a CTA that work on own keys, each on its own items
constexpr int kSharedMaxPiece = 512;    // KV tiles: see kPrefillMaxPiece

struct SharedGroup {
    int32_t row0, n_rows;  // packed rows (the launch's first row is 0)
    int32_t prefix;        // keys of the prefix, a multiple of 16
};
struct SharedRow {
    int32_t own;        // keys past the prefix
    int32_t item0;      // first item of own keys, over all kv-heads
    uint16_t n_items;   // items a kv-head
    uint16_t group;
};
// one CTA's work on a prefix: query rows [128 tiles mu, ...) of (group, kv-head)
// over KV tiles [kt0, kt1)
struct SharedPiece {
    uint16_t group, kvh, mu, kt0, kt1, pad;
};
struct SharedUnit {
    uint16_t group, kvh, mu, piece0, n_pieces, pad;
};

struct SharedParams {
    const __nv_bfloat16 *q;        // the launch's first row
    const int32_t *block_tables;   // likewise
    int32_t table_stride, num_blocks;
    int32_t n_q_heads, n_kv_heads, group;  // group: q-heads of a kv-head
    int32_t tiles;                 // Q tiles of 128 query rows a piece has room for: 1 or 2
    int32_t n_rows, n_pieces, n_items, item_pages, own_warps;
    float scale_log2;
    int32_t *err;
    float *pre_o;   // [n_pieces, tiles, 32 chunks, 128 rows, 4]
    float *pre_ml;  // [n_pieces, tiles, 128 rows, 2]
    float *own_o;   // [n_items, group, 128]
    float *own_ml;  // [n_items, group, 2]
    SharedGroup groups[kSharedMaxGroups];
    SharedRow rows[kSharedMaxRows];
    SharedPiece pieces[kSharedMaxPieces];
};
static_assert(sizeof(SharedParams) + 3 * 128 <= 32764, "kernel parameter space");

struct SharedMergeParams {
    __nv_bfloat16 *out;  // the launch's first row
    const float *pre_o, *pre_ml, *own_o, *own_ml;
    int32_t n_q_heads, group, tiles, n_units;
    int32_t ways;        // warps that share a row's partials: 1, 2, 4 or 8
    SharedGroup groups[kSharedMaxGroups];
    SharedRow rows[kSharedMaxRows];
    SharedUnit units[kSharedMaxUnits];
};
static_assert(sizeof(SharedMergeParams) <= 32764, "kernel parameter space");

// one launch of each kernel
struct SharedLaunch {
    int32_t row0 = 0, n_rows = 0, n_groups = 0;
    int32_t tiles = 1, item_pages = 1, n_items = 0, own_ctas = 0, ways = 1;
    std::vector<SharedGroup> groups;
    std::vector<SharedRow> rows;
    std::vector<SharedPiece> pieces;
    std::vector<SharedUnit> units;
    size_t pre_o_bytes = 0, pre_ml_bytes = 0, own_o_bytes = 0, own_ml_bytes = 0;
    size_t total_bytes() const { return pre_o_bytes + pre_ml_bytes + own_o_bytes + own_ml_bytes; }
};
struct SharedPlan {
    std::vector<SharedLaunch> launches;
    size_t bytes = 0;  // the largest launch's partials (the launches follow one another)
};
SharedPlan plan_shared(int32_t n_groups, const int32_t *group_rows, const int32_t *prefix_lens,
                       const int32_t *ctx_lens, int32_t n_q_heads, int32_t n_kv_heads, int32_t num_sms);

cudaError_t launch_shared(const CUtensorMap &tm_q, const CUtensorMap &tm_k, const CUtensorMap &tm_v,
                          const SharedParams &p, int32_t own_ctas, cudaStream_t st);
cudaError_t launch_shared_merge(const SharedMergeParams &p, cudaStream_t st);

}  // namespace ppas
