// Checks the plan of an adapter call against what its kernels index from it, and the
// layout of tiles in shared memory.  Lines of input: "plan copies tile_rows tile_total n", then rows
// and adapter of each sequence: "ok units listed tiles" or what is wrong; "shapes": every rank,
// number of slices and cluster: "ok refused".
#include <cstdio>
#include <iostream>
#include <sstream>
#include <string>

#include "ppas_internal.h"

using namespace ppas;

static std::string check(bool copies, int tile_rows, int tile_total, const std::vector<int> &lens,
                         const std::vector<int> &ids) {
    AdapterPlan plan;
    plan.rows = {1, 2, 3};  // of a call before
    plan.units.resize(2);
    plan.tiles.resize(2);
    plan_adapter(static_cast<int>(lens.size()), lens.data(), ids.data(), copies, tile_rows, tile_total, plan);
    std::vector<int> of, seen;
    for (size_t i = 0; i < lens.size(); ++i) of.insert(of.end(), lens[i], ids[i]);
    seen.assign(of.size(), 0);
    int listed = 0;
    for (const AdapterUnit &u : plan.units) {
        if (u.n < 1 || u.n > (u.adapter < 0 ? 32 : kAUnitRows)) return "rows of a unit";
        if (u.listed && (u.first < 0 || u.first + u.n > static_cast<int>(plan.rows.size()))) return "list";
        for (int k = 0; k < u.n; ++k) {
            const int row = u.listed ? plan.rows[u.first + k] : u.first + k;
            if (row < 0 || row >= static_cast<int>(of.size())) return "row of a unit";
            if (of[row] != u.adapter) return "adapter of a unit";
            ++seen[row];
        }
        listed += u.listed ? 1 : 0;
    }
    for (const AdapterTile &t : plan.tiles) {
        if (t.n < 1 || t.n > kTRows || t.first < 0 || t.first + t.n > static_cast<int>(of.size())) return "rows of a tile";
        for (int k = 0; k < t.n; ++k) {
            if (of[t.first + k] != t.adapter || t.adapter < 0) return "adapter of a tile";
            ++seen[t.first + k];
        }
    }
    for (size_t r = 0; r < of.size(); ++r)
        if (seen[r] != (of[r] >= 0 || copies ? 1 : 0)) return "row " + std::to_string(r) + " done " + std::to_string(seen[r]) + " times";
    return "ok " + std::to_string(plan.units.size()) + " " + std::to_string(listed) + " " + std::to_string(plan.tiles.size());
}

static std::string shapes() {
    int refused = 0;
    for (int slices = 1; slices <= kAMaxSlices; ++slices)
        for (int rank = 8; rank <= kAMaxRank; rank += 8)
            for (int ctas = 1, rows = kTRows; ctas <= kAMaxCluster; rows = rows > 32 ? rows / 2 : (++ctas, kTRows)) {
                AdapterParams p = {};
                p.rank = rank;
                p.n_slices = slices;
                TileShape s;
                if (!tile_shape(p, ctas, &s, rows)) {
                    if (ctas == 1 && (slices < 4 || rank <= 96)) return "refused alone";
                    ++refused;
                    continue;
                }
                const uint32_t block = 1u << s.block_log, y = block / 64 * rows * 128, stage = s.subs * (rows * 128 + s.a_bytes);
                const uint32_t sums = s.wide16 + 4, part = rows * sums * 4, summed = s.own_rows * sums * 4;
                if (s.rank16 < rank || s.rank16 % 16 || s.wide16 < slices * s.rank16 || s.wide16 % 32) return "widths";
                if (s.rows != rows || s.own_rows * ctas < rows || (s.own_rows - 1) * ctas >= rows) return "rows of the sums";
                if (s.tmem < s.wide16 + 2 * static_cast<int>(block) || s.tmem > 512 || (s.tmem & (s.tmem - 1))) return "tmem";
                if (s.stages < 2 || s.stages > kTMaxStages || s.y_stages < 2 || s.y_stages > kTYStages) return "stages";
                if (stage % 1024 || y % 1024 || s.b_bytes % 1024 || s.b_at % 1024 || s.bars_at % 8) return "alignment";
                if (s.x_bytes != static_cast<uint32_t>(rows * 128)) return "x";
                // the products read 128 rows of x's place, whatever they hold
                if (s.subs < 1 || s.stages * stage - (rows * 128 + s.a_bytes) + kTRows * 128 > s.bars_at) return "x past its end";
                if (s.a_bytes != static_cast<uint32_t>(slices * s.rank16 * 128)) return "A";
                if (s.b_bytes != block * ((rank + 63) / 64) * 128) return "B";
                // the rings and the sums end before B, B before the barriers, all of it within the CTA's memory
                if (s.stages * stage > s.b_at || s.y_stages * y > s.b_at) return "ring past its end";
                if (s.bars_at < s.b_at + kTBStages * s.b_bytes || s.smem < s.bars_at + kTBarBytes + 1024) return "end";
                if (s.smem > kTSmem) return "too much";
                if (s.y_free < 0 || s.y_free > s.y_stages) return "free stages";
                if (ctas > 1) {
                    if (s.part_at % 16 || s.summed_at % 16 || s.part_at + part > s.summed_at || s.summed_at + summed > s.b_at)
                        return "sums";
                    if (s.y_free * y > s.part_at) return "a stage that is free too early";
                    if (s.y_stages * y > s.summed_at) return "y over what others read";
                } else if (s.y_free != s.y_stages) return "free stages alone";
            }
    return "ok " + std::to_string(refused);
}

int main() {
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        std::string what;
        in >> what;
        if (what == "shapes") {
            std::puts(shapes().c_str());
            continue;
        }
        int copies, tile_rows, tile_total, n;
        in >> copies >> tile_rows >> tile_total >> n;
        std::vector<int> lens(n), ids(n);
        for (int i = 0; i < n; ++i) in >> lens[i] >> ids[i];
        std::puts(check(copies != 0, tile_rows, tile_total, lens, ids).c_str());
    }
}
