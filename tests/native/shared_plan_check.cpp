// Checks the plan of the attention over shared prefixes against what its
// kernels index from it.  A line of input: sms hq hk n_groups, then rows and
// prefix of each group, then the contexts; a line of output each: "ok launches
// pieces own_pages own_ctas tiles ways longest_piece warp_pages bytes" (of the first launch) or what is wrong.
#include <cstdio>
#include <iostream>
#include <set>
#include <sstream>
#include <string>

#include "attn_shared.cuh"

using namespace ppas;

static std::string check(int sms, int hq, int hk, const std::vector<int> &rows, const std::vector<int> &pre,
                         const std::vector<int> &ctx) {
    const int g = hq / hk;
    const SharedPlan plan = plan_shared(static_cast<int>(rows.size()), rows.data(), pre.data(), ctx.data(), hq, hk, sms);
    std::vector<int> prefix_of;
    for (size_t i = 0; i < rows.size(); ++i) prefix_of.insert(prefix_of.end(), rows[i], pre[i]);
    int row = 0;
    size_t bytes = 0;
    for (const SharedLaunch &l : plan.launches) {
        if (l.row0 != row) return "rows of launches";
        if (l.rows.size() > kSharedMaxRows || static_cast<int>(l.rows.size()) != l.n_rows) return "rows table";
        if (l.groups.size() > kSharedMaxGroups || l.groups.empty()) return "groups table";
        if (l.units.size() > kSharedMaxUnits) return "units table";
        if (l.pieces.size() > kSharedMaxPieces) return "pieces table";
        if (l.tiles != 1 && l.tiles != 2) return "tiles";
        if (l.warp_pages < 1) return "pages of a warp";
        if (l.ways != 1 && l.ways != 2 && l.ways != 4 && l.ways != 8) return "ways";
        int r = 0, page = 0;
        for (size_t gi = 0; gi < l.groups.size(); ++gi) {
            const SharedGroup &gr = l.groups[gi];
            if (gr.row0 != r || gr.n_rows < 1 || gr.prefix % 16) return "group";
            for (int k = 0; k < gr.n_rows; ++k, ++r) {
                const SharedRow &sr = l.rows[r];
                if (gr.prefix != prefix_of[row + r] && !(gr.prefix == 0 && (gr.n_rows == 1 || prefix_of[row + r] < 1024))) return "prefix of a row";
                if (sr.own != ctx[row + r] - gr.prefix || sr.own < 0) return "own keys";
                if (sr.table != gr.prefix / 16 || sr.page0 != page) return "first page";
                page += (sr.own + 15) / 16 * hk;
            }
        }
        if (r != l.n_rows || page != l.own_pages) return "pages";
        // every warp's slots, as the kernel numbers them: different, and inside the workspace
        const int64_t warps = static_cast<int64_t>(l.own_ctas) * kSharedWarps;
        if (warps * l.warp_pages < l.own_pages) return "warps cover the pages";
        if (l.own_ctas > 0 && static_cast<int64_t>(l.own_ctas - 1) * kSharedWarps * l.warp_pages >= l.own_pages) return "a CTA without pages";
        int64_t last_slot = -1;
        for (int q = 0; q < l.n_rows; ++q) {
            const int pages = (l.rows[q].own + 15) / 16;
            for (int h = 0; h < hk && pages; ++h) {
                const int64_t p0 = l.rows[q].page0 + static_cast<int64_t>(h) * pages;
                const int64_t w0 = p0 / l.warp_pages, w1 = (p0 + pages - 1) / l.warp_pages;
                for (int64_t w = w0; w <= w1; ++w) {
                    const int64_t slot = static_cast<int64_t>(q) * hk + h + w;
                    if (slot <= last_slot || w >= warps) return "slots";
                    last_slot = slot;
                }
            }
        }
        if (l.own_o_bytes < static_cast<size_t>(last_slot + 1) * g * 512 || l.own_ml_bytes < static_cast<size_t>(last_slot + 1) * g * 8)
            return "workspace of own keys";
        std::set<std::vector<int>> seen;
        size_t next = 0;
        for (const SharedUnit &u : l.units) {
            size_t gi = 0;
            while (gi < l.groups.size() && l.groups[gi].row0 != u.row0) ++gi;
            const SharedGroup &gr = l.groups.at(gi);
            if (u.n_rows != gr.n_rows) return "rows of a unit";
            if (u.kvh >= hk || u.mu * l.tiles * 128 >= gr.n_rows * g) return "unit";
            if (!seen.insert({u.row0, u.kvh, u.mu}).second) return "a unit twice";
            if (u.n_pieces > 0 && u.piece0 != next) return "first piece";
            const int kt = (gr.prefix + 127) / 128;
            int at = 0;
            for (int k = 0; k < u.n_pieces; ++k) {
                const SharedPiece &pc = l.pieces.at(next++);
                if (pc.group != gi || pc.kvh != u.kvh || pc.mu != u.mu) return "piece of another unit";
                if (pc.kt0 != at || pc.kt1 <= pc.kt0 || pc.kt1 - pc.kt0 > kSharedMaxPiece) return "piece's tiles";
                at = pc.kt1;
            }
            if (at != kt) return "pieces cover the prefix";
        }
        if (next != l.pieces.size()) return "pieces without a unit";
        size_t want = 0;
        for (const SharedGroup &gr : l.groups) want += hk * ((gr.n_rows * g + 128 * l.tiles - 1) / (128 * l.tiles));
        if (want != l.units.size()) return "units";
        if (l.pre_o_bytes < l.pieces.size() * l.tiles * 128 * 128 * 4 || l.pre_ml_bytes < l.pieces.size() * l.tiles * 1024)
            return "workspace";
        if (l.pre_o_bytes % 256 || l.pre_ml_bytes % 256 || l.own_o_bytes % 256 || l.own_ml_bytes % 256) return "alignment";
        bytes = std::max(bytes, l.total_bytes());
        row += l.n_rows;
    }
    if (row != static_cast<int>(ctx.size()) || bytes != plan.bytes) return "rows, bytes";
    const SharedLaunch &l = plan.launches.front();
    int longest = 0;
    for (const SharedPiece &pc : l.pieces) longest = std::max(longest, pc.kt1 - pc.kt0);
    std::ostringstream s;
    s << "ok " << plan.launches.size() << " " << l.pieces.size() << " " << l.own_pages << " " << l.own_ctas << " " << l.tiles
      << " " << l.ways << " " << longest << " " << l.warp_pages << " " << plan.bytes;
    return s.str();
}

int main() {
    std::string line;
    while (std::getline(std::cin, line)) {
        std::istringstream in(line);
        int sms, hq, hk, n;
        in >> sms >> hq >> hk >> n;
        std::vector<int> rows(n), pre(n), ctx;
        for (int i = 0; i < n; ++i) in >> rows[i] >> pre[i];
        for (int c; in >> c;) ctx.push_back(c);
        std::puts(check(sms, hq, hk, rows, pre, ctx).c_str());
    }
}
