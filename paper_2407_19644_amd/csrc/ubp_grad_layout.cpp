// Host side of the weight gradient: which products of rows of G and X it forms, cut into regions for the workgroups.
#include <algorithm>
#include <cstdint>
#include <vector>

#include "ubp_internal.h"

namespace ubp {

namespace {

// A tile before regions are cut: rows r0 .. r0 + 15 of G with up to 16 rows of X (columns of W).
struct Tile {
    int32_t r0;
    int32_t col[16];
    int32_t n; // columns used
};

// Rows of X that a run of tiles needs, ascending; rows of G likewise (numbers of M and above, of windows that reach
// over the bottom edge, included).
void union_of(const std::vector<Tile> &tiles, const int32_t *order, int64_t n, std::vector<int32_t> &g, std::vector<int32_t> &x) {
    g.clear();
    x.clear();
    for (int64_t t = 0; t < n; ++t) {
        const Tile &a = tiles[(size_t)order[t]];
        for (int i = 0; i < kStripe; ++i) g.push_back(a.r0 + i);
        x.insert(x.end(), a.col, a.col + a.n);
    }
    for (auto *v : {&g, &x}) {
        std::sort(v->begin(), v->end());
        v->erase(std::unique(v->begin(), v->end()), v->end());
    }
}

int64_t padded(size_t n) { return ((int64_t)n + 15) / 16 * 16; }

struct Rows {
    int64_t g, x; // LDS rows
    int64_t all() const { return g + x; }
};
struct Column {
    int32_t tile, k, slot; // of a tile, with its LDS row
};
// The lane that takes LDS row `cls` modulo 16, even ones first; and the row of 16 from LDS row g0 on that a lane takes.
size_t lane_of(size_t cls) { return cls % 2 * 8 + cls / 2; }
size_t row_of(size_t lane, int32_t g0) { return (lane % 8 * 2 + lane / 8 + 16 - (size_t)g0 % 16) % 16; }

struct Region {
    int64_t first, n; // run of the tile order
    Rows rows;
};

} // namespace

// Windows of 16 rows start every 17 - bh rows, so that each block lies inside one of them; a block of more than 16 rows is
// cut into runs of 16, each a window.  The columns in which a window keeps weights, 16 at a time, are its tiles.
// Regions: the tiles are halved again and again, by rows or by columns, whichever needs fewer rows of G and X
// afterwards, until there are enough and each fits a workgroup's registers and LDS.
const GradLayout &get_grad_layout(const ubp_packed *p) {
    GradLayout &L = p->grad;
    if (L.built) return L;
    GradLayout out;
    out.built = true;
    const int64_t values = p->nb * p->bh * p->bw;
    if (values >= (int64_t(1) << 31) - 1) { // (places of values are 32-bit numbers)
        L = std::move(out);
        return L;
    }
    out.usable = true;
    const int bh = p->bh, bw = p->bw;
    const int stride = bh <= kStripe ? kStripe + 1 - bh : 1;
    // pieces of blocks by window, in canonical order: rows first, then columns
    struct Piece { int32_t r0, b; };
    std::vector<Piece> pieces;
    {
        int32_t r = 0;
        for (int64_t b = 0; b < p->nb; ++b) {
            while (p->indptr[(size_t)r + 1] <= b) ++r;
            if (bh <= kStripe) {
                pieces.push_back({r / stride * stride, (int32_t)b});
            } else {
                for (int k = 0; k < bh; k += kStripe) pieces.push_back({r + k, (int32_t)b});
            }
        }
    }
    std::vector<int32_t> start((size_t)p->nb);
    {
        int32_t r = 0;
        for (int64_t b = 0; b < p->nb; ++b) {
            while (p->indptr[(size_t)r + 1] <= b) ++r;
            start[(size_t)b] = r;
        }
    }
    std::stable_sort(pieces.begin(), pieces.end(), [](const Piece &a, const Piece &b) { return a.r0 < b.r0; });
    std::vector<Tile> tiles;
    std::vector<int32_t> inv; // of the tiles in this order
    std::vector<int32_t> slot_of((size_t)p->K, -1), cols;
    for (size_t i = 0; i < pieces.size();) {
        size_t j = i;
        cols.clear();
        for (; j < pieces.size() && pieces[j].r0 == pieces[i].r0; ++j)
            for (int q = 0; q < bw; ++q) cols.push_back(p->indices[(size_t)pieces[j].b] + q);
        std::sort(cols.begin(), cols.end());
        cols.erase(std::unique(cols.begin(), cols.end()), cols.end());
        const size_t tile0 = tiles.size();
        for (size_t c = 0; c < cols.size(); ++c) {
            if (c % 16 == 0) tiles.push_back({pieces[i].r0, {0}, 0});
            Tile &t = tiles.back();
            t.col[t.n++] = cols[c];
            slot_of[(size_t)cols[c]] = (int32_t)c;
        }
        inv.resize(tiles.size() * 256, -1);
        for (size_t k = i; k < j; ++k) {
            const int64_t b = pieces[k].b;
            const int32_t first = std::max(start[(size_t)b], pieces[k].r0), last = std::min(start[(size_t)b] + bh, pieces[k].r0 + kStripe);
            for (int q = 0; q < bw; ++q) {
                const int32_t c = slot_of[(size_t)(p->indices[(size_t)b] + q)];
                int32_t *t = &inv[(tile0 + (size_t)(c / 16)) * 256];
                for (int32_t row = first; row < last; ++row) {
                    const int e = row - pieces[k].r0;
                    t[(16 * (e >> 2) + c % 16) * 4 + (e & 3)] = (int32_t)((b * bw + q) * bh + row % bh);
                }
            }
        }
        i = j;
    }
    const int64_t n = (int64_t)tiles.size();
    out.n_tiles = n;
    std::vector<int32_t> order((size_t)n);
    for (int64_t t = 0; t < n; ++t) order[(size_t)t] = (int32_t)t;
    std::vector<Region> done, open;
    std::vector<int32_t> g, x, by_row, by_col;
    auto slots = [&](const int32_t *o, int64_t count) {
        union_of(tiles, o, count, g, x);
        return Rows{padded(g.size()), padded(x.size())};
    };
    if (n) open.push_back({0, n, slots(order.data(), n)});
    auto rows_fit = [](const Rows &r) { return r.g <= kGradLargest.g_slots && r.x <= kGradLargest.x_slots; };
    // (halves that need not be cut again for their rows come first)
    auto cost = [&](const Rows (&h)[2]) {
        return h[0].all() + h[1].all() + (rows_fit(h[0]) ? 0 : int64_t(1) << 40) + (rows_fit(h[1]) ? 0 : int64_t(1) << 40);
    };
    // the workgroups of a split of the tokens are as many as an XCD has CUs, while a wavefront keeps two tiles at least
    const int64_t wanted = std::min<int64_t>(kGradRegions, (n + 2 * kGradWaves - 1) / (2 * kGradWaves));
    while (!open.empty()) {
        // the largest one next
        size_t at = 0;
        for (size_t k = 1; k < open.size(); ++k)
            if (open[k].n > open[at].n) at = k;
        const Region r = open[at];
        const bool fits = r.n <= (int64_t)kGradWaves * kGradLargest.tiles && rows_fit(r.rows);
        if ((fits && (int64_t)(open.size() + done.size()) >= wanted) || r.n == 1) {
            done.push_back(r);
            open.erase(open.begin() + (ptrdiff_t)at);
            continue;
        }
        // halves by rows, and by columns
        int32_t *o = &order[(size_t)r.first];
        by_row.assign(o, o + r.n);
        by_col = by_row;
        std::sort(by_row.begin(), by_row.end(), [&](int32_t a, int32_t b) {
            const Tile &s = tiles[(size_t)a], &t = tiles[(size_t)b];
            return s.r0 != t.r0 ? s.r0 < t.r0 : s.col[0] < t.col[0];
        });
        std::sort(by_col.begin(), by_col.end(), [&](int32_t a, int32_t b) {
            const Tile &s = tiles[(size_t)a], &t = tiles[(size_t)b];
            return s.col[0] != t.col[0] ? s.col[0] < t.col[0] : s.r0 < t.r0;
        });
        const int64_t half = (r.n + 1) / 2;
        const Rows rows[2] = {slots(by_row.data(), half), slots(by_row.data() + half, r.n - half)};
        const Rows cs[2] = {slots(by_col.data(), half), slots(by_col.data() + half, r.n - half)};
        const bool rows_win = cost(rows) <= cost(cs);
        std::copy(rows_win ? by_row.begin() : by_col.begin(), rows_win ? by_row.end() : by_col.end(), o);
        open[at] = {r.first, half, rows_win ? rows[0] : cs[0]};
        open.push_back({r.first + half, r.n - half, rows_win ? rows[1] : cs[1]});
    }
    std::sort(done.begin(), done.end(), [](const Region &a, const Region &b) { return a.first < b.first; });
    out.inv.resize((size_t)n * 256);
    out.ops.resize((size_t)n * 16);
    std::vector<int32_t> slot_x((size_t)p->K, 0);
    std::vector<Column> from;
    for (const Region &r : done) {
        out.max_g = std::max(out.max_g, (int)r.rows.g);
        out.max_x = std::max(out.max_x, (int)r.rows.x);
    }
    out.rows.reserve(done.size() * (size_t)(out.max_g + out.max_x));
    for (const Region &r : done) {
        int32_t *o = &order[(size_t)r.first];
        // tiles of one window side by side
        std::sort(o, o + r.n, [&](int32_t a, int32_t b) {
            const Tile &s = tiles[(size_t)a], &t = tiles[(size_t)b];
            return s.r0 != t.r0 ? s.r0 < t.r0 : s.col[0] < t.col[0];
        });
        union_of(tiles, o, r.n, g, x);
        const size_t first_row = out.rows.size();
        for (int32_t v : g) out.rows.push_back(std::min(v, p->M - 1));
        out.rows.resize(first_row + (size_t)out.max_g, out.rows.back());
        for (size_t k = 0; k < x.size(); ++k) slot_x[(size_t)x[k]] = (int32_t)k;
        out.rows.insert(out.rows.end(), x.begin(), x.end());
        out.rows.resize(first_row + (size_t)(out.max_g + out.max_x), out.rows.back());
        // The columns of a window's tiles are dealt out anew: LDS rows whose numbers agree modulo 16 lie in the same banks, so
        // that a tile takes as few of those as it can, and has what it takes in different halves of its lanes.
        for (int64_t t = 0, after; t < r.n; t = after) {
            const int32_t r0 = tiles[(size_t)o[t]].r0;
            from.clear();
            for (after = t; after < r.n && tiles[(size_t)o[after]].r0 == r0; ++after)
                for (int k = 0; k < tiles[(size_t)o[after]].n; ++k) from.push_back({o[after], k, slot_x[(size_t)tiles[(size_t)o[after]].col[k]]});
            std::stable_sort(from.begin(), from.end(), [](const Column &a, const Column &b) { return a.slot % 16 < b.slot % 16; });
            const int32_t g0 = (int32_t)(std::lower_bound(g.begin(), g.end(), r0) - g.begin());
            const size_t count = (size_t)(after - t);
            for (size_t k = 0; k < count * 16; ++k) {
                const size_t to = (size_t)(r.first + t) + k % count, at = lane_of(k / count);
                const Column &c = from[k < from.size() ? k : k % count];    // (a place that is left over repeats the tile's first)
                out.ops[to * 16 + at] = (uint32_t)(g0 + (int32_t)row_of(at, g0)) | (uint32_t)c.slot << 16;
                for (size_t e = 0; e < 16; ++e) {
                    const size_t row = row_of(e, g0);
                    out.inv[to * 256 + (16 * (e >> 2) + at) * 4 + (e & 3)] =
                        k < from.size() ? inv[(size_t)c.tile * 256 + (16 * (row >> 2) + (size_t)c.k) * 4 + (row & 3)] : -1;
                }
            }
        }
        out.regions.insert(out.regions.end(), {(int32_t)r.first, (int32_t)r.n, (int32_t)r.rows.g, (int32_t)r.rows.x});
        out.max_tiles = std::max(out.max_tiles, (int)((r.n + kGradWaves - 1) / kGradWaves));
    }
    while (out.max_tiles > kGradShapes[out.shape].tiles || out.max_g > kGradShapes[out.shape].g_slots || out.max_x > kGradShapes[out.shape].x_slots)
        ++out.shape; // (the largest holds them)
    out.n_regions = (int)done.size();
    L = std::move(out);
    return L;
}

// As many ranges as take the least time by an estimate in stages (0.8 us each at 4 tiles a wavefront, more at 8): rounds of
// workgroups, each of them its range's stages and about 12 for its lists, its first loads and its sums' way out; and with more
// than one range a launch, worth 5, that reads and writes 1 KB per tile and range, 2000 of them in the time of a stage.
GradRanges grad_ranges(const GradLayout &L, int64_t N, int stage_tokens) {
    const int64_t units = std::max<int64_t>(1, N / kGradUnit);             // (a short unit belongs to the last range)
    const double stages = (double)N / stage_tokens;
    int64_t best_each = units;
    double best = 0.0;
    for (int64_t s = 1; s <= std::min<int64_t>(units, kGradWorkgroups); ++s) {
        const int64_t each = (units + s - 1) / s, ranges = (units + each - 1) / each; // (none of them empty)
        const double rounds = (double)((L.n_regions * ranges + kGradWorkgroups - 1) / kGradWorkgroups);
        const double t = rounds * (stages * (double)each / (double)units + 12.0) + (ranges > 1 ? 5.0 + (double)(ranges * L.n_tiles) / 2000.0 : 0.0);
        if (s == 1 || t < best) {
            best = t;
            best_each = each;
        }
    }
    return {(int)((units + best_each - 1) / best_each), (int)(best_each * kGradUnit)};
}

} // namespace ubp
