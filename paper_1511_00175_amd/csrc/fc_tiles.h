// Which tiles a product over a list of matrices is cut into, and in which order
// its blocks take them: plain host arithmetic, run when a plan is made.
//
// A compute unit multiplies fastest on the largest tiles, but a chip of 256 of
// them works in rounds, and a last round of a few large tiles takes as long as a
// full one.  So every tile size is tried, for all tiles or for as many as fill
// whole rounds, with the rest cut smaller in a launch of its own, and the estimate
// that is least is taken.  In AlexNet's update (8 matrices) B's products went from 244
// us to 170 by that, and X's from 555 to 510; with 192 x 192 tiles 4096 x 4096's A and
// B (3 parts) from 330 and 346 us to 225 and 243.
#pragma once

#include <algorithm>
#include <cmath>
#include <cstdint>
#include <functional>
#include <queue>
#include <vector>

namespace fc {

struct TileAt {
    int mat, i, j;           // mat < 0: no tile
};

enum TileKind { TILE_LARGE, TILE_BROAD, TILE_MIDDLE, TILE_SMALL, TILE_KINDS };
constexpr int TILE_SIDE[TILE_KINDS] = {256, 192, 128, 64};
constexpr int TILE_CUS = 256, TILE_XCDS = 8;

// What a tile costs, in us: per step of 64 of k with the compute unit full of such
// tiles (`per` at a time), per step with one alone, and besides (start, epilogue).
// Measured on fp16 operands with 1 to 512 tiles of 1, 16 and 64 steps.
struct TileCost {
    double full, alone, once;
    int per;
};
constexpr TileCost TILE_COST[TILE_KINDS] = {{1.7, 1.15, 9.5, 1}, {1.1, 0.8, 7.0, 1}, {0.52, 0.6, 5.0, 2}, {0.2, 0.28, 4.0, 2}};
constexpr double LAUNCH_COST = 4.0;

// One matrix's product: rows x cols of results (symmetric: rows x rows, tiles
// on and above the diagonal), `steps` of 64 of k.
struct TileShape {
    int rows, cols, steps;   // rows 0: none
};

struct TileLaunch {
    int kind = TILE_SMALL;
    std::vector<TileAt> tiles;
};

inline int64_t tile_count(const TileShape& m, bool symmetric, int side) {
    const int64_t r = (m.rows + side - 1) / side, c = (m.cols + side - 1) / side;
    return symmetric ? r * (r + 1) / 2 : r * c;
}

// A matrix's tiles in groups of 8 tile rows, down the rows first.
inline void tile_matrix(const TileShape& m, bool symmetric, int side, int mat, std::vector<TileAt>& to) {
    const int s = (m.rows + side - 1) / side, l = symmetric ? s : (m.cols + side - 1) / side;
    for (int g = 0; g < s; g += 8)
        for (int c = 0; c < l; ++c)
            for (int r = g; r < std::min(g + 8, s); ++r)
                if (!symmetric || r <= c) to.push_back({mat, r, c});
}

// Estimated time of tiles, those of most steps first: each goes to the compute
// unit that is free first.
inline double tile_time(const std::vector<TileAt>& tiles, const std::vector<TileShape>& shapes, int kind) {
    const TileCost& c = TILE_COST[kind];
    std::priority_queue<double, std::vector<double>, std::greater<double>> free;
    for (int i = 0; i < TILE_CUS; ++i) free.push(0);
    double end = 0;
    for (const TileAt& t : tiles) {
        const int n = shapes[t.mat].steps;
        const double at = free.top() + n * c.full + c.once / c.per;
        free.pop();
        free.push(at);
        end = std::max({end, at, n * c.alone + c.once});
    }
    return end;
}

// The same tiles in the order of a launch: blocks go to the XCDs in turn, so each
// XCD has a list of its own, of neighbouring tiles, which share its L2, and of as
// much work as the others', matrix by matrix.
inline std::vector<TileAt> tile_order(const std::vector<TileAt>& tiles, const std::vector<TileShape>& shapes) {
    std::vector<TileAt> list[TILE_XCDS], order;
    int64_t load[TILE_XCDS] = {};
    for (size_t at = 0; at < tiles.size();) {
        size_t end = at;
        while (end < tiles.size() && tiles[end].mat == tiles[at].mat) ++end;
        const size_t share = (end - at + TILE_XCDS - 1) / TILE_XCDS;
        for (; at < end;) {
            const int x = (int)(std::min_element(load, load + TILE_XCDS) - load);
            const size_t to = std::min(at + share, end);
            list[x].insert(list[x].end(), tiles.begin() + at, tiles.begin() + to);
            load[x] += (int64_t)(to - at) * shapes[tiles[at].mat].steps;
            at = to;
        }
    }
    size_t longest = 0;
    for (const auto& v : list) longest = std::max(longest, v.size());
    for (size_t k = 0; k < longest; ++k)
        for (const auto& v : list) order.push_back(k < v.size() ? v[k] : TileAt{-1, 0, 0});
    return order;
}

// The launches of one product; `kinds`: the tile sizes it may use, the largest first.
inline std::vector<TileLaunch> plan_tiles(const std::vector<TileShape>& shapes, bool symmetric, const std::vector<int>& kinds) {
    std::vector<int> by_steps;
    for (int i = 0; i < (int)shapes.size(); ++i)
        if (shapes[i].rows > 0) by_steps.push_back(i);
    std::stable_sort(by_steps.begin(), by_steps.end(), [&](int i, int j) { return shapes[i].steps > shapes[j].steps; });
    double least = HUGE_VAL;
    std::vector<TileLaunch> best;
    auto consider = [&](double time, std::vector<TileLaunch> launches) {
        if (time >= least) return;
        least = time;
        best = std::move(launches);
    };
    for (int k : kinds) {
        int64_t count = 0;
        for (int i : by_steps) count += tile_count(shapes[i], symmetric, TILE_SIDE[k]);
        if (count == 0) return {};
        if (count > 1 << 18 && k != kinds.front()) continue;  // more than large tiles leave a choice for
        std::vector<TileAt> all;
        for (int i : by_steps) tile_matrix(shapes[i], symmetric, TILE_SIDE[k], i, all);
        consider(tile_time(all, shapes, k), {{k, all}});
        const size_t round = TILE_CUS * TILE_COST[k].per, whole = all.size() / round * round;
        if (whole == 0 || whole == all.size()) continue;
        const std::vector<TileAt> main(all.begin(), all.begin() + whole);
        const double time = tile_time(main, shapes, k) + LAUNCH_COST;
        for (int k2 : kinds) {
            if (TILE_SIDE[k2] >= TILE_SIDE[k] || TILE_SIDE[k] % TILE_SIDE[k2]) continue;
            const int f = TILE_SIDE[k] / TILE_SIDE[k2];
            std::vector<TileAt> rest;
            for (size_t q = whole; q < all.size(); ++q) {
                const TileAt& t = all[q];
                const TileShape& m = shapes[t.mat];
                for (int c = t.j * f; c < t.j * f + f; ++c)
                    for (int r = t.i * f; r < t.i * f + f; ++r)
                        if (r * TILE_SIDE[k2] < m.rows && c * TILE_SIDE[k2] < (symmetric ? m.rows : m.cols) && (!symmetric || r <= c))
                            rest.push_back({t.mat, r, c});
            }
            consider(time + tile_time(rest, shapes, k2), {{k, main}, {k2, rest}});
        }
    }
    for (TileLaunch& l : best) l.tiles = tile_order(l.tiles, shapes);
    return best;
}

}  // namespace fc
