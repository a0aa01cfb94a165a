// Every result of a product's list of matrices is in exactly one of its tiles
// (in a symmetric product: it or its mirror image is), in the order of the launches.
#include <cstdio>
#include <cstdlib>
#include <vector>

#include "fc_tiles.h"

using namespace fc;

static int fails = 0;

static void check(const std::vector<TileShape>& shapes, bool symmetric, const std::vector<int>& kinds) {
    const auto launches = plan_tiles(shapes, symmetric, kinds);
    for (size_t m = 0; m < shapes.size(); ++m) {
        const TileShape& s = shapes[m];
        const int rows = s.rows, cols = symmetric ? s.rows : s.cols;
        std::vector<unsigned char> seen((size_t)rows * cols, 0);
        for (const TileLaunch& l : launches) {
            const int side = TILE_SIDE[l.kind];
            for (const TileAt& t : l.tiles) {
                if (t.mat != (int)m) continue;
                if (t.i * side >= rows || t.j * side >= cols || (symmetric && t.i > t.j)) {
                    std::printf("matrix %zu: tile %d %d of %d is outside\n", m, t.i, t.j, side);
                    ++fails;
                    continue;
                }
                for (int r = t.i * side; r < t.i * side + side && r < rows; ++r)
                    for (int c = t.j * side; c < t.j * side + side && c < cols; ++c) {
                        ++seen[(size_t)r * cols + c];
                        if (symmetric && t.i != t.j) ++seen[(size_t)c * cols + r];
                    }
            }
        }
        size_t bad = 0;
        for (unsigned char v : seen) bad += v != 1;
        if (bad) {
            std::printf("matrix %zu of %d x %d: %zu results not in one tile\n", m, rows, cols, bad);
            ++fails;
        }
    }
    for (const TileLaunch& l : launches)
        if (l.tiles.size() > (size_t)1 << 20 || l.tiles.empty()) ++fails;
}

int main() {
    const std::vector<int> all{TILE_LARGE, TILE_BROAD, TILE_MIDDLE, TILE_SMALL}, fine{TILE_BROAD, TILE_MIDDLE, TILE_SMALL},
        next{TILE_LARGE, TILE_MIDDLE, TILE_SMALL};
    if (!plan_tiles({}, true, all).empty() || !plan_tiles({{0, 0, 1}}, false, next).empty()) ++fails;
    std::srand(3);
    for (int round = 0; round < 60; ++round) {
        std::vector<TileShape> shapes;
        const int n = 1 + std::rand() % (round % 3 ? 4 : 20);
        for (int i = 0; i < n; ++i) {
            const int top = round % 12 ? 700 : 4200;
            shapes.push_back({std::rand() % 7 ? 2 + std::rand() % top : 0, 2 + std::rand() % top, 1 + std::rand() % 70});
        }
        check(shapes, true, round % 2 ? all : fine);
        check(shapes, false, next);
    }
    check({{4096, 4096, 192}}, true, fine);
    // more than three rounds of large tiles: the rest of them cut smaller
    check({{4096, 9216, 64}, {4096, 4096, 64}, {1000, 4096, 16}}, false, next);
    if (plan_tiles({{4096, 9216, 64}, {4096, 4096, 64}, {1000, 4096, 16}}, false, next).size() != 2) ++fails;
    check({{2, 200000, 1}}, false, next);
    std::printf("%s\n", fails ? "failed" : "ok");
    return fails != 0;
}
