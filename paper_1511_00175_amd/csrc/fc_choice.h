// Which tiles the operators' products are cut into, whether k is split, and which products go
// in one launch of their own form: plain host arithmetic.
#pragma once

#include <algorithm>
#include <cstdint>

#include "fc_launches.h"

namespace {

constexpr int STEP = 64;  // of k

enum TileKind { LARGE, BROAD, MIDDLE, SHORT, NARROW, KINDS };

constexpr int CUS = 256;

// In us, measured with 1 to 512 tiles: a step of 64 of k with the compute unit full
// of such tiles (`per` at a time) and alone, and a tile's start and end.
struct KindCost {
    int bm, bn;
    double full, alone, once;
    int per;
    double before = 0;  // of what the kind needs done first
};
constexpr KindCost COST[KINDS] = {{256, 256, 1.7, 1.15, 9.5, 1}, {256, 192, 1.38, 1.0, 8.0, 1}, {128, 128, 0.52, 0.6, 5.0, 2}, {64, 128, 0.55, 0.6, 4.0, 2}, {64, 32, 0.2, 0.3, 4.0, 2}};

struct Choice {
    TileKind kind;
    int splits;      // parts of k, of `steps` of 64 each
    int steps;
    double us;       // estimated
};

constexpr int64_t SPLIT_FLOATS = (int64_t)1 << 27;

// The tiles of an m x n product of `total` steps of k, kinds first to last of `cost` (not
// `skip`), and the parts k is split into, by the least estimated time; m is taken up to
// multiples of 64, so that the choice is one for every list of as many 64s of tokens.
// `most`: floats of partial sums.
inline Choice choose_tiles(const KindCost* cost, int first, int last, int skip, int64_t m, int64_t n, int64_t total, bool may_split, int64_t most) {
    m = fc::ceil_div(m, 64) * 64;
    Choice best{(TileKind)last, 1, (int)total, 0};
    double least = 1e300;
    for (int kind = first; kind <= last; ++kind) {
        if (kind == skip) continue;
        const KindCost& c = cost[kind];
        const int64_t tiles = fc::ceil_div(m, c.bm) * fc::ceil_div(n, c.bn);
        const int fill = (int)std::min<int64_t>(64, CUS * c.per / tiles);  // as many as the chip takes at once
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, fill}) {
            if (s < 1) continue;
            const int64_t steps = fc::ceil_div(total, s), parts = fc::ceil_div(total, steps), blocks = tiles * parts;
            if (s > 1 && (!may_split || steps < 2 || parts * m * n > most)) continue;
            const double at_once = (double)std::min<int64_t>(c.per, fc::ceil_div(blocks, CUS));
            double t = c.before + fc::ceil_div(blocks, CUS * c.per) * (steps * std::max(c.alone, c.full * at_once) + c.once);
            if (parts > 1) t += 5.0 + 8.0 * parts * m * n / 4.5e6;  // partial sums, written and read
            if (t < least) {
                least = t;
                best = {(TileKind)kind, (int)parts, (int)steps, t};
            }
        }
    }
    return best;
}

inline Choice choose(int64_t m, int64_t n, int64_t k, bool few, bool may_split, bool broad, int64_t most = SPLIT_FLOATS) {
    return choose_tiles(COST, few ? SHORT : LARGE, few ? NARROW : MIDDLE, broad ? -1 : BROAD, m, n, fc::ceil_div(k, STEP), may_split, most);
}

// Partial sums that a split product may write: two rounds of the chip's largest tiles.
constexpr int64_t SUMS_LIMIT = (int64_t)1 << 25;

// What choose_tiles may count on for products of up to m x n, and the floats of it that any of
// them writes when k is at most `total` steps: a part has at least two steps, there are at most
// 64, and m is counted as it is.
inline int64_t sums_limit(int64_t m, int64_t n) { return std::min<int64_t>(SUMS_LIMIT, 64 * fc::ceil_div(m, 64) * 64 * n); }
inline int64_t sums_room(int64_t m, int64_t n, int64_t total) {
    const int64_t parts = std::min<int64_t>(64, fc::ceil_div(total, 2));
    return parts > 1 ? std::min(sums_limit(m, n), parts * m * n) : 0;
}

// ---- a weight's gradient from 8-bit activations (fc_ckpt.hip) ----------------------------

// Of a weight's gradient: COST's kinds, 128 x 128 slower alone with both operands across their
// rows, and 64 x 64 in 4 stages.  1003 tokens, 1001 x 520: 40 tiles of 128 x 128 take 21 us, 144
// of the last 9 (the form for few tiles takes that case).
constexpr int TINY = 3;
constexpr KindCost COST_DW[] = {COST[LARGE], COST[BROAD], {128, 128, 0.52, 0.7, 5.0, 2}, {64, 64, 0.25, 0.3, 4.0, 2}};

inline int64_t ckpt_limit(int64_t max_outs, int64_t dim) { return sums_limit(max_outs, dim); }
inline int64_t ckpt_room(int64_t max_tokens, int64_t max_outs, int64_t dim) { return sums_room(max_outs, dim, fc::ceil_div(max_tokens, STEP)); }

inline Choice ckpt_choice(int64_t n, int64_t outs, int64_t dim, int64_t most) {
    return choose_tiles(COST_DW, LARGE, TINY, -1, outs, dim, fc::ceil_div(n, STEP), true, most);
}

// Whether small_kernel takes it, estimated as KindCost's, instead of `c` with the launch that
// brings the operands.
constexpr int CKPT_SMALL = 64, CKPT_GROUPS = 4;
inline bool ckpt_small(const Choice& c, int64_t n, int64_t outs, int64_t dim) {
    const int64_t tiles = fc::ceil_div(outs, CKPT_SMALL) * fc::ceil_div(dim, CKPT_SMALL), rounds = fc::ceil_div(n, CKPT_SMALL * CKPT_GROUPS);
    return fc::ceil_div(tiles, CUS) * (3.6 + 1.4 * rounds) < c.us + 3.0;
}

// ---- products in 4 bits (fc_mxfp.hip) ------------------------------------------------------

constexpr int64_t MXFP_CHUNK = 1 << 18;  // tokens of one launch, and of linear's packed inputs

enum { WIDE4, HALF4, SMALL4, KINDS4 };

// As COST, for steps of 256 of k.
constexpr KindCost COST4[KINDS4] = {{256, 256, 1.78, 1.34, 4.5, 1, 6.0}, {128, 128, 0.56, 0.64, 5.2, 2}, {64, 64, 0.29, 0.38, 4.3, 2}};

inline int64_t mxfp_limit(int64_t max_tokens, int64_t rows) { return sums_limit(std::min(max_tokens, MXFP_CHUNK), rows); }
inline int64_t mxfp_room(int64_t max_tokens, int64_t rows, int64_t dim) { return sums_room(std::min(max_tokens, MXFP_CHUNK), rows, fc::ceil_div(dim, 256)); }

inline Choice mxfp_choice(int64_t n, int64_t rows, int64_t dim, int64_t most) {
    return choose_tiles(COST4, WIDE4, SMALL4, -1, n, rows, fc::ceil_div(dim, 256), true, most);
}

// Whether few_kernel takes a linear's inputs: n tokens take the time of a block's packing for
// each round of blocks, against a launch of its own.  us, taken / not: 4096 x 9216, 3 tokens
// 10.0 / 12.7; 9216 x 9216, 2 tokens 20.0 / 19.5, 4 tokens 22 / 19; 8192 x 2048, 4 tokens 6.4 /
// 8.5, 8 tokens 8.0 / 8.0; 65536 x 2048, 1 token 19.7 / 20, 2 tokens 21.9 / 20; 1001 x 520, 16
// tokens 5.6 / 6.8.
inline bool mxfp_few(int64_t n, int64_t rows, int64_t dim) { return n <= 16 && n * dim <= 32768 && n * dim * fc::ceil_div(rows, 16) <= 9000000; }

// Whether small_kernel does, for up to a block to a compute unit: as long as that takes no more
// than packing in a launch of its own and the tiles, by when the host has saved a launch (3 us).
// In graphs, us, taken / not, fp32: 1003 tokens, 1001 x 520 8.5 / 8.8; 2048, 64 x 64 4.2 / 6.1; 256,
// 4096 x 512 7.8 / 7.4; 256, 1024 x 1024 11.6 / 7.3; two blocks to a unit: 2048, 1001 x 520 15.1 / 11.0.
constexpr int MXFP_SMALL = 64, MXFP_SMALL_DIM = 576;
inline bool mxfp_small(int64_t n, int64_t rows, int64_t dim) { return dim <= MXFP_SMALL_DIM && fc::ceil_div(n, MXFP_SMALL) * fc::ceil_div(rows, MXFP_SMALL) <= CUS; }

}  // namespace
