// Momentum updates made orthogonal by Newton-Schulz products (fc_lm.h).
//
//   X = D / |D|_F (rows <= columns; a taller matrix is transposed)
//   repeat: A = X X^T, B = b A + c A A, X <- a X + B X
//
// for every matrix of a flat vector at once: each of a step's three products is
// one launch over the tiles of all matrices, or two of tiles of two sizes; small
// matrices take all their steps in one block of one launch beside them.  A step
// is s^2 l + s^3 + 2 s^2 l
// operations for s x l (A and B are symmetric: only tiles on and above the
// diagonal are computed, the others are their mirror image); the bytes are
// small beside them, so the products are bound by the matrix cores where the
// matrices fill the chip and by their longest k loop where they do not: 5 matrices of
// 75 x 8073 with 3 parts take 0.66 ms, A's products most of it, each tile alone with 381
// steps of 64 of k (plain fp32 products 0.54).
//
// Measured, 5 steps: all of AlexNet's layers, fp32 to bf16, 4.1 TFLOP in 4.5 ms (0.91
// PFLOP/s); 4096 x 4096 with 3 parts, fp32, 4.1 TFLOP in 4.0 ms (1.02); GoogLeNet's 58
// matrices 0.29 ms in 17 launches, 0.04 TFLOP, bound by each launch's longest tile;
// 96 x 363 in one block 58 us (93 in 17 launches), bound by latency.
//
// Numbers.  Everything is fp16 times a power of two that puts the largest
// possible value (known from the polynomial) below 2^15, so that small entries
// keep all their bits; sums are fp32.  X is kept as a sum of two fp16 numbers,
// high and low (22 bits).  With `parts` 1 the products read the high halves
// alone: the relative error of a step is that of one rounding to 11 bits, but
// only along directions X already has -- a X, which carries X's weak directions
// (a rounding there would be noise of full rank, grown by 3.4 a step), is formed
// from both halves.  With 3 parts every operand is such a sum and a product is
// high * high + high * low + low * high: fp32's accuracy for 3 times the work.
// Sums are taken in runs of 512 of k, but for tiles of 256 x 256: X's of 3 parts
// are one chain of 3 s terms there (fp32 results, error relative to the norm, in
// 256 x 256 tiles / in 128 x 128 with runs / plain fp32: 4096 x 4096 1.6e-6 / 5.7e-7 /
// 4.4e-6, 2048 x 8192 1.2e-6 / 5.9e-7 / 3.1e-6; the time 3.91 / 4.35 ms and 2.49 /
// 2.68).  A matrix of at most 32 rows or
// columns always has 3 parts: roundings average out over few terms only (with one
// part the products' error was 1.0 times a bf16 result's own at 16 x 20, 0.7 at
// 64 x 64, 0.4 at 512 x 512), and its launches are too short for the work to matter.
#include <algorithm>
#include <cmath>
#include <cstring>
#include <type_traits>
#include <vector>

#include "fc_gemm.h"
#include "fc_lm_host.h"
#include "fc_tiles.h"

using fc::f16x4;
using fc::f32x4;
using fc::f32x4_any;
using fc::Operand;
using Tile = fc::TileAt;

namespace {

typedef _Float16 f16;
typedef __bf16 bf16;

extern __shared__ __align__(1024) char lds[];

constexpr int PIECES = 1024;  // of a matrix's sum of squares, at most

struct Matrix {
    uint64_t offset;         // in the flat vectors
    int rows, cols;
    int s, l;                // of X: the shorter and the longer side
    int sp, lp;              // row strides: s, l up to multiples of 64
    int turned;              // X is the matrix transposed
    int parts;
    float lr_mult, decay_mult, scale;
    f16* x[2];               // [s][lp], low halves x_lo behind
    f16* a;                  // [s][sp], low halves a_lo behind
    f16* b;
    int64_t x_lo, a_lo;
    int piece0, pieces;      // of the sum of squares
    int64_t piece_len;
};

// Where results go: to out, or into the weights w.
struct Output {
    void* out;
    int dt;
    float* w;
    float lr, wd;
};

__device__ __forceinline__ void store_one(const Output& a, const Matrix& m, uint64_t at, float u) {
    if (!a.out) {
        const float w = a.w[at];
        a.w[at] = w - a.lr * m.lr_mult * (m.scale * u + a.wd * m.decay_mult * w);
    } else if (a.dt == FC_F32) {
        static_cast<float*>(a.out)[at] = u;
    } else if (a.dt == FC_F16) {
        static_cast<f16*>(a.out)[at] = (f16)u;
    } else {
        static_cast<bf16*>(a.out)[at] = (bf16)u;
    }
}

// Four neighbours of a row of the result, of which those in the matrix are
// stored: as one vector, which may start at any element (a row's last few one by one).
__device__ __forceinline__ void store_out(const Output& a, const Matrix& m, int row, int col, f32x4 u) {
    if (col >= m.cols) return;
    const uint64_t at = m.offset + (uint64_t)row * m.cols + col;
    if (col + 4 > m.cols) {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (col + e < m.cols) store_one(a, m, at + e, u[e]);
    } else if (!a.out) {
        f32x4_any* p = reinterpret_cast<f32x4_any*>(a.w + at);
        const f32x4 w = *p;
        const float k = a.lr * m.lr_mult, d = a.wd * m.decay_mult;
#pragma unroll
        for (int e = 0; e < 4; ++e) u[e] = w[e] - k * (m.scale * u[e] + d * w[e]);
        *p = u;
    } else if (a.dt == FC_F32) {
        *reinterpret_cast<f32x4_any*>(static_cast<float*>(a.out) + at) = u;
    } else if (a.dt == FC_F16) {
        *reinterpret_cast<fc::f16x4_any*>(static_cast<f16*>(a.out) + at) = __builtin_convertvector(u, f16x4);
    } else {
        *reinterpret_cast<fc::b16x4_any*>(static_cast<bf16*>(a.out) + at) = __builtin_convertvector(u, fc::b16x4);
    }
}

// The direction made orthogonal: g itself, or a momentum update of it.
struct Source {
    const void* g;
    float* v;                // momentum, or null: g itself
    float c, mu;             // 1 / batch
    int nesterov;
};

// Element i of the direction; `update`: the momentum is updated and stored first.
template <typename T, bool STEP> __device__ __forceinline__ float direction(const Source& a, uint64_t i, bool update) {
    float g = (float)static_cast<const T*>(a.g)[i];
    if constexpr (STEP) {
        g *= a.c;
        float v = a.v[i];
        if (update) {
            v = a.mu * v + g;
            a.v[i] = v;
        }
        return a.nesterov ? g + a.mu * v : v;
    }
    return g;
}

// Four elements from i on; UPDATE: the momentum is updated and stored first.
template <typename T, bool STEP, bool UPDATE> __device__ __forceinline__ void direction4(const Source& a, uint64_t i, float* x) {
    T g[4];
    __builtin_memcpy(g, static_cast<const T*>(a.g) + i, sizeof(g));
    f32x4 v;
    if constexpr (STEP) v = *reinterpret_cast<const f32x4_any*>(a.v + i);
#pragma unroll
    for (int e = 0; e < 4; ++e) {
        x[e] = (float)g[e];
        if constexpr (STEP) {
            x[e] *= a.c;
            if (UPDATE) v[e] = a.mu * v[e] + x[e];
            x[e] = a.nesterov ? x[e] + a.mu * v[e] : v[e];
        }
    }
    if constexpr (STEP && UPDATE) *reinterpret_cast<f32x4_any*>(a.v + i) = v;
}

// Sums of squares of one piece of a matrix, in 64 bits: neither tiny nor huge
// gradients leave its range.
struct NormArgs {
    const Matrix* mats;
    const int2* pieces;      // (matrix, piece)
    double* partial;
    Source d;
};

__device__ __forceinline__ double block_sum(double sum, double* part) {
#pragma unroll
    for (int k = 32; k > 0; k /= 2) sum += __shfl_xor(sum, k);
    if ((threadIdx.x & 63) == 0) part[threadIdx.x >> 6] = sum;
    __syncthreads();
    return (part[0] + part[1]) + (part[2] + part[3]);
}

// Bound by reading the gradient (4096 x 4096 fp32: 16 us, 4.3 TB/s).
template <typename T, bool STEP> __global__ __launch_bounds__(256) void norm_kernel(NormArgs a) {
    __shared__ double part[4];
    const int2 pc = a.pieces[blockIdx.x];
    const Matrix& m = a.mats[pc.x];
    const int64_t total = (int64_t)m.rows * m.cols, lo = pc.y * m.piece_len, hi = min(lo + m.piece_len, total);
    double sum = 0;
    const int64_t whole = lo + (hi - lo) / 4 * 4;  // lo is a multiple of 4, as the offset is
#pragma unroll 4
    for (int64_t i = lo + 4 * threadIdx.x; i < whole; i += 1024) {
        float x[4];
        direction4<T, STEP, true>(a.d, m.offset + i, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) sum += (double)x[e] * x[e];
    }
    if (whole + threadIdx.x < hi) {
        const double x = direction<T, STEP>(a.d, m.offset + whole + threadIdx.x, true);
        sum += x * x;
    }
    sum = block_sum(sum, part);
    if (threadIdx.x == 0) a.partial[m.piece0 + pc.y] = sum;
}

__device__ __forceinline__ void split(float v, f16& hi, f16& lo) {
    hi = (f16)v;
    lo = (f16)(v - (float)hi);
}

struct ScaleArgs {
    const Matrix* mats;
    const Tile* tiles;       // 64 x 64 of X
    const double* partial;
    double top;              // the scale of X
    double alone;            // what the steps make of a singular value of 1
    Source d;
    Output to;
};

// Up to 4 neighbours of the direction, `left` of them in the matrix's row.
template <typename T, bool STEP> __device__ __forceinline__ f32x4 direction_row(const Source& a, uint64_t i, int left) {
    f32x4 v{0.f, 0.f, 0.f, 0.f};
    if (left >= 4) {
        float x[4];
        direction4<T, STEP, false>(a, i, x);
#pragma unroll
        for (int e = 0; e < 4; ++e) v[e] = x[e];
    } else {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) v[e] = direction<T, STEP>(a, i + e, false);
    }
    return v;
}

// X of one tile: the direction over its norm.  A matrix of one row or column has
// the one singular value 1 and is finished here.  Bound by HBM (4096 x 4096 fp32:
// 134 MB in 29 us, 4.6 TB/s).
template <typename T, bool STEP> __global__ __launch_bounds__(256) void scale_kernel(ScaleArgs a) {
    __shared__ float tile[64][65];
    __shared__ double part[4];
    const Tile t = a.tiles[blockIdx.x];
    const Matrix& m = a.mats[t.mat];
    const int r0 = 64 * (m.turned ? t.j : t.i), c0 = 64 * (m.turned ? t.i : t.j);
    const int y = threadIdx.x / 16, z = threadIdx.x % 16 * 4;
    f32x4 d[4];  // rows y, y + 16, ... of the tile in the vector's order
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int r = r0 + y + 16 * q, left = r < m.rows ? m.cols - c0 - z : 0;
        d[q] = direction_row<T, STEP>(a.d, m.offset + (uint64_t)r * m.cols + c0 + z, left);
    }
    double sum = 0;
#pragma unroll
    for (int k = 0; k < PIECES / 256; ++k)
        if (k * 256 + threadIdx.x < m.pieces) sum += a.partial[m.piece0 + k * 256 + threadIdx.x];
    sum = block_sum(sum, part);
    const double f = sum == 0 ? 0 : (m.s == 1 ? a.alone : a.top) / sqrt(sum);
#pragma unroll
    for (int q = 0; q < 4; ++q)
#pragma unroll
        for (int e = 0; e < 4; ++e) d[q][e] = (float)(d[q][e] * f);
    if (m.turned) {
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) tile[y + 16 * q][z + e] = d[q][e];
        __syncthreads();
#pragma unroll
        for (int q = 0; q < 4; ++q)
#pragma unroll
            for (int e = 0; e < 4; ++e) d[q][e] = tile[z + e][y + 16 * q];
    }
#pragma unroll
    for (int q = 0; q < 4; ++q) {
        const int r = 64 * t.i + y + 16 * q, c = 64 * t.j + z;
        if (r >= m.s) break;
        if (m.s == 1) {
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (c + e < m.l) store_one(a.to, m, m.offset + c + e, d[q][e]);
            continue;
        }
        f16x4 hi, lo;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f16 h, l;
            split(d[q][e], h, l);
            hi[e] = h;
            lo[e] = l;
        }
        f16* p = m.x[0] + (int64_t)r * m.lp + c;
        *reinterpret_cast<f16x4*>(p) = hi;
        *reinterpret_cast<f16x4*>(p + m.x_lo) = lo;
    }
}

enum Stage { GRAM, POLY, NEXT, LAST };

struct ProductArgs {
    const Matrix* mats;
    const Tile* tiles;
    int from;                // which x holds X
    // GRAM: A = f0 acc; POLY: B = f0 acc + f1 A; NEXT: X = f0 acc + f1 X.  Each the
    // sum of two floats: a coefficient's rounding is an error of every entry's alike.
    float f0, f1, f0_low, f1_low;
    float unscale;           // LAST: 1 / the scale of X
    Output to;
};

// 4096 x 4096, fp16, a product's launch: with 3 parts A 257 us, B 271, X 390 (0.80, 0.76
// and 1.06 PFLOP/s, the matrix cores busy 56%, 53% and 68% of a unit's cycles at 1.66 to 1.8
// GHz: A's and B's 253 tiles of 192 x 192 take one round of the chip); with
// one part X 141, of which its end 41: it reads and writes X's 8 bytes per element,
// and no other block's products run beside it.
template <typename P, int STAGE> __global__ __launch_bounds__(P::THREADS, 2) void product_kernel(ProductArgs a) {
    const Tile t = a.tiles[blockIdx.x];
    if (t.mat < 0) return;
    const Matrix& m = a.mats[t.mat];
    const f16* x = m.x[a.from];
    Operand A, B;
    int k;
    if constexpr (STAGE == GRAM) {
        A = B = Operand{x, m.lp, m.s, m.lp, m.x_lo};
        k = m.lp;
    } else if constexpr (STAGE == POLY) {
        A = B = Operand{m.a, m.sp, m.s, m.sp, m.a_lo};
        k = m.sp;
    } else {
        A = Operand{m.b, m.sp, m.s, m.sp, m.a_lo};
        B = Operand{x, m.lp, m.l, m.s, m.x_lo};
        k = m.s;
    }
    P p;
    p.run(lds, A, B, t.i * P::BM, t.j * P::BN, 0, k, m.parts);
    const bool both = m.parts == 3;
    f16* const to = STAGE == GRAM ? m.a : STAGE == POLY ? m.b : m.x[1 - a.from];
    const int ld = STAGE <= POLY ? m.sp : m.lp;
    const int64_t lo = STAGE <= POLY ? m.a_lo : m.x_lo;
    const bool halves = STAGE == NEXT || both;
    auto store = [&](int r, int c, const f32x4& v) {  // 4 neighbours of row r
        f16x4 hi, low;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f16 h, l;
            split(v[e], h, l);
            hi[e] = h;
            low[e] = l;
        }
        f16* q = to + (int64_t)r * ld + c;
        *reinterpret_cast<f16x4*>(q) = hi;
        if (halves) *reinterpret_cast<f16x4*>(q + lo) = low;
    };
    // Strip by strip of 16 rows, each wave takes its results through LDS, so that a
    // row's neighbours are in neighbouring lanes where A or X are read and results
    // stored; the next strip's reads are on their way meanwhile.
    float(*const part)[P::WN + 4] = reinterpret_cast<float(*)[P::WN + 4]>(lds + (threadIdx.x >> 6) * 16 * (P::WN + 4) * sizeof(float));
    static_assert(P::WAVES * 16 * (P::WN + 4) * sizeof(float) <= P::LDS, "the strips of all waves fit");
    constexpr int QUADS = P::WN / 4, PER = 16 * QUADS / 64;  // 4 neighbours each, of a row, of a lane
    const int lane = threadIdx.x & 63;
    const int r0 = t.i * P::BM + P::row(0) - (lane & 15), c0 = t.j * P::BN + P::col(0) - 4 * (lane >> 4);
    const f16* const from = STAGE == POLY ? m.a : x;
    const bool second = STAGE != POLY || both;
    const bool mirror = STAGE <= POLY && t.i != t.j;
    constexpr int AHEAD = P::FM < 4 ? P::FM : 4;  // strips whose reads are on their way
    f16x4 high[AHEAD][PER], low[AHEAD][PER];
    auto fetch = [&](int i) {
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int r = r0 + 16 * i + (lane + 64 * k) / QUADS, c = c0 + (lane + 64 * k) % QUADS * 4;
            const f16* q = from + (int64_t)r * ld + c;
            const bool in = r < m.s && c < ld;
            high[i % AHEAD][k] = in ? *reinterpret_cast<const f16x4*>(q) : f16x4{};
            low[i % AHEAD][k] = in && second ? *reinterpret_cast<const f16x4*>(q + lo) : f16x4{};
        }
    };
    if constexpr (STAGE != GRAM) {
#pragma unroll
        for (int i = 0; i < AHEAD; ++i) fetch(i);
    }
    __syncthreads();  // the tiles in LDS are done with
#pragma unroll
    for (int i = 0; i < P::FM; ++i) {
#pragma unroll
        for (int j = 0; j < P::FN; ++j) *reinterpret_cast<f32x4*>(part[lane & 15] + 16 * j + 4 * (lane >> 4)) = p.acc[i][j];
        f32x4 q[PER];
#pragma unroll
        for (int k = 0; k < PER; ++k)
#pragma unroll
            for (int e = 0; e < 4; ++e) q[k][e] = STAGE == GRAM ? 0.f : (float)high[i % AHEAD][k][e] + (float)low[i % AHEAD][k][e];
        if (STAGE != GRAM && i + AHEAD < P::FM) fetch(i + AHEAD);
        __builtin_amdgcn_wave_barrier();
#pragma unroll
        for (int k = 0; k < PER; ++k) {
            const int y = (lane + 64 * k) / QUADS, z = (lane + 64 * k) % QUADS * 4, r = r0 + 16 * i + y, c = c0 + z;
            f32x4 v = *reinterpret_cast<const f32x4*>(part[y] + z);
#pragma unroll
            for (int e = 0; e < 4; ++e)
                v[e] = STAGE == GRAM ? a.f0 * v[e] : fmaf(v[e], a.f0, fmaf(q[k][e], a.f1, fmaf(v[e], a.f0_low, q[k][e] * a.f1_low)));
            if constexpr (STAGE == LAST) {
                *reinterpret_cast<f32x4*>(part[y] + z) = a.unscale * v;
            } else {
                if (r < m.s && c < ld) store(r, c, v);
                if (mirror) *reinterpret_cast<f32x4*>(part[y] + z) = v;
            }
        }
        if constexpr (STAGE == LAST) {
            __builtin_amdgcn_wave_barrier();
#pragma unroll 1
            for (int k = lane; k < 16 * QUADS; k += 64) {
                const int y = m.turned ? k % 4 * 4 : k / QUADS, z = m.turned ? k / 4 : k % QUADS * 4, r = r0 + 16 * i + y, c = c0 + z;
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = m.turned ? part[y + e][z] : part[y][z + e];
                if (m.turned ? c < m.l : r < m.s) store_out(a.to, m, m.turned ? c : r, m.turned ? r : c, v);
            }
        } else if (mirror) {  // 4 neighbours down a column at a time
            __builtin_amdgcn_wave_barrier();
#pragma unroll
            for (int k = 0; k < PER; ++k) {
                const int y = (lane + 64 * k) % 4 * 4, z = (lane + 64 * k) / 4, r = r0 + 16 * i + y, c = c0 + z;
                f32x4 v;
#pragma unroll
                for (int e = 0; e < 4; ++e) v[e] = part[y + e][z];
                if (c < m.s && r < ld) store(c, r, v);
            }
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
    }
}

// ---- small matrices in one block ---------------------------------------------

// All steps of a matrix of at most 128 rows in one block, where it fits: X in
// registers in fp32 (in the layout of the products' results), its high halves (and
// low ones, with 3 parts), A and B in LDS.  Products this small are bound by
// latency: as launches of their own they took 5 us each (96 x 363: 93 us in 17
// launches).  In one block LDS reads would bound them, so that fragments are
// shared: X X^T and A A are computed by a wave per tile row (and per part of k
// where rows are few), B X by a wave per 16 columns, for all rows.
struct WholeArgs {
    const Matrix* mats;
    const int* which;                    // the launch's matrices
    int dt;                              // of the gradient
    bool step;                           // a momentum step
    double top, alone;                   // as ScaleArgs
    Source d;
    Output to;
    int steps;
    float fa;                            // A = fa acc
    float fb, fb_low, fb1, fb1_low;      // B = fb acc + fb1 A
    float fx, fx1, fx1_low;              // X = fx acc + fx1 X
    float unscale;
};

constexpr int WHOLE_WAVES = 8, WHOLE_TILES = 20, WHOLE_ROWS = 8;  // waves; tiles of X of 16 x 16 per wave; tile rows

template <int ST> struct Whole {
    static constexpr int ROWS = ST;
    static constexpr int NJ = WHOLE_TILES / ST;                  // tile columns of a wave
    static constexpr int S32 = (ST + 1) / 2 * 32, PA = S32 + 8;  // k of A and B, and their row pitch in LDS
    static constexpr int KS = ST <= 2 ? 4 : ST <= 4 ? 2 : 1;     // waves that share a tile row of A
    static constexpr int TILES = ST * ST;
    static __host__ __device__ int pitch(int l) { return (l + 63) / 64 * 64 + 8; }
    static __host__ __device__ int halves(int l) { return S32 * pitch(l) + 2 * S32 * PA; }
    static int bytes(int l, int parts) {
        const int lt = (l + 63) / 64 * 4, flat = 256 + 16 * ST * (16 * lt + 4) * 4;
        const int b = std::max(flat, 256 + halves(l) * 2 * (parts == 3 ? 2 : 1) + (KS - 1) * TILES * 1024);
        return lt <= NJ * WHOLE_WAVES && b <= 160 * 1024 ? b : 0;
    }
};

typedef FC_LDS const fc::f16x8* RowAt;
typedef FC_LDS fc::s16x4* TurnAt;

template <int ST> __global__ __launch_bounds__(64 * WHOLE_WAVES) void whole_kernel(WholeArgs a) {
    typedef Whole<ST> W;
    typedef fc::Half<f16> H;
    constexpr int NJ = W::NJ, S32 = W::S32, PA = W::PA, KS = W::KS;
    const Matrix& m = a.mats[a.which[blockIdx.x]];
    const int parts = m.parts, l64 = (m.l + 63) / 64 * 64, px = W::pitch(m.l), lt = l64 / 16;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
    int row = lane & 15, four = 4 * (lane >> 4);
    double* const part = reinterpret_cast<double*>(lds);
    f16* const xs = reinterpret_cast<f16*>(lds + 256);
    f16* const as = xs + S32 * px;
    f16* const bs = as + S32 * PA;
    const int low = W::halves(m.l);      // from a high half to its low one
    f32x4* const sums = reinterpret_cast<f32x4*>(xs + low * (parts == 3 ? 2 : 1));  // [part of k][tile][lane]
    // The direction, read in the order of memory, goes through LDS in fp32 to the
    // layout of results: tile (i, j) of a wave is X's tile row i, column
    // wave + 8 j, a lane's 4 neighbours of a row.  (Short loops: code run once is
    // read from memory, and unrolled it cost more time than the steps.)
    float* const flat = reinterpret_cast<float*>(lds + 256);
    const int pf = l64 + 4, count = m.rows * m.cols;
    for (int i = threadIdx.x; i < 16 * ST * pf / 4; i += 64 * WHOLE_WAVES) reinterpret_cast<f32x4*>(flat)[i] = f32x4{0.f, 0.f, 0.f, 0.f};
    __syncthreads();
    double sum = 0;
    constexpr int THREADS = 64 * WHOLE_WAVES, AHEAD = 16;  // elements of a thread whose reads are under way together
    const int down = THREADS / m.cols, right = THREADS % m.cols;
    // body(u, element's place in LDS) for a thread's elements k0 + THREADS u that are in the matrix
    auto each = [&](int k0, int& r, int& c, auto&& body) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            if (k0 + THREADS * u < count) body(u, m.turned ? c * pf + r : r * pf + c);
            r += down;
            c += right;
            if (c >= m.cols) {
                c -= m.cols;
                ++r;
            }
        }
    };
    auto read = [&](auto* type) {
        typedef std::remove_pointer_t<decltype(type)> T;
        const T* const g = static_cast<const T*>(a.d.g) + m.offset;
        int r = threadIdx.x / m.cols, c = threadIdx.x % m.cols;
        for (int k0 = threadIdx.x; k0 < count; k0 += THREADS * AHEAD) {
            T q[AHEAD];
#pragma unroll
            for (int u = 0; u < AHEAD; ++u) q[u] = g[min(k0 + THREADS * u, count - 1)];
            each(k0, r, c, [&](int u, int place) {
                float d = (float)q[u];
                if (a.step) {
                    float* const p = a.d.v + m.offset + k0 + THREADS * u;
                    d *= a.d.c;
                    const float v = a.d.mu * *p + d;
                    *p = v;
                    d = a.d.nesterov ? d + a.d.mu * v : v;
                }
                flat[place] = d;
                sum += (double)d * d;
            });
        }
    };
    if (a.dt == FC_F32) read(static_cast<float*>(nullptr));
    else if (a.dt == FC_F16) read(static_cast<f16*>(nullptr));
    else read(static_cast<bf16*>(nullptr));
#pragma unroll
    for (int k = 32; k > 0; k /= 2) sum += __shfl_xor(sum, k);
    if (lane == 0) part[wave] = sum;
    __syncthreads();
    sum = 0;
#pragma unroll
    for (int k = 0; k < WHOLE_WAVES; ++k) sum += part[k];
    const bool alone = m.s == 1;  // has the one singular value 1
    const double f = sum == 0 ? 0 : (alone ? a.alone : a.top) / sqrt(sum);
    const float unscale = alone ? 1.f : a.unscale;

    auto four_of = [](const float* q, float k) { return f32x4{q[0] * k, q[1] * k, q[2] * k, q[3] * k}; };
    // Returns the values as stored: b A + c A A is formed from one A, of which the
    // rounding then cancels where the terms do.
    auto put = [&](f16* p, const f32x4& v) {
        f16x4 hi, lo;
        f32x4 kept;
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            f16 h, l;
            split(v[e], h, l);
            hi[e] = h;
            lo[e] = l;
            kept[e] = parts == 3 ? (float)h + (float)l : (float)h;
        }
        *reinterpret_cast<f16x4*>(p) = hi;
        if (parts == 3) *reinterpret_cast<f16x4*>(p + low) = lo;
        return kept;
    };
    float x[NJ][ST][4];
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < ST; ++i) {
            // past X's last column: that one again, not kept
            const f32x4 q = *reinterpret_cast<const f32x4*>(flat + (16 * i + row) * pf + 16 * min(wave + WHOLE_WAVES * j, lt - 1) + four);
#pragma unroll
            for (int e = 0; e < 4; ++e) x[j][i][e] = (float)(q[e] * f);
            __builtin_amdgcn_sched_barrier(0);
        }
    __syncthreads();
    for (int i = threadIdx.x; i < low * (parts == 3 ? 2 : 1) / 4; i += 64 * WHOLE_WAVES) reinterpret_cast<f16x4*>(xs)[i] = f16x4{};
    __syncthreads();
    auto put_x = [&]() {
#pragma unroll
        for (int j = 0; j < NJ; ++j) {
#pragma unroll
            for (int i = 0; i < ST; ++i) {
                if (wave + WHOLE_WAVES * j < lt) put(xs + (16 * i + row) * px + 16 * (wave + WHOLE_WAVES * j) + four, four_of(x[j][i], 1.f));
                __builtin_amdgcn_sched_barrier(0);
            }
        }
    };
    put_x();
    __syncthreads();

    // Fragments: 16 rows by 32 of k, along k; and 16 columns by 32 of k, across it.
    auto along = [](uint32_t at) { return *(RowAt)(uintptr_t)at; };
    auto across = [](uint32_t at, uint32_t four_rows) {
        union {
            fc::s16x4 s[2];
            fc::f16x8 v;
        } u;
        u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TurnAt)(uintptr_t)at);
        u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((TurnAt)(uintptr_t)(at + four_rows));
        return u.v;
    };
    // products of `parts` parts: high by low, low by high, high by high
    auto first = [&](int q) -> uint32_t { return parts == 3 && q == 1 ? 2 * low : 0; };
    auto second = [&](int q) -> uint32_t { return parts == 3 && q == 0 ? 2 * low : 0; };
    const uint32_t xa = fc::lds_address(xs), aa = fc::lds_address(as), ba = fc::lds_address(bs);
    const int mine = wave % ST, share = wave / ST;  // the tile row of A, the part of k

    // the tile row `mine` of P P^T, P's rows along k of k32 in all
    auto square = [&](uint32_t base, int pitch, int k32, bool active, f32x4* acc) {
#pragma unroll
        for (int j = 0; j < ST; ++j) acc[j] = f32x4{0.f, 0.f, 0.f, 0.f};
        if (!active) return;
        const uint32_t at = base + 2 * (row * pitch + 2 * four);
        constexpr int UNROLL = ST <= 4 ? 2 : 1;
        for (int q = 0; q < parts; ++q)
#pragma unroll UNROLL
            for (int k = share * 64; k < 2 * k32; k += 64 * KS) {
                const fc::f16x8 fa = along(at + first(q) + 32 * mine * pitch + k);
                fc::f16x8 fb[ST];
#pragma unroll
                for (int j = 0; j < ST; ++j)
                    fb[j] = along(at + second(q) + 32 * j * pitch + k);
#pragma unroll
                for (int j = 0; j < ST; ++j)
                    acc[j] = H::mma(fb[j], fa, acc[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        if constexpr (KS > 1) {
            if (share > 0) {
#pragma unroll
                for (int j = 0; j < ST; ++j)
                    sums[((share - 1) * W::TILES + mine * ST + j) * 64 + lane] = acc[j];
            }
        }
    };
    auto join = [&](f32x4* acc) {
        if constexpr (KS > 1) {
            __syncthreads();
            if (share > 0) return;
#pragma unroll
            for (int k = 0; k < KS - 1; ++k)
#pragma unroll
                for (int j = 0; j < ST; ++j)
                    acc[j] += sums[(k * W::TILES + mine * ST + j) * 64 + lane];
        }
    };

    for (int step = 0; step < a.steps && !alone; ++step) {
        f32x4 g[ST], b[ST];
        asm volatile("" : "+v"(row), "+v"(four));  // addresses are made again in every step: kept, they would not fit
        square(xa, px, l64, share < KS, g);
        join(g);
        if (share == 0) {
#pragma unroll
            for (int j = 0; j < ST; ++j) {
                g[j] = put(as + (16 * mine + row) * PA + 16 * j + four, a.fa * g[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();
        square(aa, PA, S32, share < KS, b);
        join(b);
        if (share == 0) {
#pragma unroll
            for (int j = 0; j < ST; ++j) {
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    b[j][e] = fmaf(b[j][e], a.fb, fmaf(g[j][e], a.fb1, fmaf(b[j][e], a.fb_low, g[j][e] * a.fb1_low)));
                put(bs + (16 * mine + row) * PA + 16 * j + four, b[j]);
                __builtin_amdgcn_sched_barrier(0);
            }
        }
        __syncthreads();
        f32x4 acc[NJ][ST];
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < ST; ++i) acc[j][i] = f32x4{0.f, 0.f, 0.f, 0.f};
        for (int q = 0; q < parts; ++q)
            for (int k = 0; k < S32; k += 32) {
                fc::f16x8 fa[ST];
#pragma unroll
                for (int i = 0; i < ST; ++i) fa[i] = along(ba + first(q) + 2 * ((16 * i + row) * PA + k + 2 * four));
#pragma unroll
                for (int j = 0; j < NJ; ++j) {
                    const int c = wave + WHOLE_WAVES * j;
                    if (c >= lt) break;
                    const fc::f16x8 fb = across(xa + second(q) + 2 * ((k + 2 * four + (row >> 2)) * px + 16 * c + 4 * (row & 3)), 8 * px);
#pragma unroll
                    for (int i = 0; i < ST; ++i) acc[j][i] = H::mma(fb, fa[i], acc[j][i]);
                    __builtin_amdgcn_sched_barrier(0);
                }
            }
#pragma unroll
        for (int j = 0; j < NJ; ++j)
#pragma unroll
            for (int i = 0; i < ST; ++i)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    x[j][i][e] = fmaf(acc[j][i][e], a.fx, fmaf(x[j][i][e], a.fx1, x[j][i][e] * a.fx1_low));
        __builtin_amdgcn_sched_barrier(0);
        if (step + 1 < a.steps) {
            __syncthreads();
            put_x();
            __syncthreads();
        }
    }
    __syncthreads();  // A, B and X in LDS are done with
#pragma unroll
    for (int j = 0; j < NJ; ++j)
#pragma unroll
        for (int i = 0; i < ST; ++i) {
            const int c = 16 * (wave + WHOLE_WAVES * j) + four;
            if (c < l64) *reinterpret_cast<f32x4*>(flat + (16 * i + row) * pf + c) = four_of(x[j][i], unscale);
        }
    __syncthreads();
    auto write = [&](auto&& store) {
        int r = threadIdx.x / m.cols, c = threadIdx.x % m.cols;
        for (int k0 = threadIdx.x; k0 < count; k0 += THREADS * AHEAD)
            each(k0, r, c, [&](int u, int place) { store(m.offset + k0 + THREADS * u, flat[place]); });
    };
    if (!a.to.out) {
        const float k = a.to.lr * m.lr_mult, d = a.to.wd * m.decay_mult;
        write([&](uint64_t at, float u) {
            const float w = a.to.w[at];
            a.to.w[at] = w - k * (m.scale * u + d * w);
        });
    } else if (a.to.dt == FC_F32) {
        write([&](uint64_t at, float u) { static_cast<float*>(a.to.out)[at] = u; });
    } else if (a.to.dt == FC_F16) {
        write([&](uint64_t at, float u) { static_cast<f16*>(a.to.out)[at] = (f16)u; });
    } else {
        write([&](uint64_t at, float u) { static_cast<bf16*>(a.to.out)[at] = (bf16)u; });
    }
}

// f(Whole<tile rows>) for a matrix's shorter side.
template <typename F> auto with_rows(int tile_rows, F&& f) {
    switch (tile_rows) {
        case 1: return f(Whole<1>{});
        case 2: return f(Whole<2>{});
        case 3: return f(Whole<3>{});
        case 4: return f(Whole<4>{});
        case 5: return f(Whole<5>{});
        case 6: return f(Whole<6>{});
        case 7: return f(Whole<7>{});
        default: return f(Whole<8>{});
    }
}

// Bytes of LDS of a matrix in one block, or 0 where it is too large.
int whole_lds(int s, int l, int parts) {
    if (s > 16 * WHOLE_ROWS || l > 8192) return 0;
    return with_rows((s + 15) / 16, [&](auto w) { return decltype(w)::bytes(l, parts); });
}

template <int ST> hipError_t prepare_whole() {
    return hipFuncSetAttribute((const void*)whole_kernel<ST>, hipFuncAttributeMaxDynamicSharedMemorySize, 160 * 1024);
}

// By fc::TileKind.  LARGE has no registers left for sums in runs: symmetric products
// of fp32's accuracy do without it, X's take it for its speed.  BROAD serves the
// symmetric products alone; for X it has not been measured.
template <bool BS> using Large = fc::Product<f16, 256, 256, 128, 64, false, BS>;
template <bool BS> using Broad = fc::Product<f16, 192, 192, 96, 48, false, BS, 2, 8>;
template <bool BS> using Middle = fc::Product<f16, 128, 128, 64, 64, false, BS, 2, 8>;
template <bool BS> using Small = fc::Product<f16, 64, 64, 32, 32, false, BS, 4, 8>;

template <typename P, int STAGE> hipError_t prepare_one() {
    return hipFuncSetAttribute((const void*)product_kernel<P, STAGE>, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS);
}

hipError_t prepare() {
    for (hipError_t e : {prepare_one<Large<false>, GRAM>(), prepare_one<Large<false>, POLY>(), prepare_one<Large<true>, NEXT>(),
                         prepare_one<Large<true>, LAST>(), prepare_one<Broad<false>, GRAM>(), prepare_one<Broad<false>, POLY>(),
                         prepare_one<Middle<false>, GRAM>(), prepare_one<Middle<false>, POLY>(), prepare_one<Middle<true>, NEXT>(),
                         prepare_one<Middle<true>, LAST>(), prepare_one<Small<false>, GRAM>(), prepare_one<Small<false>, POLY>(),
                         prepare_one<Small<true>, NEXT>(), prepare_one<Small<true>, LAST>(), prepare_whole<1>(),
                         prepare_whole<2>(), prepare_whole<3>(), prepare_whole<4>(), prepare_whole<5>(), prepare_whole<6>(),
                         prepare_whole<7>(), prepare_whole<8>()})
        if (e != hipSuccess) return e;
    return hipSuccess;
}

template <typename P, int STAGE> void launch(const ProductArgs& a, int count, hipStream_t s) {
    product_kernel<P, STAGE><<<count, P::THREADS, P::LDS, s>>>(a);
}

template <int STAGE> void launch_kind(int kind, const ProductArgs& a, int count, hipStream_t s) {
    constexpr bool BS = STAGE >= NEXT;
    if (kind == fc::TILE_LARGE) return launch<Large<BS>, STAGE>(a, count, s);
    if (kind == fc::TILE_MIDDLE) return launch<Middle<BS>, STAGE>(a, count, s);
    if (kind == fc::TILE_SMALL) return launch<Small<BS>, STAGE>(a, count, s);
    if constexpr (!BS) launch<Broad<BS>, STAGE>(a, count, s);
}

constexpr int64_t SIDE_LIMIT = 1 << 20;
constexpr int64_t COUNT_LIMIT = 1 << 20;
constexpr int MOST_STEPS = 64;

double most(double a, double b, double c, double top) {  // of |a x + b x^3 + c x^5| on [0, top]
    double m = 0;
    for (int i = 0; i <= 4096; ++i) {
        const double x = top * i / 4096, y = x * x;
        m = std::max(m, std::fabs(x * (a + y * (b + y * c))));
    }
    return std::isfinite(a) && std::isfinite(b) && std::isfinite(c) ? m : HUGE_VAL;
}

double pow2_below(double x) { return std::exp2(std::floor(std::log2(x))); }

}  // namespace

struct fc_muon {
    fc::CallOrder order;
    fc::DeviceBlock block;
    std::vector<fc_matrix> host;
    uint64_t extent = 0;
    int dtype = FC_BF16;
    int steps = 5, nesterov = 1;
    double a = 0, b = 0, c = 0;
    double sx = 1, sa = 1, sb = 1;   // scales of X, A, B
    double alone = 1;                // what the steps make of a singular value of 1
    const Matrix* mats = nullptr;
    const int2* pieces = nullptr;
    int n_pieces = 0;
    double* partial = nullptr;
    const Tile* scale_tiles = nullptr;
    int n_scale = 0;
    struct Launch {
        int kind, count;
        const Tile* tiles;
    };
    std::vector<Launch> launches[3];  // of the products GRAM, POLY, NEXT
    struct WholeLaunch {
        int tile_rows, count, lds;
        const int* which;
    };
    std::vector<WholeLaunch> whole;   // where every matrix is one block's
};

namespace {

// Everything of the plan in device memory, built on the host.
int build(fc_muon* p) {
    const int n = (int)p->host.size();
    std::vector<Matrix> mats(n);
    fc::Layout at;
    const uint64_t o_mats = at.take(n * sizeof(Matrix));
    std::vector<int2> pieces;
    std::vector<Tile> scale;
    std::vector<fc::TileShape> shapes[3];
    for (int i = 0; i < n; ++i) {
        const fc_matrix& h = p->host[i];
        Matrix& m = mats[i];
        std::memset(&m, 0, sizeof m);
        m.offset = h.offset;
        m.rows = (int)h.rows;
        m.cols = (int)h.cols;
        m.turned = h.rows > h.cols;
        m.s = std::min(m.rows, m.cols);
        m.l = std::max(m.rows, m.cols);
        m.sp = (m.s + 63) / 64 * 64;
        m.lp = (m.l + 63) / 64 * 64;
        m.parts = p->dtype == FC_BF16 && m.s > 32 ? 1 : 3;
        m.lr_mult = h.lr_mult;
        m.decay_mult = h.decay_mult;
        m.scale = (float)std::sqrt(std::max(1.0, (double)h.rows / h.cols));
        const int64_t total = (int64_t)m.rows * m.cols;
        m.piece_len = fc::ceil_div(fc::ceil_div(total, std::min<int64_t>(PIECES, fc::ceil_div(total, 4096))), 4) * 4;
        m.pieces = (int)fc::ceil_div(total, m.piece_len);
        m.piece0 = (int)pieces.size();
        for (int k = 0; k < m.pieces; ++k) pieces.push_back({i, k});
        for (int r = 0; r < (m.s + 63) / 64; ++r)
            for (int c = 0; c < m.lp / 64; ++c) scale.push_back({i, r, c});
        const bool alone = m.s == 1;  // needs no products
        shapes[GRAM].push_back({alone ? 0 : m.s, m.s, m.parts * m.lp / 64});
        shapes[POLY].push_back({alone ? 0 : m.s, m.s, m.parts * m.sp / 64});
        shapes[NEXT].push_back({alone ? 0 : m.s, m.l, m.parts * m.sp / 64});
    }
    // Every matrix in a block of its own, where all of them fit: beside the larger
    // ones of a mixed list they would only add a launch.
    std::vector<int> lists[WHOLE_ROWS];
    int bytes[WHOLE_ROWS] = {};
    bool whole = n > 0;
    for (int i = 0; i < n && whole; ++i) {
        const int need = whole_lds(mats[i].s, mats[i].l, mats[i].parts), t = std::min((mats[i].s + 15) / 16, WHOLE_ROWS) - 1;
        whole = need > 0;
        lists[t].push_back(i);
        bytes[t] = std::max(bytes[t], need);
    }
    std::vector<int> which;
    if (whole) {
        pieces.clear();
        scale.clear();
        for (auto& v : shapes) v.clear();
        for (const auto& v : lists) which.insert(which.end(), v.begin(), v.end());
    }
    const bool fine = p->dtype != FC_BF16;
    std::vector<int> symmetric{fc::TILE_LARGE, fc::TILE_BROAD, fc::TILE_MIDDLE, fc::TILE_SMALL};
    if (fine) symmetric.erase(symmetric.begin());
    std::vector<fc::TileLaunch> plans[3] = {fc::plan_tiles(shapes[GRAM], true, symmetric), fc::plan_tiles(shapes[POLY], true, symmetric),
                                            fc::plan_tiles(shapes[NEXT], false, {fc::TILE_LARGE, fc::TILE_MIDDLE, fc::TILE_SMALL})};
    const uint64_t o_pieces = at.take(pieces.size() * sizeof(int2)), o_partial = at.take(pieces.size() * sizeof(double)),
                   o_scale = at.take(scale.size() * sizeof(Tile)), o_which = at.take(which.size() * sizeof(int));
    std::vector<uint64_t> o_tiles;
    for (const auto& v : plans)
        for (const fc::TileLaunch& l : v) o_tiles.push_back(at.take(l.tiles.size() * sizeof(Tile)));
    const uint64_t tables = at.size;
    std::vector<uint64_t> places(n * 4);
    for (int i = 0; i < n; ++i) {
        Matrix& m = mats[i];
        m.x_lo = (int64_t)m.s * m.lp;
        m.a_lo = (int64_t)m.s * m.sp;
        if (whole) continue;
        for (int k = 0; k < 2; ++k) places[4 * i + k] = at.take(2 * m.x_lo * sizeof(f16));
        for (int k = 2; k < 4; ++k) places[4 * i + k] = at.take((m.parts == 3 ? 2 : 1) * m.a_lo * sizeof(f16));
    }
    int rc = p->block.create(at.size);
    if (rc) return rc;
    char* b = p->block.p;
    for (int i = 0; i < n && !whole; ++i) {
        mats[i].x[0] = reinterpret_cast<f16*>(b + places[4 * i]);
        mats[i].x[1] = reinterpret_cast<f16*>(b + places[4 * i + 1]);
        mats[i].a = reinterpret_cast<f16*>(b + places[4 * i + 2]);
        mats[i].b = reinterpret_cast<f16*>(b + places[4 * i + 3]);
    }
    std::vector<char> image(tables);
    auto put = [&](uint64_t to, const void* from, size_t bytes) {
        if (bytes) std::memcpy(image.data() + to, from, bytes);
    };
    put(o_mats, mats.data(), n * sizeof(Matrix));
    put(o_pieces, pieces.data(), pieces.size() * sizeof(int2));
    put(o_scale, scale.data(), scale.size() * sizeof(Tile));
    put(o_which, which.data(), which.size() * sizeof(int));
    const int* list = reinterpret_cast<const int*>(b + o_which);
    for (int t = 0; t < WHOLE_ROWS && whole; ++t) {
        const int count = (int)lists[t].size();
        if (count) p->whole.push_back({t + 1, count, bytes[t], list});
        list += count;
    }
    size_t next = 0;
    for (int q = 0; q < 3; ++q)
        for (const fc::TileLaunch& l : plans[q]) {
            put(o_tiles[next], l.tiles.data(), l.tiles.size() * sizeof(Tile));
            p->launches[q].push_back({l.kind, (int)l.tiles.size(), reinterpret_cast<const Tile*>(b + o_tiles[next])});
            ++next;
        }
    if (tables && hipMemcpy(b, image.data(), tables, hipMemcpyHostToDevice) != hipSuccess) return FC_EHIP;
    p->mats = reinterpret_cast<const Matrix*>(b + o_mats);
    p->pieces = reinterpret_cast<const int2*>(b + o_pieces);
    p->n_pieces = (int)pieces.size();
    p->partial = reinterpret_cast<double*>(b + o_partial);
    p->scale_tiles = reinterpret_cast<const Tile*>(b + o_scale);
    p->n_scale = (int)scale.size();
    return FC_OK;
}

// A coefficient as the sum of two floats.
void halve(double f, float& high, float& low) {
    high = (float)f;
    low = (float)(f - high);
}

template <typename T, bool STEP> int run(fc_muon* p, const Source& d, int dt, const Output& to, hipStream_t s) {
    const double fa = p->sa / (p->sx * p->sx), fb = p->c * p->sb / (p->sa * p->sa), fb1 = p->b * p->sb / p->sa;
    if (!p->whole.empty()) {
        WholeArgs a{};
        a.mats = p->mats;
        a.dt = dt;
        a.step = STEP;
        a.top = p->sx;
        a.alone = p->alone;
        a.d = d;
        a.to = to;
        a.steps = p->steps;
        a.fa = (float)fa;
        halve(fb, a.fb, a.fb_low);
        halve(fb1, a.fb1, a.fb1_low);
        a.fx = (float)(1 / p->sb);
        halve(p->a, a.fx1, a.fx1_low);
        a.unscale = (float)(1 / p->sx);
        for (const auto& w : p->whole) {
            a.which = w.which;
            with_rows(w.tile_rows, [&](auto k) {
                whole_kernel<decltype(k)::ROWS><<<w.count, 64 * WHOLE_WAVES, w.lds, s>>>(a);
                return 0;
            });
        }
        return fc::hip_code(hipGetLastError());
    }
    NormArgs norm{p->mats, p->pieces, p->partial, d};
    norm_kernel<T, STEP><<<p->n_pieces, 256, 0, s>>>(norm);
    ScaleArgs scale{p->mats, p->scale_tiles, p->partial, p->sx, p->alone, d, to};
    scale_kernel<T, STEP><<<p->n_scale, 256, 0, s>>>(scale);
    int from = 0;
    for (int k = 0; k < p->steps; ++k) {
        ProductArgs a{};
        a.to = to;
        a.mats = p->mats;
        a.from = from;
        a.f0 = (float)fa;
        for (const auto& l : p->launches[GRAM]) {
            a.tiles = l.tiles;
            launch_kind<GRAM>(l.kind, a, l.count, s);
        }
        halve(fb, a.f0, a.f0_low);
        halve(fb1, a.f1, a.f1_low);
        for (const auto& l : p->launches[POLY]) {
            a.tiles = l.tiles;
            launch_kind<POLY>(l.kind, a, l.count, s);
        }
        halve(1 / p->sb, a.f0, a.f0_low);
        halve(p->a, a.f1, a.f1_low);
        a.unscale = (float)(1 / p->sx);
        for (const auto& l : p->launches[NEXT]) {
            a.tiles = l.tiles;
            if (k + 1 < p->steps) launch_kind<NEXT>(l.kind, a, l.count, s);
            else launch_kind<LAST>(l.kind, a, l.count, s);
        }
        from ^= 1;
    }
    return fc::hip_code(hipGetLastError());
}

int orthogonalize_body(fc_muon* p, const void* g, int gdt, void* out, hipStream_t s) {
    if (!p) return FC_EINVAL;
    const int64_t n = (int64_t)p->extent;
    int rc = fc::check_spans({{g, 1, n, n, fc::dtype_bytes(gdt), false}, {out, 1, n, n, fc::dtype_bytes(p->dtype), true}});
    if (rc || n == 0) return rc;
    if (reinterpret_cast<uintptr_t>(g) % 16 || reinterpret_cast<uintptr_t>(out) % 16) return FC_EALIGN;
    bool note;
    rc = p->order.begin(s, note);
    if (rc) return rc;
    const Source d{g, nullptr, 1.f, 0.f, 0};
    const Output to{out, p->dtype, nullptr, 0.f, 0.f};
    if (gdt == FC_F32) rc = run<float, false>(p, d, gdt, to, s);
    else if (gdt == FC_F16) rc = run<f16, false>(p, d, gdt, to, s);
    else rc = run<bf16, false>(p, d, gdt, to, s);
    p->order.done(s, note);
    return rc;
}

int step_body(fc_muon* p, float* w, float* v, const float* g, float lr, float mu, float wd, int batch, hipStream_t s) {
    if (!p || batch < 1) return FC_EINVAL;
    const int64_t n = (int64_t)p->extent;
    int rc = fc::check_spans({{w, 1, n, n, 4, true}, {v, 1, n, n, 4, true}, {g, 1, n, n, 4, false}});
    if (rc || n == 0) return rc;
    for (const void* q : {(const void*)w, (const void*)v, (const void*)g})
        if (reinterpret_cast<uintptr_t>(q) % 16) return FC_EALIGN;
    bool note;
    rc = p->order.begin(s, note);
    if (rc) return rc;
    const Source d{g, v, 1.0f / (float)batch, mu, p->nesterov};
    const Output to{nullptr, FC_F32, w, lr, wd};
    rc = run<float, true>(p, d, FC_F32, to, s);
    p->order.done(s, note);
    return rc;
}

}  // namespace

extern "C" {

int fc_muon_create(fc_muon** plan, const fc_matrix* mats, int n, int dtype, int steps, const double* coefficients, int nesterov) {
    if (!plan) return FC_EINVAL;
    *plan = nullptr;
    if (n < 0 || n > COUNT_LIMIT || (n > 0 && !mats) || !fc::dtype_bytes(dtype) || steps < 1 || steps > MOST_STEPS) return FC_EINVAL;
    const double usual[3] = {3.4445, -4.7750, 2.0315};
    const double* q = coefficients ? coefficients : usual;
    uint64_t end = 0;
    for (int i = 0; i < n; ++i) {
        const fc_matrix& m = mats[i];
        if (m.rows < 1 || m.cols < 1 || m.rows > SIDE_LIMIT || m.cols > SIDE_LIMIT || m.offset < end || m.offset >= (uint64_t)1 << 48) return FC_EINVAL;
        if (m.offset % 4) return FC_EALIGN;
        end = m.offset + m.rows * m.cols;
    }
    // singular values start in [0, 1]; the scales hold for what the polynomial makes of them
    double top = 1;
    for (int k = 0; k < steps; ++k) {
        top = std::max(top, most(q[0], q[1], q[2], top));
        if (!(top <= 2)) return FC_EINVAL;
    }
    double by = 0;
    for (int i = 0; i <= 4096; ++i) {
        const double y = top * top * i / 4096;
        by = std::max(by, std::fabs(y * (q[1] + y * q[2])));
    }
    if (!(by <= 1024)) return FC_EINVAL;
    return fc::no_throw([&] {
        fc_muon* p = new fc_muon;
        p->host.assign(mats, mats + n);
        p->extent = end;
        p->dtype = dtype;
        p->steps = steps;
        p->nesterov = nesterov != 0;
        p->a = q[0];
        p->b = q[1];
        p->c = q[2];
        for (int k = 0; k < steps; ++k) {
            const double y = p->alone * p->alone;
            p->alone *= q[0] + y * (q[1] + y * q[2]);
        }
        p->sx = pow2_below(32768 / top);
        p->sa = pow2_below(32768 / (top * top));
        p->sb = by > 0 ? pow2_below(32768 / by) : 1;
        int rc = p->order.create();
        if (!rc) rc = fc::hip_code(prepare());
        if (!rc) rc = build(p);
        if (rc) {
            fc_muon_destroy(p);
            return rc;
        }
        *plan = p;
        return FC_OK;
    });
}

void fc_muon_destroy(fc_muon* p) {
    if (!p) return;
    p->block.destroy();
    p->order.destroy();
    delete p;
}

int fc_muon_orthogonalize(fc_muon* p, const void* g, int g_dtype, void* out, void* stream) {
    return fc::no_throw([&] { return orthogonalize_body(p, g, g_dtype, out, static_cast<hipStream_t>(stream)); });
}

int fc_muon_step(fc_muon* p, float* w, float* v, const float* g, float lr, float mu, float wd, int batch, void* stream) {
    return fc::no_throw([&] { return step_body(p, w, v, g, lr, mu, wd, batch, static_cast<hipStream_t>(stream)); });
}

}  // extern "C"
