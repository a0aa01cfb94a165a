// Softmax cross entropy over a vocabulary, with its gradients (fc_lm.h).
//
//   l = x w^T, lse[t] = log sum exp l[t, :], loss[t] = lse[t] - l[t, y[t]]
//   d = softmax(l) - onehot(y), dx = scale d w, dw = scale d^T x
//
// The products are 2 tokens rows dim operations each and bound everything but
// short lists, where reading w does.  The logits are never stored, but for gradients
// 16 bits per token and row are.  A block of the
// first product holds a piece of the vocabulary for its tokens in fp32: it takes
// the piece's maximum m and sum of exponentials, keeps both (8 bytes), the
// target's logit, and, when gradients are wanted, the numerators exp(l - m) in 16
// bits (fp32 for up to 64 tokens).  One small kernel joins a token's pieces into lse and the loss; one pass
// over the numerators then turns them into d (numerator * exp(m - lse), minus one
// at the target), and two products make the gradients of it.  The alternative
// that keeps nothing computes the first product twice: 8 instead of 6 units of
// work, against one read and one write of 16 bits per token and row.
//
// Tokens go through in chunks so that the numerators take at most 4 GiB; with
// more than one chunk, dw is summed in fp32 over them and rounded after the last.
//
// Measured, fp16, 8192 tokens, 131072 rows of 2048: 12.6 ms for 13.2 TFLOP (1.05
// PFLOP/s; a library's three products of these shapes alone 10.9); in a trace (13.4
// in all) the first product 4.5 ms, dw 4.3, dx 3.8, the pass from numerators to d 0.81
// (4.3 GB), join 0.02, the copy of x 0.02.  bf16, 24 tokens, 65536 rows of 2048, losses
// only: 67 us with other data in the caches (268 MB at 4.0 TB/s), 47 call after call.
#include <algorithm>

#include "fc_gemm.h"
#include "fc_lm_host.h"

using fc::Operand;
using fc::f32x2;
using fc::f32x4;
using fc::Half;

namespace {

typedef _Float16 f16;
typedef __bf16 bf16;

extern __shared__ __align__(1024) char lds[];

constexpr float LOG2E = 1.44269504088896341f;

// Numerators of 16 bits and d are stored times this: fp16 then keeps what is down to
// 2^-29 of a piece's largest (a numerator) or of 1 (d) with all its bits, and the
// largest, 1, is still in range.  bf16 needs no scale.
template <typename T> constexpr float D_SCALE = 1.f;
template <> constexpr float D_SCALE<f16> = 32768.f;

// Results below 2^-126 are zero.
__device__ __forceinline__ float exp_(float x) { return __builtin_amdgcn_exp2f(x * LOG2E); }

__device__ __forceinline__ int64_t target_of(const void* p, int bytes, int64_t t) {
    return bytes == 8 ? static_cast<const int64_t*>(p)[t] : static_cast<const int32_t*>(p)[t];
}

// Up to so many tokens d is kept as a sum of two 16-bit numbers, of numerators in
// fp32: the rounding of d at the target, up to 2^-9 in bf16, averages out over
// many tokens, not over a few (5 tokens: the error of dw was 1.5 times its output's
// own rounding), and so short a product is bound by reading w.
constexpr int FINE = 64;

// ---- the first product ----------------------------------------------------

struct LogitArgs {
    Operand x, w;            // both along k = dim
    int n, rows, dim;
    const void* targets;
    int target_bytes;
    f32x2* stats;            // [piece][token]: maximum, sum
    float* target_logit;
    void* numer;             // [token][ld], or null
    int64_t ld;
    bool fine;               // numerators in fp32
    int tm, tn;
};

// Where dim is long (2048: 4.5 ms in a trace, 0.98 PFLOP/s) the matrix cores are busy
// 57% of a unit's cycles, at the 1.55 GHz that the card then runs at, with no LDS conflicts
// and 80% of the reads in L2; the rest is tiles' starts and ends and the meetings of
// a block's waves.  Where dim is short it is bound by its end, the numerators' stores
// most: 1003 tokens, 50001 rows of 520, bf16: 114 us, 89 without those stores (100 MB),
// 113 without the exponentials; the blocks of one round end together, so that stores do
// not run beside products.
template <typename P> __global__ __launch_bounds__(P::THREADS, P::THREADS / 256) void logit_kernel(LogitArgs a) {
    typedef typename P::T T;
    int ti, tj;
    fc::tile_place(fc::xcd_order(blockIdx.x, a.tm * a.tn), a.tm, a.tn, 4, ti, tj);
    P p;
    p.run(lds, a.x, a.w, ti * P::BM, tj * P::BN, 0, a.dim, 1);
    const int n0 = tj * P::BN + P::col(0);
    const int wn = (threadIdx.x >> 6) % (P::BN / P::WN), lane = threadIdx.x & 63;
    constexpr int SIDE = P::BN / P::WN;                            // waves that share a token
    float(*const part)[P::BM] = reinterpret_cast<float(*)[P::BM]>(lds);  // [SIDE][token of the tile]
    int* const target = reinterpret_cast<int*>(lds + sizeof(float) * SIDE * P::BM);  // in the tile's columns
    float tops[P::FM];
    __syncthreads();  // the tiles in LDS are done with
    if (threadIdx.x < P::BM) {
        const int m = ti * P::BM + threadIdx.x;
        const int64_t y = m < a.n ? target_of(a.targets, a.target_bytes, m) : -1;
        target[threadIdx.x] = y >= 0 && y < a.rows ? (int)y - tj * P::BN : -1;
    }
    if ((tj + 1) * P::BN > a.rows) {  // past the vocabulary's end: no weight in maxima and sums
#pragma unroll
        for (int j = 0; j < P::FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (n0 + 16 * j + e >= a.rows) {
#pragma unroll
                    for (int i = 0; i < P::FM; ++i) p.acc[i][j][e] = -__builtin_inff();
                }
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < P::FM; ++i) {
        const int m = ti * P::BM + P::row(i);
        const int at = target[P::row(i)] - P::col(0);
        float top = -__builtin_inff();
#pragma unroll
        for (int j = 0; j < P::FN; ++j)
#pragma unroll
            for (int e = 0; e < 4; ++e) top = fmaxf(top, p.acc[i][j][e]);
        if (__any(at >= 0 && at < P::WN)) {  // few tiles hold a target
#pragma unroll
            for (int j = 0; j < P::FN; ++j)
#pragma unroll
                for (int e = 0; e < 4; ++e)
                    if (at == 16 * j + e) a.target_logit[m] = p.acc[i][j][e];
        }
        top = fmaxf(top, __shfl_xor(top, 16));
        top = fmaxf(top, __shfl_xor(top, 32));
        tops[i] = top;
        if (lane < 16) part[wn][P::row(i)] = top;
        __builtin_amdgcn_sched_barrier(0);  // row by row: the registers hold no more
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < P::FM; ++i)
#pragma unroll
        for (int q = 0; q < SIDE; ++q) tops[i] = fmaxf(tops[i], part[q][P::row(i)]);
    __syncthreads();
#pragma unroll
    for (int i = 0; i < P::FM; ++i) {
        const int m = ti * P::BM + P::row(i);
        const bool keep = a.numer && m < a.n;
        const int64_t to = (int64_t)m * a.ld + n0;
        const float ref = tops[i] == -__builtin_inff() ? 0.f : tops[i];
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < P::FN; ++j) {
            f32x4 q;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                q[e] = exp_(p.acc[i][j][e] - ref);
                sum += q[e];
            }
            if (keep && n0 + 16 * j < a.ld) {
                if (P::BM <= FINE && a.fine)
                    *reinterpret_cast<f32x4*>(static_cast<float*>(a.numer) + to + 16 * j) = q;
                else
                    *reinterpret_cast<typename Half<T>::v4*>(static_cast<T*>(a.numer) + to + 16 * j) = __builtin_convertvector(q * D_SCALE<T>, typename Half<T>::v4);
            }
        }
        sum += __shfl_xor(sum, 16);
        sum += __shfl_xor(sum, 32);
        if (lane < 16) part[wn][P::row(i)] = sum;
        __builtin_amdgcn_sched_barrier(0);
    }
    __syncthreads();
#pragma unroll
    for (int i = 0; i < P::FM; ++i) {
        const int m = ti * P::BM + P::row(i);
        if (wn || lane >= 16 || m >= a.n) continue;
        float sum = 0.f;
#pragma unroll
        for (int q = 0; q < SIDE; ++q) sum += part[q][P::row(i)];
        a.stats[(int64_t)tj * a.n + m] = f32x2{tops[i], sum};
    }
}

// ---- a token's pieces joined ------------------------------------------------

struct JoinArgs {
    const f32x2* stats;
    const float* target_logit;
    const void* targets;
    int target_bytes;
    int n, rows, pieces;
    float* lse;
    int* row;                // the token's target, or -1
    float* loss;
};

// The sums of exponentials s and q, of what lies below their maxima, as one.
__device__ __forceinline__ f32x2 join(f32x2 s, f32x2 q) {
    const float m = fmaxf(s.x, q.x);
    if (!(m > -__builtin_inff())) return f32x2{m, s.y + q.y};
    return f32x2{m, s.y * exp_(s.x - m) + q.y * exp_(q.x - m)};
}

// T tokens per block of 256 threads, 256 / T threads each: 16 where there are
// enough tokens (a piece's stats of 16 tokens are neighbours), else 1.  24 tokens of
// 512 pieces take 4.5 us with 1 per block, 40 more with 16; 8192 tokens 25.
template <int T> __global__ __launch_bounds__(256) void join_kernel(JoinArgs a) {
    constexpr int Q = 256 / T;
    __shared__ f32x2 part[T][Q + 1];
    const int i = threadIdx.x % T, q = threadIdx.x / T;
    const int64_t t = (int64_t)blockIdx.x * T + i;
    f32x2 sum{-__builtin_inff(), 0.f};
    if (t < a.n) {
#pragma unroll 8
        for (int k = q; k < a.pieces; k += Q) sum = join(sum, a.stats[(int64_t)k * a.n + t]);
    }
    part[i][q] = sum;
#pragma unroll
    for (int half = Q / 2; half > 0; half /= 2) {
        __syncthreads();
        if (q < half) part[i][q] = sum = join(sum, part[i][q + half]);
    }
    if (q || t >= a.n) return;
    const int64_t y = target_of(a.targets, a.target_bytes, t);
    const bool real = y >= 0 && y < a.rows;
    const float lse = sum.x + logf(sum.y);
    if (a.lse) {
        a.lse[t] = lse;
        a.row[t] = real ? (int)y : -1;
    }
    a.loss[t] = real ? lse - a.target_logit[t] : 0.f;
}

// ---- numerators to d --------------------------------------------------------

struct DiffArgs {
    const void* numer;       // T, or fp32 where d has two halves
    void* d;                 // may be numer
    int64_t low;             // from a high half to its low one
    int64_t ld;
    int n;
    int width;               // of a piece
    int pieces;
    const f32x2* stats;
    const float* lse;
    const int* row;
};

constexpr int DIFF_ROWS = 8;

// A block's 256 threads hold 8 columns each, of DIFF_ROWS tokens one after the
// other, whose stats are neighbours in memory.  Bound by HBM: 8192 tokens of 131072
// rows 0.81 ms, 4.3 GB at 5.3 TB/s.
template <typename T, typename N> __global__ __launch_bounds__(256) void diff_kernel(DiffArgs a) {
    typedef typename Half<T>::v8 v8;
    typedef N n8 __attribute__((ext_vector_type(8)));
    const int64_t col = ((int64_t)blockIdx.x * 256 + threadIdx.x) * 8;
    if (col >= a.ld) return;
    const int piece = min((int)(col / a.width), a.pieces - 1);
    const int t0 = blockIdx.y * DIFF_ROWS;
    n8 x[DIFF_ROWS];
    float f[DIFF_ROWS];
    int row[DIFF_ROWS];
#pragma unroll
    for (int i = 0; i < DIFF_ROWS; ++i) {
        const int t = min(t0 + i, a.n - 1);
        x[i] = *reinterpret_cast<const n8*>(static_cast<const N*>(a.numer) + t * a.ld + col);
        row[i] = a.row[t];
        f[i] = exp_(a.stats[(int64_t)piece * a.n + t].x - a.lse[t]) * (sizeof(N) == 4 ? D_SCALE<T> : 1.f);  // 16-bit ones have the scale
    }
#pragma unroll
    for (int i = 0; i < DIFF_ROWS; ++i) {
        if (t0 + i >= a.n) break;
        v8 y, z;
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            float v = (float)x[i][e] * f[i];
            if (col + e == row[i]) v -= D_SCALE<T>;
            if (row[i] < 0) v = 0.f;
            y[e] = (T)v;
            z[e] = (T)(v - (float)y[e]);
        }
        T* const p = static_cast<T*>(a.d) + (t0 + i) * a.ld + col;
        *reinterpret_cast<v8*>(p) = y;
        if constexpr (sizeof(N) == 4) *reinterpret_cast<v8*>(p + a.low) = z;
    }
}

// ---- the gradients' products ------------------------------------------------

__device__ __forceinline__ void store_one(void* p, int dt, int64_t at, float v) {
    if (dt == FC_F32) static_cast<float*>(p)[at] = v;
    else if (dt == FC_F16) static_cast<f16*>(p)[at] = (f16)v;
    else static_cast<bf16*>(p)[at] = (bf16)v;
}

// Up to four neighbouring elements of a row, of which `left` are in it.
__device__ __forceinline__ void store_four(void* p, int dt, int64_t at, f32x4 v, int left) {
    if (left < 4) {
#pragma unroll
        for (int e = 0; e < 3; ++e)
            if (e < left) store_one(p, dt, at + e, v[e]);
    } else if (dt == FC_F32) {
        *reinterpret_cast<fc::f32x4_any*>(static_cast<float*>(p) + at) = v;
    } else if (dt == FC_F16) {
        *reinterpret_cast<fc::f16x4_any*>(static_cast<f16*>(p) + at) = __builtin_convertvector(v, fc::f16x4);
    } else {
        *reinterpret_cast<fc::b16x4_any*>(static_cast<bf16*>(p) + at) = __builtin_convertvector(v, fc::b16x4);
    }
}

struct GradArgs {
    Operand a, b;
    int m, n, k;             // of the product
    int kper;                // of one split, a multiple of 64
    int parts;               // 2: a has two halves
    float scale;
    const int* row;          // per m: below 0, the result is zero; or null
    void* out;
    int dt;
    int64_t ld;
    float* sum;              // fp32 sums over calls or splits, [split][m][n], or null
    bool first, last;        // of the calls that add to `sum`
    int tm, tn;
};

// 8192 tokens, 131072 rows of 2048 take 3.8 ms for dx and 4.3 for dw in a trace (1.17 and
// 1.02 PFLOP/s): the matrix cores are busy 69% and 60% of a unit's cycles, at 1.54 and 1.66
// GHz.  Tiles in groups of 8 rows keep what the blocks of an XCD read in its L2 (80% hits).
// Few tokens give few tiles: k is then split.
template <typename P> __global__ __launch_bounds__(P::THREADS, P::THREADS / 256) void grad_kernel(GradArgs a) {
    int ti, tj;
    fc::tile_place(fc::xcd_order(blockIdx.x, a.tm * a.tn), a.tm, a.tn, 8, ti, tj);
    const int kb = blockIdx.y * a.kper, ke = min(a.k, kb + a.kper);
    P p;
    p.run(lds, a.a, a.b, ti * P::BM, tj * P::BN, kb, ke, a.parts);
    float* const sum = a.sum ? a.sum + (int64_t)blockIdx.y * a.m * a.n : nullptr;
    // Results go through LDS by strips of 16 rows, so that a row's neighbours are
    // stored by neighbouring lanes, whatever its start's alignment.
    float(*const part)[P::WN + 4] = reinterpret_cast<float(*)[P::WN + 4]>(lds + (threadIdx.x >> 6) * 16 * (P::WN + 4) * sizeof(float));
    static_assert(P::WAVES * 16 * (P::WN + 4) * sizeof(float) <= P::LDS, "the strips of all waves fit");
    const int lane = threadIdx.x & 63, n0 = tj * P::BN + P::col(0) - 4 * (lane >> 4);
    __syncthreads();  // the tiles in LDS are done with
#pragma unroll
    for (int i = 0; i < P::FM; ++i) {
        const int m0 = ti * P::BM + P::row(i) - (lane & 15);
#pragma unroll
        for (int j = 0; j < P::FN; ++j) *reinterpret_cast<f32x4*>(part[lane & 15] + 16 * j + 4 * (lane >> 4)) = p.acc[i][j];
        __builtin_amdgcn_wave_barrier();
#pragma unroll 2
        for (int k = lane; k < 16 * P::WN / 4; k += 64) {
            const int y = k / (P::WN / 4), z = k % (P::WN / 4) * 4, m = m0 + y, left = a.n - n0 - z;
            if (m >= a.m || left <= 0) continue;
            f32x4 v = *reinterpret_cast<const f32x4*>(part[y] + z);
            if (sum) {
                float* const s = sum + (int64_t)m * a.n + n0 + z;
                if (!a.first) {
#pragma unroll
                    for (int e = 0; e < 4; ++e) v[e] += s[min(e, left - 1)];
                }
                if (!a.last) {
                    store_four(s, FC_F32, 0, v, left);
                    continue;
                }
            }
            store_four(a.out, a.dt, (int64_t)m * a.ld + n0 + z, a.row && a.row[m] < 0 ? f32x4{0.f, 0.f, 0.f, 0.f} : a.scale * v, left);
        }
        __builtin_amdgcn_wave_barrier();
        __builtin_amdgcn_sched_barrier(0);
    }
}

struct SplitArgs {
    const float* sum;
    int splits, m, n;
    float scale;
    const int* row;
    void* out;
    int dt;
    int64_t ld;
};

// The splits of a product added in order: 4 to 7 us, a launch's latency and one
// trip to memory.
__global__ __launch_bounds__(256) void split_kernel(SplitArgs a) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x, total = (int64_t)a.m * a.n;
    if (i >= total) return;
    const int m = (int)(i / a.n), n = (int)(i % a.n);
    float v = 0.f;
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) v += a.sum[s * total + i];
    store_one(a.out, a.dt, (int64_t)m * a.ld + n, a.row && a.row[m] < 0 ? 0.f : v * a.scale);
}

// Copies with rows of a multiple of 8 elements: bound by HBM (8192 x 2048, 67 MB in
// all, 16 us).
struct PackArgs {
    const void* in;
    int64_t ld_in;
    void* out;
    int64_t ld_out;          // a multiple of 8; the elements past the row's length are zeros
    int64_t rows;
    int len;
    const void* targets;     // or null: rows without a target become zeros
    int target_bytes;
    int targets_below;
};

__global__ __launch_bounds__(256) void pack_kernel(PackArgs a) {
    typedef unsigned short u16;
    const int per_row = (int)(a.ld_out / 8);
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    const int64_t r = i / per_row;
    const int c = (int)(i % per_row) * 8;
    if (r >= a.rows) return;
    bool keep = true;
    if (a.targets) {
        const int64_t y = target_of(a.targets, a.target_bytes, r);
        keep = y >= 0 && y < a.targets_below;
    }
    typedef u16 u16x8 __attribute__((ext_vector_type(8)));
    typedef u16x8 u16x8_any __attribute__((aligned(2)));
    const u16* in = static_cast<const u16*>(a.in) + r * a.ld_in + c;
    u16x8 v{};
    if (keep && c + 8 <= a.len) {
        v = *reinterpret_cast<const u16x8_any*>(in);
    } else if (keep) {
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (c + e < a.len) v[e] = in[e];
    }
    *reinterpret_cast<u16x8*>(static_cast<u16*>(a.out) + r * a.ld_out + c) = v;
}

// Tiles by size; BROAD is for the gradients, where dim is often just above a multiple
// of 256 or fills the chip's rounds better so (the first product's tiles end with more
// work: 1003 tokens, 50001 rows of 520 took 122 us with it, 119 with LARGE; dx 74, 104
// with MIDDLE; 8192 tokens, 8192 rows of 1280 in all 565, 657).  The estimate is not always
// right: for dw of the 1003 tokens it takes MIDDLE (115 us in a trace, the whole call 355
// to 360), with which BROAD's call takes 341 to 350.  SHORT and NARROW are for up to 64
// tokens, which are bound by reading w: a compute unit reads at most about 50 GB/s, so
// that few rows of w are read faster by more blocks.
template <typename T, bool AS, bool BS> using Large = fc::Product<T, 256, 256, 128, 64, AS, BS>;
template <typename T, bool AS, bool BS> using Broad = fc::Product<T, 256, 192, 128, 48, AS, BS>;
template <typename T, bool AS, bool BS> using Middle = fc::Product<T, 128, 128, 64, 64, AS, BS>;
template <typename T, bool AS, bool BS> using Short = fc::Product<T, 64, 128, 64, 32, AS, BS, 3>;
template <typename T, bool AS, bool BS> using Narrow = fc::Product<T, 64, 32, 16, 32, AS, BS, 6>;
template <typename T, bool AS, bool BS> using Once = fc::Product<T, 64, 128, 64, 32, AS, BS, 3, 0, true>;

enum TileKind { LARGE, BROAD, MIDDLE, SHORT, NARROW, KINDS };

constexpr int CUS = 256;

// In us, measured with 1 to 512 tiles: a step of 64 of k with the compute unit full
// of such tiles (`per` at a time) and alone, and a tile's start and end.
struct KindCost {
    int bm, bn;
    double full, alone, once;
    int per;
};
constexpr KindCost COST[KINDS] = {{256, 256, 1.7, 1.15, 9.5, 1}, {256, 192, 1.38, 1.0, 8.0, 1}, {128, 128, 0.52, 0.6, 5.0, 2}, {64, 128, 0.55, 0.6, 4.0, 2}, {64, 32, 0.2, 0.3, 4.0, 2}};

struct Choice {
    TileKind kind;
    int splits;      // parts of k, of `steps` of 64 each
    int steps;
};

constexpr int64_t SPLIT_FLOATS = (int64_t)1 << 27;

// The tiles of an m x n product over k, and the parts k is split into, by the
// least estimated time; m and k are taken up to multiples of 64, so that the
// choice is one for every list of as many 64s of tokens.
Choice choose(int64_t m, int64_t n, int64_t k, bool few, bool may_split, bool broad) {
    m = fc::ceil_div(m, 64) * 64;
    const int64_t total = fc::ceil_div(k, fc::GEMM_BK);
    Choice best{MIDDLE, 1, (int)total};
    double least = 1e300;
    for (int kind = few ? SHORT : LARGE; kind <= (few ? NARROW : MIDDLE); ++kind) {
        if (kind == BROAD && !broad) continue;
        const KindCost& c = COST[kind];
        const int64_t tiles = fc::ceil_div(m, c.bm) * fc::ceil_div(n, c.bn);
        const int fill = (int)std::min<int64_t>(64, CUS * c.per / tiles);  // as many as the chip takes at once
        for (int s : {1, 2, 3, 4, 6, 8, 12, 16, 24, 32, 48, 64, fill}) {
            if (s < 1) continue;
            const int64_t steps = fc::ceil_div(total, s), parts = fc::ceil_div(total, steps), blocks = tiles * parts;
            if (s > 1 && (!may_split || steps < 2 || parts * m * n > SPLIT_FLOATS)) continue;
            const double at_once = (double)std::min<int64_t>(c.per, fc::ceil_div(blocks, CUS));
            double t = fc::ceil_div(blocks, CUS * c.per) * (steps * std::max(c.alone, c.full * at_once) + c.once);
            if (parts > 1) t += 5.0 + 8.0 * parts * m * n / 4.5e6;  // partial sums, written and read
            if (t < least) {
                least = t;
                best = {(TileKind)kind, (int)parts, (int)steps};
            }
        }
    }
    return best;
}

template <typename P> hipError_t prepare(const void* kernel) {
    return P::LDS > 64 * 1024 ? hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS) : hipSuccess;
}

template <typename P> void launch_logit(LogitArgs a, hipStream_t s) {
    a.tm = (int)fc::ceil_div(a.n, P::BM);
    a.tn = (int)fc::ceil_div(a.rows, P::BN);
    logit_kernel<P><<<a.tm * a.tn, P::THREADS, P::LDS, s>>>(a);
}

template <typename P> void launch_grad(GradArgs a, hipStream_t s) {
    a.tm = (int)fc::ceil_div(a.m, P::BM);
    a.tn = (int)fc::ceil_div(a.n, P::BN);
    grad_kernel<P><<<dim3(a.tm * a.tn, (unsigned)fc::ceil_div(a.k, a.kper)), P::THREADS, P::LDS, s>>>(a);
}

template <typename T> hipError_t prepare_all() {
    for (hipError_t e : {prepare<Large<T, false, false>>((const void*)logit_kernel<Large<T, false, false>>),
                         prepare<Middle<T, false, false>>((const void*)logit_kernel<Middle<T, false, false>>),
                         prepare<Short<T, false, false>>((const void*)logit_kernel<Short<T, false, false>>),
                         prepare<Narrow<T, false, false>>((const void*)logit_kernel<Narrow<T, false, false>>),
                         prepare<Once<T, false, false>>((const void*)logit_kernel<Once<T, false, false>>),
                         prepare<Large<T, false, true>>((const void*)grad_kernel<Large<T, false, true>>),
                         prepare<Broad<T, false, true>>((const void*)grad_kernel<Broad<T, false, true>>),
                         prepare<Broad<T, true, true>>((const void*)grad_kernel<Broad<T, true, true>>),
                         prepare<Middle<T, false, true>>((const void*)grad_kernel<Middle<T, false, true>>),
                         prepare<Short<T, false, true>>((const void*)grad_kernel<Short<T, false, true>>),
                         prepare<Narrow<T, false, true>>((const void*)grad_kernel<Narrow<T, false, true>>),
                         prepare<Once<T, false, true>>((const void*)grad_kernel<Once<T, false, true>>),
                         prepare<Large<T, true, true>>((const void*)grad_kernel<Large<T, true, true>>),
                         prepare<Middle<T, true, true>>((const void*)grad_kernel<Middle<T, true, true>>)})
        if (e != hipSuccess) return e;
    return hipSuccess;
}

// Columns of the first product's tiles, a piece of the vocabulary.
int piece_width(TileKind k) { return COST[k].bn; }

// The choices of the three products for m tokens.
Choice logit_choice(int64_t m, int64_t rows, int64_t dim) { return choose(m, rows, dim, m <= 64, false, false); }
Choice dx_choice(int64_t m, int64_t rows, int64_t dim) { return choose(m, dim, rows, m <= 64, true, true); }
Choice dw_choice(int64_t m, int64_t rows, int64_t dim, bool one_chunk) { return choose(rows, dim, m, false, one_chunk, true); }

constexpr int64_t ROWS_LIMIT = 1 << 21, LD_LIMIT = 1 << 21, TOKENS_LIMIT = (int64_t)1 << 31;
// A w well beyond the memory-side cache (256 MB) is read past the caches (up to 64
// tokens, when every tile of it is read once): from the size on at which that is
// faster or as fast whether the caches hold something else or the end of w.  16
// tokens, fp16, rows of 2048, us, past the caches / through them, first with 1 GB read
// between the calls, then call after call:
//   w of   losses alone     with dx, which reads w again
//   134 MB 39/42   36/28    92/91   91/77
//   268 MB 65/70   62/47   162/160 160/136
//   302 MB 79/83   77/75   185/187 182/163
//   336 MB 80/86   78/84   198/200 195/182
//   403 MB 99/104  94/103  248/254 246/234
//   537 MB 121/129 118/129 319/335 316/321
// (Where the caches hold 1 GB of results not yet written, 268 MB take 65 / 125.)
constexpr int64_t CACHE_BYTES = (int64_t)5 << 26, CACHE_BYTES_DX = (int64_t)1 << 29;
constexpr int64_t NUMER_BYTES = (int64_t)4 << 30;
constexpr int64_t CHUNK_LIMIT = 1 << 18;  // a launch has at most 65535 blocks along y, of 8 tokens each

}  // namespace

struct fc_xent {
    fc::CallOrder order;
    fc::DeviceBlock block;
    int64_t rows = 0, dim = 0, max_tokens = 0;
    int dtype = FC_F16;
    int64_t chunk = 0;       // tokens that go through together
    int64_t ld = 0;          // of the numerators
    int64_t ldp = 0;         // of packed x and w
    bool pack = false;       // dim is not a multiple of 8: x and w go through packed copies
    char* numer = nullptr;
    char* fine = nullptr;    // numerators in fp32, of up to FINE tokens
    f32x2* stats = nullptr;
    float* target_logit = nullptr;
    float* lse = nullptr;
    int* row = nullptr;
    char* x = nullptr;
    char* w = nullptr;
    float* sum = nullptr;    // splits of dx
    float* dw = nullptr;     // dw over chunks
};

namespace {

template <typename T>
int run(fc_xent* p, const void* x, int64_t ldx, const void* w, int64_t ldw, const void* targets, int target_bytes, int64_t n,
        float scale, float* loss, void* dx, int xdt, int64_t lddx, void* dw, int wdt, int64_t lddw, hipStream_t s) {
    const bool grads = dx || dw;
    auto join_splits = [&](const GradArgs& g, int splits) {
        SplitArgs q{g.sum, splits, g.m, g.n, g.scale, g.row, g.out, g.dt, g.ld};
        split_kernel<<<(unsigned)fc::ceil_div((int64_t)g.m * g.n, 256), 256, 0, s>>>(q);
    };
    auto pack = [&](const void* in, int64_t ld, void* out, int64_t rows, const void* mask) {
        fc::by_launches(rows, p->ldp / 8, [&](int64_t r0, int64_t count) {
            PackArgs a{static_cast<const char*>(in) + r0 * ld * 2, ld, static_cast<char*>(out) + r0 * p->ldp * 2, p->ldp, count, (int)p->dim,
                       mask ? static_cast<const char*>(mask) + r0 * target_bytes : nullptr, target_bytes, (int)p->rows};
            pack_kernel<<<(unsigned)fc::ceil_div(count * (p->ldp / 8), 256), 256, 0, s>>>(a);
        });
    };
    if (p->pack) {
        pack(w, ldw, p->w, p->rows, nullptr);
        w = p->w;
        ldw = p->ldp;
    }
    const int dimk = (int)(p->pack ? p->ldp : p->dim);
    const bool once = p->rows * dimk * 2 >= (dx ? CACHE_BYTES_DX : CACHE_BYTES);
    for (int64_t t0 = 0; t0 < n; t0 += p->chunk) {
        const int m = (int)std::min(p->chunk, n - t0);
        const void* xt = static_cast<const char*>(x) + t0 * ldx * 2;
        const void* yt = static_cast<const char*>(targets) + t0 * target_bytes;
        // dw's product must not meet what padding's rows hold (0 * NaN)
        if (p->pack || dw) pack(xt, ldx, p->x, m, yt);
        const Operand ox{p->pack || dw ? p->x : xt, p->pack || dw ? p->ldp : ldx, m, dimk, 0};
        const Operand ow{w, ldw, (int)p->rows, dimk, 0};
        const TileKind kind = logit_choice(m, p->rows, dimk).kind;
        const bool fine = m <= FINE;
        LogitArgs l{ox, ow, m, (int)p->rows, dimk, yt, target_bytes, p->stats, p->target_logit, grads ? fine ? p->fine : p->numer : nullptr, p->ld, fine, 0, 0};
        if (kind == LARGE) launch_logit<Large<T, false, false>>(l, s);
        else if (kind == MIDDLE) launch_logit<Middle<T, false, false>>(l, s);
        else if (kind == SHORT && once) launch_logit<Once<T, false, false>>(l, s);
        else if (kind == SHORT) launch_logit<Short<T, false, false>>(l, s);
        else launch_logit<Narrow<T, false, false>>(l, s);
        const int width = piece_width(kind), pieces = (int)fc::ceil_div(p->rows, width);
        JoinArgs j{p->stats, p->target_logit, yt, target_bytes, m, (int)p->rows, pieces, p->lse, p->row, loss + t0};
        if (m >= 16 * CUS) join_kernel<16><<<(unsigned)fc::ceil_div(m, 16), 256, 0, s>>>(j);
        else join_kernel<1><<<(unsigned)m, 256, 0, s>>>(j);
        if (!grads) continue;
        const int64_t low = m * p->ld;
        DiffArgs d{fine ? p->fine : p->numer, p->numer, low, p->ld, m, width, pieces, p->stats, p->lse, p->row};
        const dim3 grid((unsigned)fc::ceil_div(p->ld, 2048), (unsigned)fc::ceil_div(m, DIFF_ROWS));
        if (fine) diff_kernel<T, float><<<grid, 256, 0, s>>>(d);
        else diff_kernel<T, T><<<grid, 256, 0, s>>>(d);
        const float back = scale / D_SCALE<T>;
        if (dx) {
            GradArgs g{};
            // past the last row's 8 columns the first product's tiles may end
            g.a = Operand{p->numer, p->ld, m, (int)fc::ceil_div(p->rows, 8) * 8, low};
            g.parts = fine ? 2 : 1;
            g.b = Operand{w, ldw, (int)p->dim, (int)p->rows, 0};
            g.m = m;
            g.n = (int)p->dim;
            g.k = (int)p->rows;
            const Choice c = dx_choice(m, p->rows, p->dim);
            g.kper = c.steps * fc::GEMM_BK;
            g.scale = back;
            g.row = p->row;
            g.dt = xdt;
            g.out = static_cast<char*>(dx) + t0 * lddx * fc::dtype_bytes(xdt);
            g.ld = lddx;
            g.sum = c.splits > 1 ? p->sum : nullptr;
            g.first = true;
            g.last = c.splits == 1;
            if (c.kind == LARGE) launch_grad<Large<T, false, true>>(g, s);
            else if (c.kind == BROAD) launch_grad<Broad<T, false, true>>(g, s);
            else if (c.kind == MIDDLE) launch_grad<Middle<T, false, true>>(g, s);
            else if (c.kind == SHORT && once) launch_grad<Once<T, false, true>>(g, s);
            else if (c.kind == SHORT) launch_grad<Short<T, false, true>>(g, s);
            else launch_grad<Narrow<T, false, true>>(g, s);
            if (c.splits > 1) join_splits(g, c.splits);
        }
        if (dw) {
            GradArgs g{};
            g.a = Operand{p->numer, p->ld, (int)p->rows, m, low};
            g.parts = fine ? 2 : 1;
            g.b = Operand{p->x, p->ldp, (int)p->dim, m, 0};
            g.m = (int)p->rows;
            g.n = (int)p->dim;
            g.k = m;
            const Choice c = dw_choice(m, p->rows, p->dim, n <= p->chunk);
            g.kper = c.steps * fc::GEMM_BK;
            g.scale = back;
            g.out = dw;
            g.dt = wdt;
            g.ld = lddw;
            g.sum = n > p->chunk ? p->dw : c.splits > 1 ? p->sum : nullptr;
            g.first = t0 == 0;
            g.last = c.splits == 1 && t0 + p->chunk >= n;
            if (c.kind == LARGE) launch_grad<Large<T, true, true>>(g, s);
            else if (c.kind == BROAD) launch_grad<Broad<T, true, true>>(g, s);
            else launch_grad<Middle<T, true, true>>(g, s);
            if (c.splits > 1) join_splits(g, c.splits);
        }
    }
    return fc::hip_code(hipGetLastError());
}

// Zeros for a gradient without tokens.
__global__ __launch_bounds__(256) void zero_kernel(void* p, int dt, int64_t rows, int64_t len, int64_t ld) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < rows * len) store_one(p, dt, i / len * ld + i % len, 0.f);
}

int call(fc_xent* p, const void* x, int64_t ldx, const void* w, int64_t ldw, const void* targets, int target_bytes, int64_t n,
         float scale, float* loss, void* dx, int xdt, int64_t lddx, void* dw, int wdt, int64_t lddw, hipStream_t s) {
    if (!p || n < 0 || n > p->max_tokens || (target_bytes != 4 && target_bytes != 8)) return FC_EINVAL;
    if (ldx > LD_LIMIT || ldw > LD_LIMIT) return FC_EINVAL;
    const fc::Span none{nullptr, 0, 0, 0, 1, false};
    int rc = fc::check_spans({{x, n, p->dim, ldx, 2, false},
                              {w, p->rows, p->dim, ldw, 2, false},
                              {targets, 1, n, n, target_bytes, false},
                              {loss, 1, n, n, 4, true},
                              dx ? fc::Span{dx, n, p->dim, lddx, fc::dtype_bytes(xdt), true} : none,
                              dw ? fc::Span{dw, p->rows, p->dim, lddw, fc::dtype_bytes(wdt), true} : none});
    if (rc) return rc;
    // rows of whole 16-byte vectors, unless they are copied anyway
    if (!p->pack && (ldx % 8 || ldw % 8 || reinterpret_cast<uintptr_t>(x) % 16 || reinterpret_cast<uintptr_t>(w) % 16)) return FC_EALIGN;
    bool note;
    rc = p->order.begin(s, note);
    if (rc) return rc;
    if (n == 0) {
        if (dw)
            fc::by_launches(p->rows, p->dim, [&](int64_t r0, int64_t count) {
                zero_kernel<<<(unsigned)fc::ceil_div(count * p->dim, 256), 256, 0, s>>>(static_cast<char*>(dw) + r0 * lddw * fc::dtype_bytes(wdt), wdt,
                                                                                        count, p->dim, lddw);
            });
        rc = fc::hip_code(hipGetLastError());
    } else if (p->dtype == FC_F16) {
        rc = run<f16>(p, x, ldx, w, ldw, targets, target_bytes, n, scale, loss, dx, xdt, lddx, dw, wdt, lddw, s);
    } else {
        rc = run<bf16>(p, x, ldx, w, ldw, targets, target_bytes, n, scale, loss, dx, xdt, lddx, dw, wdt, lddw, s);
    }
    p->order.done(s, note);
    return rc;
}

}  // namespace

extern "C" {

int fc_xent_create(fc_xent** plan, int64_t rows, int64_t dim, int64_t max_tokens, int dtype, int64_t chunk_tokens) {
    if (!plan) return FC_EINVAL;
    *plan = nullptr;
    if (rows < 1 || dim < 1 || max_tokens < 0 || rows > ROWS_LIMIT || dim > LD_LIMIT || max_tokens >= TOKENS_LIMIT ||
        chunk_tokens < 0 || (dtype != FC_F16 && dtype != FC_BF16))
        return FC_EINVAL;
    return fc::no_throw([&] {
        fc_xent* p = new fc_xent;
        p->rows = rows;
        p->dim = dim;
        p->max_tokens = max_tokens;
        p->dtype = dtype;
        p->ld = fc::ceil_div(rows, 64) * 64;
        p->ldp = fc::ceil_div(dim, 8) * 8;
        p->pack = dim % 8 != 0;
        int64_t most = NUMER_BYTES / (2 * p->ld);
        most = std::min<int64_t>(std::max<int64_t>(256, most / 256 * 256), CHUNK_LIMIT);
        if (chunk_tokens) most = std::min<int64_t>(most, chunk_tokens);
        p->chunk = std::max<int64_t>(1, std::min(most, max_tokens));
        const int64_t c = p->chunk;
        const int64_t stats = std::max(c * fc::ceil_div(rows, 128), std::min(c, (int64_t)64) * fc::ceil_div(rows, 32));
        int64_t sums = 0;  // of the most splits of any number of tokens up to c
        for (int64_t m = 64; m < c + 64; m += 64) {
            const Choice x = dx_choice(m, rows, dim), w = dw_choice(m, rows, dim, true);
            if (x.splits > 1) sums = std::max(sums, x.splits * std::min(m, c) * dim);
            if (w.splits > 1) sums = std::max(sums, w.splits * rows * dim);
        }
        fc::Layout at;
        const int64_t few = std::min<int64_t>(c, FINE);
        const uint64_t o_numer = at.take(std::max(c, 2 * few) * p->ld * 2), o_fine = at.take(few * p->ld * 4), o_stats = at.take(stats * 8), o_logit = at.take(c * 4),
                       o_lse = at.take(c * 4), o_row = at.take(c * 4), o_x = at.take(c * p->ldp * 2),
                       o_w = at.take(p->pack ? rows * p->ldp * 2 : 0), o_sum = at.take(sums * 4),
                       o_dw = at.take(max_tokens > c ? rows * dim * 4 : 0);
        int rc = p->order.create();
        if (!rc) rc = fc::hip_code(dtype == FC_F16 ? prepare_all<f16>() : prepare_all<bf16>());
        if (!rc) rc = p->block.create(at.size);
        if (rc) {
            fc_xent_destroy(p);
            return rc;
        }
        char* b = p->block.p;
        p->numer = b + o_numer;
        p->fine = b + o_fine;
        p->stats = reinterpret_cast<f32x2*>(b + o_stats);
        p->target_logit = reinterpret_cast<float*>(b + o_logit);
        p->lse = reinterpret_cast<float*>(b + o_lse);
        p->row = reinterpret_cast<int*>(b + o_row);
        p->x = b + o_x;
        p->w = b + o_w;
        p->sum = reinterpret_cast<float*>(b + o_sum);
        p->dw = reinterpret_cast<float*>(b + o_dw);
        *plan = p;
        return FC_OK;
    });
}

void fc_xent_destroy(fc_xent* p) {
    if (!p) return;
    p->block.destroy();
    p->order.destroy();
    delete p;
}

int fc_xent_loss(fc_xent* p, const void* x, int64_t ld_x, const void* w, int64_t ld_w, const void* targets, int token_bytes,
                 int64_t n, float* loss, void* stream) {
    return fc::no_throw([&] {
        return call(p, x, ld_x, w, ld_w, targets, token_bytes, n, 1.f, loss, nullptr, 0, 0, nullptr, 0, 0,
                    static_cast<hipStream_t>(stream));
    });
}

int fc_xent_loss_grad(fc_xent* p, const void* x, int64_t ld_x, const void* w, int64_t ld_w, const void* targets,
                      int token_bytes, int64_t n, float scale, float* loss, void* dx, int dx_dtype, int64_t ld_dx, void* dw,
                      int dw_dtype, int64_t ld_dw, void* stream) {
    return fc::no_throw([&] {
        return call(p, x, ld_x, w, ld_w, targets, token_bytes, n, scale, loss, dx, dx_dtype, ld_dx, dw, dw_dtype, ld_dw,
                    static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
