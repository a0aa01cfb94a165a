// Norms before and after a block, with its gate and residual scale (fc_lm.h).
//
//   N(x) = (x - m) r, m = mean(x) or 0, r = 1 / sqrt(mean((x - m)^2) + eps)
//   out = h + s a(g) w N(b),  y = w2 N(out)
// backward, u = w2 dy, xh = N(out), bh = N(b):
//   do = dout + r (u - mean(u) [where m is a mean] - xh mean(u xh)),  dh = do
//   e = s do, q = e a(g), v = w q
//   db = r_b (v - mean(v) [same] - bh mean(v bh)),  dg = e a'(g) w bh
//   dw = sum over tokens of q bh,  dw2 = sum of dy xh
//
// A few operations for each element, so that memory bounds all of it: every matrix is read
// once and written once.  A row's elements stay in registers from its loads to its stores,
// and the statistics are taken anew from them in the backward pass, so that the forward pass
// keeps none.  Sums, statistics and everything between loads and stores are fp32; one
// rounding to the stored type, and y is of `out` as it was rounded.  The sums over tokens are
// kept by blocks that go through their share of the rows; their partial sums go through
// memory, and a second launch adds them in order.  Where the gate is a vector or none, a(g)
// and w are the same for all tokens, so that one sum, P = sum of e bh, gives both
// dw = a(g) P and dg = a'(g) w P.
//
// Measured, forward (out and y) and backward (all gradients): 16384 rows of 4096, bf16 and a
// residual in fp32, 805 MB, 164 to 167 us or 4.9 TB/s; 16384 rows of 2048, all bf16, with the gate
// a matrix, 537 MB, 125 us or 4.3 TB/s, where a copy of 4 GiB reaches 4.8.  One row of 4096
// forward 3.9 us, and 1003 rows of 1001 backward 14.3 (14.4 to 15.2 in a graph), of which 11.8 are the
// first launch and 4.0 the second by themselves and 4 the bytes' time.
#include <algorithm>
#include <type_traits>

#include "fc_eight.h"
#include "fc_lm_host.h"

namespace {

typedef _Float16 f16;
typedef __bf16 bf16;
typedef float f32x4 __attribute__((ext_vector_type(4)));
using fc::f32x8;
using fc::load8;
using fc::put8;
using fc::raw8;
using fc::store8;

// A channel vector's elements from c on; 1 where there is no vector.
__device__ __forceinline__ f32x8 channels(const float* p, int c, int left) {
    if (!p) return f32x8{1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f, 1.f};
    return load8(p + c, left);
}

// s = 1 / (1 + exp(-g)) and 1 - s, both from t = exp(-|g|), so that neither is a difference:
// relative to themselves to 2^-20 (0 where t is below 2^-126).  FINE keeps the exponential's
// argument to twice fp32's bits, since its rounding is up to 1.5 |g| 2^-24 of t; a 16-bit
// gate's results are rounded far above that (2^-16 at the most), and the operations would show:
// 16384 rows of 2048, bf16, gradients with a gate per token 130 us with them, 127 without.
template <bool FINE> __device__ __forceinline__ void sigmoid(float g, float& s, float& rest) {
    constexpr float L = 1.44269504088896341f, LOW = (float)(1.44269504088896340736 - (double)L);  // log2(e)
    float t;
    if constexpr (FINE) {
        const float m = fabsf(g) > 128.f ? 128.f : fabsf(g);  // a NaN stays, an infinity has no low part
        const float high = m * -L, low = __builtin_fmaf(m, -L, -high) - m * LOW;
        t = __builtin_amdgcn_exp2f(high);
        t = __builtin_fmaf(t, low * 0.693147180559945309f, t);
    } else {
        t = __builtin_amdgcn_exp2f(fabsf(g) * -L);
    }
    const float near = __builtin_amdgcn_rcpf(1.f + t), far = t * near;
    s = g < 0.f ? far : near;
    rest = g < 0.f ? near : far;
}

// Of a gate kept in T.
template <typename T> __device__ __forceinline__ float gate_value(float g, int kind) {
    if (kind == FC_GATE_NONE) return g;
    float s, rest;
    sigmoid<sizeof(T) == 4>(g, s, rest);
    return kind == FC_GATE_SIGMOID ? s : g * s;
}

// a(g) and a'(g).
template <typename T> __device__ __forceinline__ void gate_both(float g, int kind, float& a, float& slope) {
    if (kind == FC_GATE_NONE) {
        a = g;
        slope = 1.f;
        return;
    }
    float s, rest;
    sigmoid<sizeof(T) == 4>(g, s, rest);
    a = kind == FC_GATE_SIGMOID ? s : g * s;
    slope = kind == FC_GATE_SIGMOID ? s * rest : s * (1.f + g * rest);
}

// ---- how a row lies on threads -------------------------------------------------

// `lanes` threads hold a row, VECTORS times 8 elements each, a vector's neighbours in
// neighbouring threads: 8 to 64 lanes of a wave, with several rows to a block of 256, or
// a block of whole waves for one row.  Rows of more than 8192 elements take two or four vectors
// to a thread: at 9216 two, 9 waves, take 113 us forward and 327 backward where four, 5 waves,
// took 159 and 495 (3640 rows, 16 bits).  Rows of fewer than 8 elements go as they do.
struct Shape {
    int lanes, vectors, threads;
    int groups;  // rows to a block of the backward pass
};

constexpr int DIM_LIMIT = 16384;
constexpr int BLOCK = 256;  // threads of a backward pass's blocks, where a row takes no more
constexpr int MIDDLE = 640;  // threads of rows of two vectors each, at most

Shape shape_of(int64_t dim) {
    if (dim < 8) return {64, 2, 64, 1};
    if (dim <= 512) {
        int lanes = 8;
        while (lanes * 8 < dim) lanes *= 2;
        return {lanes, 1, 256, BLOCK / lanes};
    }
    const int vectors = dim <= 8192 ? 1 : dim <= 1024 * MIDDLE / 64 ? 2 : 4, threads = (int)fc::ceil_div(dim, 512 * vectors) * 64;
    return {threads, vectors, threads, vectors > 1 ? 1 : std::max(1, BLOCK / threads)};
}

// Sums over a row's lanes, N at once, the same in every lane.  Rows of several waves go
// through LDS, where a block meets once per call; the parts of one call and the next lie in
// different places, and a thread that writes a place again has met the others since they
// read it.
constexpr int WAVES = 16;

// A sum over 8, 16, 32 or 64 neighbouring lanes, without a trip through LDS: within a row of
// 16 lanes by its permutations, of which the mirrors pair what is already the same in 4 or 8
// lanes, beyond by exchanges of rows.
__device__ __forceinline__ float sum_lanes(float v, int lanes) {
    auto from = [&](auto control) __attribute__((always_inline)) {
        return __builtin_bit_cast(float, __builtin_amdgcn_update_dpp(0, __builtin_bit_cast(int, v), decltype(control)::value, 0xf, 0xf, true));
    };
    v += from(std::integral_constant<int, 0xb1>{});    // lanes 1, 0, 3, 2 of 4
    v += from(std::integral_constant<int, 0x4e>{});    // lanes 2, 3, 0, 1 of 4
    v += from(std::integral_constant<int, 0x141>{});   // 8 lanes mirrored
    if (lanes > 8) v += from(std::integral_constant<int, 0x140>{});  // 16 lanes mirrored
    if (lanes > 16) {
        const auto both = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        const uint32_t lo = both[0], hi = both[1];
        v = __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
    }
    if (lanes > 32) {
        const auto both = __builtin_amdgcn_permlane32_swap(__builtin_bit_cast(uint32_t, v), __builtin_bit_cast(uint32_t, v), false, false);
        const uint32_t lo = both[0], hi = both[1];
        v = __builtin_bit_cast(float, lo) + __builtin_bit_cast(float, hi);
    }
    return v;
}

template <int N> struct RowSums {
    float (*part)[N][WAVES];  // [2]
    int lanes, turn;
    __device__ __forceinline__ void add(float (&v)[N]) {
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = sum_lanes(v[k], lanes);
        if (lanes <= 64) return;
        const int wave = threadIdx.x >> 6, waves = lanes >> 6, first = wave - wave % waves;
        if ((threadIdx.x & 63) == 0) {
#pragma unroll
            for (int k = 0; k < N; ++k) part[turn][k][wave] = v[k];
        }
        __syncthreads();
#pragma unroll
        for (int k = 0; k < N; ++k) v[k] = 0.f;
#pragma unroll 4
        for (int w = 0; w < waves; ++w)
#pragma unroll
            for (int k = 0; k < N; ++k) v[k] += part[turn][k][first + w];
        turn ^= 1;
    }
};

// Where in its block's rows a thread is.  Rows of whole waves: the same for a wave, so that
// a row's address is; a block of several of them has 4 of one wave or 2 of two.
template <bool SHARED> struct Place {
    int lane, group, groups;
    __device__ __forceinline__ explicit Place(int lanes) {
        if constexpr (SHARED) {
            const int log = 31 - __builtin_clz(lanes);
            lane = threadIdx.x & (lanes - 1);
            group = threadIdx.x >> log;
            groups = blockDim.x >> log;
        } else {
            const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
            groups = (int)blockDim.x == lanes ? 1 : lanes == 64 ? blockDim.x >> 6 : blockDim.x >> 7;
            group = groups == 1 ? 0 : lanes == 64 ? wave : wave >> 1;
            lane = threadIdx.x - group * lanes;
        }
    }
};

// ---- forward -------------------------------------------------------------------

struct ForwardArgs {
    const void *h, *b, *gate;   // b null: y of h alone
    int64_t ldh, ldb, ldgate;   // ldgate 0: a vector
    const float *weight, *next;
    float scale, eps;
    int kind, act;
    int64_t n;
    int dim, lanes;
    void *out, *y;              // y null: out alone
    int64_t ldout, ldy;
};

// A row's last 8 elements overlap those before them where its length is no multiple of 8:
// both threads store the same, and only one counts them.
// SHARED: several rows to a wave.
template <typename T, typename H, bool SHARED> __global__ __launch_bounds__(1024) void forward_kernel(ForwardArgs a) {
    __shared__ __align__(16) float part[2][1][WAVES];
    RowSums<1> sums{part, a.lanes, 0};
    const Place<SHARED> at(a.lanes);
    const int lane = at.lane, per = at.groups;
    const float inv = 1.f / (float)a.dim;
    const bool active = lane * 8 < a.dim;
    const int col = min(lane * 8, a.dim - 8), mine = active ? lane * 8 - col : 8;  // elements below `mine` are another's
    // x becomes x - m; returns r
    auto normalize = [&](f32x8& x) __attribute__((always_inline)) {
        float s[1] = {0.f};
        if (a.kind == FC_NORM_LAYER) {
#pragma unroll
            for (int e = 0; e < 8; ++e)
                if (e >= mine) s[0] += x[e];
            sums.add(s);
            x -= s[0] * inv;
            s[0] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e)
            if (e >= mine) s[0] += x[e] * x[e];
        sums.add(s);
        return 1.f / sqrtf(s[0] * inv + a.eps);
    };
    const int64_t step = (int64_t)gridDim.x * per;
    // every row of a block goes as far, since the block meets; those past the last are the last again
    for (int64_t first = (int64_t)blockIdx.x * per; first < a.n; first += step) {
        const int64_t mine_t = first + at.group, t = min(mine_t, a.n - 1);
        const bool live = active && mine_t < a.n;
        f32x8 x = load8(static_cast<const H*>(a.h) + t * a.ldh + col, 8), next{};
        if (a.y) next = channels(a.next, col, 8);
        if (a.b) {
            f32x8 b = load8(static_cast<const T*>(a.b) + t * a.ldb + col, 8), f = channels(a.weight, col, 8);
            if (a.gate) {
                auto times = [&](auto type, f32x8 g) __attribute__((always_inline)) {
#pragma unroll
                    for (int e = 0; e < 8; ++e) f[e] *= gate_value<decltype(type)>(g[e], a.act);
                };
                if (sizeof(T) == 4 || !a.ldgate) times(float{}, load8(static_cast<const float*>(a.gate) + t * a.ldgate + col, 8));
                else times(T{}, load8(static_cast<const T*>(a.gate) + t * a.ldgate + col, 8));
            }
            const float r = normalize(b) * a.scale;
#pragma unroll
            for (int e = 0; e < 8; ++e) x[e] = (float)(H)(x[e] + f[e] * (b[e] * r));
            if (live) put8(static_cast<H*>(a.out) + t * a.ldout + col, x);
        }
        if (!a.y) continue;
        const float r = normalize(x);
        if (live) put8(static_cast<T*>(a.y) + t * a.ldy + col, x * r * next);
    }
}

// Rows of more than 8192 elements, and of fewer than 8.
template <typename T, typename H, int V> __global__ __launch_bounds__(V == 2 ? MIDDLE : 512) void forward_wide_kernel(ForwardArgs a) {
    __shared__ __align__(16) float part[2][1][WAVES];
    RowSums<1> sums{part, a.lanes, 0};
    const int lane = threadIdx.x;
    const float inv = 1.f / (float)a.dim;
    int c[V], left[V];
#pragma unroll
    for (int v = 0; v < V; ++v) {
        c[v] = (v * a.lanes + lane) * 8;
        left[v] = a.dim - c[v];
    }
    // x becomes x - m; returns r
    auto normalize = [&](f32x8 (&x)[V]) {
        float s[1] = {0.f};
        if (a.kind == FC_NORM_LAYER) {
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) s[0] += x[v][e];
            sums.add(s);
            const float m = s[0] * inv;
#pragma unroll
            for (int v = 0; v < V; ++v)
#pragma unroll
                for (int e = 0; e < 8; ++e) x[v][e] = e < left[v] ? x[v][e] - m : 0.f;
            s[0] = 0.f;
        }
#pragma unroll
        for (int v = 0; v < V; ++v)
#pragma unroll
            for (int e = 0; e < 8; ++e) s[0] += x[v][e] * x[v][e];
        sums.add(s);
        return 1.f / sqrtf(s[0] * inv + a.eps);
    };
    for (int64_t t = blockIdx.x; t < a.n; t += gridDim.x) {
        f32x8 x[V];
        const H* const hp = static_cast<const H*>(a.h) + t * a.ldh;
#pragma unroll
        for (int v = 0; v < V; ++v) x[v] = load8(hp + c[v], left[v]);
        if (a.b) {
            f32x8 b[V], g[V];
            const T* const bp = static_cast<const T*>(a.b) + t * a.ldb;
#pragma unroll
            for (int v = 0; v < V; ++v) b[v] = load8(bp + c[v], left[v]);
            if (a.gate && a.ldgate) {
                const T* const gp = static_cast<const T*>(a.gate) + t * a.ldgate;
#pragma unroll
                for (int v = 0; v < V; ++v) g[v] = load8(gp + c[v], left[v]);
            } else {
#pragma unroll
                for (int v = 0; v < V; ++v) g[v] = channels(static_cast<const float*>(a.gate), c[v], left[v]);
            }
            const float r = normalize(b) * a.scale;
            H* const op = static_cast<H*>(a.out) + t * a.ldout;
#pragma unroll
            for (int v = 0; v < V; ++v) {
                const f32x8 w = channels(a.weight, c[v], left[v]);
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    const float f = a.gate ? gate_value<float>(g[v][e], a.act) * w[e] : w[e];
                    const float o = x[v][e] + f * (b[v][e] * r);
                    x[v][e] = e < left[v] ? (float)(H)o : 0.f;
                }
                store8(op + c[v], left[v], x[v]);
            }
        }
        if (!a.y) continue;
        const float r = normalize(x);
        T* const yp = static_cast<T*>(a.y) + t * a.ldy;
#pragma unroll
        for (int v = 0; v < V; ++v) {
            const f32x8 w = channels(a.next, c[v], left[v]);
            store8(yp + c[v], left[v], x[v] * r * w);
        }
    }
}

// ---- backward ------------------------------------------------------------------

struct BackwardArgs {
    const void *x, *dy, *dout, *b, *gate;     // dy null: no norm before; b null: none after; dout null: 0
    int64_t ldx, lddy, lddout, ldb, ldgate;
    const float *weight, *next;
    float scale, eps;
    int kind, act;
    int64_t n;
    int dim, lanes;
    void *dh, *db, *dgate;                     // dh null after a block alone; dgate: rows of a gate that is a matrix
    int64_t lddh, lddb, lddgate;
    float *sum1, *sum2;                        // [block][ldp]: of the norm after and before, or null
    int ldp;
};

extern __shared__ __align__(32) float column_sums[];

// Rows of up to 8192 elements, 8 to a thread, `groups` rows to a block at a time.  The sums
// over tokens lie in LDS, of which every thread uses its own part: in registers they
// would cost waves.  A row's last 8 elements overlap those
// before them where its length is no multiple of 8: both threads store the same, and only
// one counts them.
template <typename T, typename H, bool SHARED> __global__ __launch_bounds__(1024) void backward_kernel(BackwardArgs a) {
    typedef typename fc::Eight<T>::vec Tv;
    typedef typename fc::Eight<H>::vec Hv;
    __shared__ __align__(16) float part[2][3][WAVES];
    const Place<SHARED> at(a.lanes);
    const int lane = at.lane, group = at.group, groups = at.groups;
    RowSums<3> sums{part, a.lanes, 0};
    const float inv = 1.f / (float)a.dim;
    const bool layer = a.kind == FC_NORM_LAYER, matrix = a.gate && a.ldgate;
    const bool active = lane * 8 < a.dim;
    const int col = min(lane * 8, a.dim - 8), mine = active ? lane * 8 - col : 8;  // elements below `mine` are another's
    const f32x8 next = channels(a.next, col, 8);
    f32x8 weight = channels(a.weight, col, 8);  // from the first row on times a(gate) where that is a vector
    bool gates = a.gate && !matrix;
    f32x4* const own = reinterpret_cast<f32x4*>(column_sums) + threadIdx.x;  // sum1, sum2, four by four
    for (int k = 0; k < 4; ++k) own[k * blockDim.x] = f32x4{};
    auto add = [&](int which, f32x8 q) __attribute__((always_inline)) {
        own[(2 * which) * blockDim.x] += __builtin_shufflevector(q, q, 0, 1, 2, 3);
        own[(2 * which + 1) * blockDim.x] += __builtin_shufflevector(q, q, 4, 5, 6, 7);
    };
    auto total = [&](int which) __attribute__((always_inline)) {
        return __builtin_shufflevector(own[(2 * which) * blockDim.x], own[(2 * which + 1) * blockDim.x], 0, 1, 2, 3, 4, 5, 6, 7);
    };
    const int64_t step = (int64_t)gridDim.x * groups;
    // every group goes through as many rows, since the block meets; those past the last are the last again
    for (int64_t first = (int64_t)blockIdx.x * groups; first < a.n; first += step) {
        const int64_t mine_t = first + group, t = min(mine_t, a.n - 1);
        Hv x{}, dx{};
        Tv dy{}, b{}, g{};
        if (a.dy) {
            x = raw8(static_cast<const H*>(a.x) + t * a.ldx + col);
            dy = raw8(static_cast<const T*>(a.dy) + t * a.lddy + col);
        }
        if (a.b) b = raw8(static_cast<const T*>(a.b) + t * a.ldb + col);
        if (a.dout) dx = raw8(static_cast<const H*>(a.dout) + t * a.lddout + col);
        if (a.b && matrix) g = raw8(static_cast<const T*>(a.gate) + t * a.ldgate + col);
        const bool live = mine_t < a.n && active;
        const int from = live ? mine : 8;  // elements that count
        float s[3] = {0.f, 0.f, 0.f}, mean_x = 0.f, mean_u = 0.f, mean_b = 0.f;
        if (layer) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                if (e < from) continue;
                s[0] += (float)x[e];
                s[1] += next[e] * (float)dy[e];
                s[2] += (float)b[e];
            }
            sums.add(s);
            mean_x = s[0] * inv;
            mean_u = s[1] * inv;
            mean_b = s[2] * inv;
            s[0] = s[1] = s[2] = 0.f;
        }
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            if (e < from) continue;
            const float xm = (float)x[e] - mean_x, bm = (float)b[e] - mean_b;
            s[0] += xm * xm;
            s[1] += next[e] * (float)dy[e] * xm;
            s[2] += bm * bm;
        }
        sums.add(s);
        const float r = 1.f / sqrtf(s[0] * inv + a.eps), rb = 1.f / sqrtf(s[2] * inv + a.eps), along = s[1] * inv * r;
        f32x8 d = __builtin_convertvector(dx, f32x8);
        f32x8 q;
        if (a.dy) {
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float xh = ((float)x[e] - mean_x) * r, u = (float)dy[e];
                d[e] += r * (next[e] * u - mean_u - xh * along);
                q[e] = e >= from ? u * xh : 0.f;
            }
            add(1, q);
            if (live) put8(static_cast<H*>(a.dh) + t * a.lddh + col, d);
        }
        if (a.b) {
            // d becomes the gradient of N(b)
            f32x8 dg;
            if (gates) {  // here, so that the first row's loads do not wait for it
                const f32x8 v = load8(static_cast<const float*>(a.gate) + col, 8);
#pragma unroll
                for (int e = 0; e < 8; ++e) weight[e] *= gate_value<float>(v[e], a.act);
                gates = false;
            }
            s[0] = s[1] = s[2] = 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float bh = ((float)b[e] - mean_b) * rb, ee = a.scale * d[e];
                float f = 1.f, slope = 0.f;
                if (matrix) gate_both<T>((float)g[e], a.act, f, slope);
                dg[e] = ee * slope * weight[e] * bh;
                d[e] = weight[e] * (ee * f);
                q[e] = e < from ? 0.f : ee * f * bh;
                if (e < from) continue;
                s[0] += d[e] * bh;
                s[1] += d[e];
            }
            add(0, q);
            if (a.dgate && live) put8(static_cast<T*>(a.dgate) + t * a.lddgate + col, dg);
            sums.add(s);
            const float along_b = s[0] * inv, mean = layer ? s[1] * inv : 0.f;
#pragma unroll
            for (int e = 0; e < 8; ++e) d[e] = rb * (d[e] - mean - ((float)b[e] - mean_b) * rb * along_b);
            if (live) put8(static_cast<T*>(a.db) + t * a.lddb + col, d);
        }
    }
    // This block's sums, over its rows at a time in order.
    auto put = [&](float* to, f32x8 sum) __attribute__((always_inline)) {
        if (!to) return;
        to += (int64_t)blockIdx.x * a.ldp + col;
        if (mine == 0) {
            put8(to, sum);
        } else {
#pragma unroll
            for (int e = 1; e < 8; ++e)
                if (e >= mine) to[e] = sum[e];
        }
    };
    if constexpr (SHARED) {
        // over a wave's rows, which leaves them in its first `lanes`
        f32x8 sum[2] = {total(0), total(1)};
#pragma unroll
        for (int off = 8; off < 64; off *= 2)
            if (off >= a.lanes) {
#pragma unroll
                for (int k = 0; k < 16; ++k) sum[k / 8][k % 8] += __shfl_xor(sum[k / 8][k % 8], off);
            }
        own[0] = __builtin_shufflevector(sum[0], sum[0], 0, 1, 2, 3);
        own[blockDim.x] = __builtin_shufflevector(sum[0], sum[0], 4, 5, 6, 7);
        own[2 * blockDim.x] = __builtin_shufflevector(sum[1], sum[1], 0, 1, 2, 3);
        own[3 * blockDim.x] = __builtin_shufflevector(sum[1], sum[1], 4, 5, 6, 7);
    }
    // over the block's waves or groups: the first `lanes` threads add what as many threads `apart` hold
    const int apart = SHARED ? 64 : a.lanes, parts = blockDim.x / apart;
    if (parts > 1) __syncthreads();
    if ((int)threadIdx.x >= a.lanes || !active) return;
    f32x4 all[4]{};
    for (int q = 0; q < parts; ++q)
#pragma unroll
        for (int k = 0; k < 4; ++k) all[k] += own[k * blockDim.x + q * apart];
    put(a.sum1, __builtin_shufflevector(all[0], all[1], 0, 1, 2, 3, 4, 5, 6, 7));
    put(a.sum2, __builtin_shufflevector(all[2], all[3], 0, 1, 2, 3, 4, 5, 6, 7));
}

// Rows of more than 8192 elements are read again in each pass over them, from the caches (rows of
// fewer than 8 come here too), and the sums over tokens lie in LDS, of which every thread uses its
// own part: 1.6 TB/s, 327 us for 3640 rows of 9216.  9 or 10 waves have 168 registers each, in which
// the rows as stored would fit, as backward_kernel holds them; such a form has not been built.
template <typename T, typename H, int V> __global__ __launch_bounds__(V == 2 ? MIDDLE : 512) void backward_wide_kernel(BackwardArgs a) {
    __shared__ __align__(16) float part[2][3][WAVES];
    RowSums<3> sums{part, a.lanes, 0};
    const int lane = threadIdx.x;
    const float inv = 1.f / (float)a.dim;
    const bool layer = a.kind == FC_NORM_LAYER, matrix = a.gate && a.ldgate;
    auto col = [&](int v) __attribute__((always_inline)) { return (v * a.lanes + lane) * 8; };
    auto left = [&](int v) __attribute__((always_inline)) { return a.dim - col(v); };
    constexpr int vectors = V;
    auto held = [&](int which, int v) __attribute__((always_inline)) { return reinterpret_cast<f32x8*>(column_sums) + (which * vectors + v) * a.lanes + lane; };
    for (int v = 0; v < 2 * vectors; ++v) *held(0, v) = f32x8{};
    for (int64_t t = blockIdx.x; t < a.n; t += gridDim.x) {
        f32x8 x, dy, b, d, g;  // of one vector at a time
        float s[3], mean_x = 0.f, mean_u = 0.f, mean_b = 0.f, r = 0.f, rb = 0.f, along = 0.f;
        auto fetch = [&](int v, bool all) __attribute__((always_inline)) {  // `all`: not for the statistics alone
            const int n = left(v);
            x = dy = b = d = g = f32x8{};
            if (a.dy) {
                x = load8(static_cast<const H*>(a.x) + t * a.ldx + col(v), n);
                dy = load8(static_cast<const T*>(a.dy) + t * a.lddy + col(v), n);
            }
            if (a.b) b = load8(static_cast<const T*>(a.b) + t * a.ldb + col(v), n);
            if (all && a.dout) d = load8(static_cast<const H*>(a.dout) + t * a.lddout + col(v), n);
            if (all && a.b && matrix) g = load8(static_cast<const T*>(a.gate) + t * a.ldgate + col(v), n);
        };
        auto centre = [&](int v) __attribute__((always_inline)) {
            if (!layer) return;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                x[e] = e < left(v) ? x[e] - mean_x : 0.f;
                b[e] = e < left(v) ? b[e] - mean_b : 0.f;
            }
        };
        // d becomes the gradient of `out`, dy * N(out) is added to its sum
        auto before = [&](int v, bool first) __attribute__((always_inline)) {
            const f32x8 w = channels(a.next, col(v), left(v)), xh = x * r;
            d += r * (w * dy - mean_u - xh * along);
            if (first) *held(1, v) += dy * xh;
        };
        // d becomes the gradient of N(b), b N(b)
        auto after = [&](int v, bool first) __attribute__((always_inline)) {
            const f32x8 w = channels(a.weight, col(v), left(v));
            const f32x8 gv = matrix ? g : channels(static_cast<const float*>(a.gate), col(v), left(v));
            f32x8 dg, q;
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                const float bh = b[e] * rb, ee = e < left(v) ? a.scale * d[e] : 0.f;
                float f = 1.f, slope = 0.f;
                if (matrix) gate_both<T>(gv[e], a.act, f, slope);
                else if (a.gate) f = gate_value<float>(gv[e], a.act);
                dg[e] = ee * slope * w[e] * bh;
                q[e] = (matrix ? ee * f : ee) * bh;
                b[e] = bh;
                d[e] = e < left(v) ? w[e] * (ee * f) : 0.f;
            }
            if (first) *held(0, v) += q;
            if (first && a.dgate && matrix) store8(static_cast<T*>(a.dgate) + t * a.lddgate + col(v), left(v), dg);
        };
        s[0] = s[1] = s[2] = 0.f;
        if (layer) {
#pragma unroll 1
            for (int v = 0; v < vectors; ++v) {
                fetch(v, false);
                const f32x8 w = a.dy ? channels(a.next, col(v), left(v)) : f32x8{};
#pragma unroll
                for (int e = 0; e < 8; ++e) {
                    s[0] += x[e];
                    s[1] += w[e] * dy[e];
                    s[2] += b[e];
                }
            }
        }
        if (layer) {
            sums.add(s);
            mean_x = s[0] * inv;
            mean_u = s[1] * inv;
            mean_b = s[2] * inv;
            s[0] = s[1] = s[2] = 0.f;
        }
#pragma unroll 1
        for (int v = 0; v < vectors; ++v) {
            fetch(v, false);
            centre(v);
            const f32x8 w = a.dy ? channels(a.next, col(v), left(v)) : f32x8{};
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[0] += x[e] * x[e];
                s[1] += w[e] * dy[e] * x[e];
                s[2] += b[e] * b[e];
            }
        }
        sums.add(s);
        rb = 1.f / sqrtf(s[2] * inv + a.eps);
        r = 1.f / sqrtf(s[0] * inv + a.eps);
        along = s[1] * inv * r;
        s[0] = s[1] = s[2] = 0.f;
#pragma unroll 1
        for (int v = 0; v < vectors; ++v) {
            fetch(v, true);
            centre(v);
            if (a.dy) {
                before(v, true);
                store8(static_cast<H*>(a.dh) + t * a.lddh + col(v), left(v), d);
            }
            if (!a.b) continue;
            after(v, true);
#pragma unroll
            for (int e = 0; e < 8; ++e) {
                s[0] += d[e] * b[e];
                s[1] += d[e];
            }
        }
        if (!a.b) continue;
        sums.add(s);
        const float along_b = s[0] * inv, mean = layer ? s[1] * inv : 0.f;
#pragma unroll 1
        for (int v = 0; v < vectors; ++v) {
            fetch(v, true);
            centre(v);
            if (a.dy) before(v, false);
            after(v, false);
            store8(static_cast<T*>(a.db) + t * a.lddb + col(v), left(v), rb * (d - mean - b * along_b));
        }
    }
#pragma unroll
    for (int which = 0; which < 2; ++which) {
        float* const to = which ? a.sum2 : a.sum1;
        if (!to) continue;
        for (int v = 0; v < vectors; ++v)
            if (left(v) > 0) *reinterpret_cast<f32x8*>(to + (int64_t)blockIdx.x * a.ldp + col(v)) = *held(which, v);
    }
}

// ---- vectors' gradients -----------------------------------------------------------

struct FinishArgs {
    const float *sum1, *sum2;   // [blocks][ldp], or null
    int blocks, ldp, dim;
    const float *gate, *weight;  // gate: a vector, or null
    int act;
    void *dweight, *dgate, *dnext;
    int dvec, accumulate;
};

__device__ __forceinline__ void put_channel(void* p, int dt, int c, float v, int accumulate) {
    if (accumulate) v += dt == FC_F32 ? static_cast<float*>(p)[c] : dt == FC_F16 ? (float)static_cast<f16*>(p)[c] : (float)static_cast<bf16*>(p)[c];
    if (dt == FC_F32) static_cast<float*>(p)[c] = v;
    else if (dt == FC_F16) static_cast<f16*>(p)[c] = (f16)v;
    else static_cast<bf16*>(p)[c] = (bf16)v;
}

// 32 channels to a block: 128 rows' worth of threads add every 128th partial sum of 4
// channels each, 32 lanes these.
__global__ __launch_bounds__(1024) void finish_kernel(FinishArgs a) {
    const float* const p = blockIdx.y ? a.sum2 : a.sum1;
    if (!p) return;
    __shared__ float part[128][33];
    {
        const int x = 4 * (threadIdx.x & 7), y = threadIdx.x >> 3, c = blockIdx.x * 32 + x;
        f32x4 s{};
        for (int k0 = y; k0 < a.blocks; k0 += 128 * 4) {  // 4 on their way at a time
            f32x4 v[4];
#pragma unroll
            for (int q = 0; q < 4; ++q) {
                const int k = k0 + 128 * q;
                v[q] = k < a.blocks && c < a.ldp ? *reinterpret_cast<const f32x4*>(p + (int64_t)k * a.ldp + c) : f32x4{};
            }
#pragma unroll
            for (int q = 0; q < 4; ++q) s += v[q];
        }
#pragma unroll
        for (int e = 0; e < 4; ++e) part[y][x + e] = s[e];
    }
    __syncthreads();
    const int j = threadIdx.x & 31, c = blockIdx.x * 32 + (threadIdx.x >> 5);
    float s = 0.f;
#pragma unroll
    for (int q = 0; q < 4; ++q) s += part[4 * j + q][threadIdx.x >> 5];
    s = sum_lanes(s, 32);
    if (j || c >= a.dim) return;
    if (blockIdx.y) {
        put_channel(a.dnext, a.dvec, c, s, a.accumulate);
        return;
    }
    float f = 1.f, slope = 0.f;
    if (a.gate) gate_both<float>(a.gate[c], a.act, f, slope);
    if (a.dgate) put_channel(a.dgate, a.dvec, c, slope * (a.weight ? a.weight[c] : 1.f) * s, a.accumulate);
    if (a.dweight) put_channel(a.dweight, a.dvec, c, f * s, a.accumulate);
}

constexpr int64_t TOKENS_LIMIT = (int64_t)1 << 31;
constexpr int64_t FORWARD_BLOCKS = 1 << 20;

// The sums over tokens of a block of rows of several vectors to a thread.
int wide_lds(Shape s) { return 2 * s.vectors * s.lanes * (int)sizeof(f32x8); }

// Blocks of a backward pass that the chip holds at once: 16 waves to a compute unit, of rows of
// several vectors to a thread 12 and as many blocks as its LDS holds, 8 at most.
int64_t blocks_limit(Shape s) {
    if (s.vectors == 1) return 256 * (1024 / (s.groups * s.lanes));
    return 256 * std::max(1, std::min({160 * 1024 / (wide_lds(s) + 1024), 768 / s.lanes, 8}));
}

// Blocks of a backward pass of n rows.
int64_t backward_blocks(Shape s, int64_t n) { return std::min<int64_t>(fc::ceil_div(n, s.groups), blocks_limit(s)); }

}  // namespace

struct fc_norm {
    fc::CallOrder order;
    fc::DeviceBlock block;
    int64_t dim = 0, max_tokens = 0;
    int dtype = FC_F16, residual = FC_F32, kind = FC_NORM_RMS, act = FC_GATE_NONE;
    float eps = 0;
    Shape shape{};
    int ldp = 0;
    float *sum1 = nullptr, *sum2 = nullptr;
};

namespace {

template <typename T, typename H> void forward(const Shape& s, unsigned grid, const ForwardArgs& a, hipStream_t st) {
    if (s.vectors == 4) forward_wide_kernel<T, H, 4><<<grid, s.threads, 0, st>>>(a);
    else if (s.vectors == 2) forward_wide_kernel<T, H, 2><<<grid, s.threads, 0, st>>>(a);
    else if (s.lanes < 64) forward_kernel<T, H, true><<<grid, s.threads, 0, st>>>(a);
    else forward_kernel<T, H, false><<<grid, s.threads, 0, st>>>(a);
}

// The LDS of the longest rows.
template <typename T, typename H> hipError_t prepare() {
    const hipError_t e = hipFuncSetAttribute((const void*)backward_wide_kernel<T, H, 2>, hipFuncAttributeMaxDynamicSharedMemorySize, 128 * MIDDLE);
    return e != hipSuccess ? e : hipFuncSetAttribute((const void*)backward_wide_kernel<T, H, 4>, hipFuncAttributeMaxDynamicSharedMemorySize, 8 * DIM_LIMIT);
}

template <typename T, typename H> void backward(const Shape& s, unsigned grid, const BackwardArgs& a, hipStream_t st) {
    if (s.vectors == 4) backward_wide_kernel<T, H, 4><<<grid, s.threads, wide_lds(s), st>>>(a);
    else if (s.vectors == 2) backward_wide_kernel<T, H, 2><<<grid, s.threads, wide_lds(s), st>>>(a);
    else {
        const int threads = s.groups * s.lanes;
        if (s.lanes < 64) backward_kernel<T, H, true><<<grid, threads, threads * 2 * sizeof(f32x8), st>>>(a);
        else backward_kernel<T, H, false><<<grid, threads, threads * 2 * sizeof(f32x8), st>>>(a);
    }
}

// f<block side's type, residual side's type>() of a plan.
template <typename F> void by_types(const fc_norm* p, F&& f) {
    const bool wide = p->residual == FC_F32;
    if (p->dtype == FC_F32) f(float{}, float{});
    else if (p->dtype == FC_F16 && wide) f(f16{}, float{});
    else if (p->dtype == FC_F16) f(f16{}, f16{});
    else if (wide) f(bf16{}, float{});
    else f(bf16{}, bf16{});
}

// A matrix of a call, or nothing where it is null.
fc::Span matrix(const void* p, int64_t n, int64_t dim, int64_t ld, int dt, bool written) {
    return p ? fc::Span{p, n, dim, ld, fc::dtype_bytes(dt), written} : fc::Span{nullptr, 0, 0, 0, 1, false};
}

// A gate, its gradient: a vector where ld is 0, else n rows.
fc::Span gate_span(const void* p, int64_t n, int64_t dim, int64_t ld, int dt, int vec, bool vector, bool written) {
    return vector ? matrix(p, 1, dim, dim, vec, written) : matrix(p, n, dim, ld, dt, written);
}

int call_forward(fc_norm* p, const void* h, int64_t ldh, const void* b, int64_t ldb, int64_t n, const void* gate, int64_t ldgate,
                 const float* weight, const float* next, float scale, void* out, int64_t ldout, void* y, int64_t ldy,
                 bool after, bool before, hipStream_t s) {
    if (!p || n < 0 || n >= TOKENS_LIMIT) return FC_EINVAL;
    if (n && (!h || (after && (!b || !out)) || (before && !y))) return FC_EINVAL;
    const int64_t dim = p->dim;
    int rc = fc::check_spans({matrix(h, n, dim, ldh, p->residual, false), matrix(b, n, dim, ldb, p->dtype, false),
                              gate_span(gate, n, dim, ldgate, p->dtype, FC_F32, ldgate == 0, false), matrix(weight, 1, dim, dim, FC_F32, false),
                              matrix(next, 1, dim, dim, FC_F32, false), matrix(out, n, dim, ldout, p->residual, true),
                              matrix(y, n, dim, ldy, p->dtype, true)});
    if (rc) return rc;
    bool note;
    rc = p->order.begin(s, note);
    if (rc) return rc;
    if (n) {
        const ForwardArgs a{h, after ? b : nullptr, gate, ldh, ldb, ldgate, weight, next, scale, p->eps, p->kind, p->act, n, (int)dim, p->shape.lanes,
                            out, before ? y : nullptr, ldout, ldy};
        const int64_t per = p->shape.threads / p->shape.lanes;
        const unsigned grid = (unsigned)std::min(fc::ceil_div(n, per), FORWARD_BLOCKS);
        by_types(p, [&](auto t, auto r) { forward<decltype(t), decltype(r)>(p->shape, grid, a, s); });
    }
    rc = fc::hip_code(hipGetLastError());
    p->order.done(s, note);
    return rc;
}

int call_backward(fc_norm* p, const void* x, int64_t ldx, const void* b, int64_t ldb, const void* dy, int64_t lddy, const void* dout,
                  int64_t lddout, int64_t n, const void* gate, int64_t ldgate, const float* weight, const float* next, float scale,
                  void* dh, int64_t lddh, void* db, int64_t lddb, void* dgate, int64_t lddgate, void* dweight, void* dnext, int dvec,
                  int accumulate, bool after, bool before, hipStream_t s) {
    if (!p || n < 0 || n > p->max_tokens) return FC_EINVAL;
    if (n && ((before && (!x || !dy || !dh)) || (after && (!b || !db)) || (!before && !dout))) return FC_EINVAL;
    if (dgate && !gate) return FC_EINVAL;
    const bool vector = ldgate == 0;
    if ((dweight || dnext || (dgate && vector)) && !fc::dtype_bytes(dvec)) return FC_EINVAL;
    const int64_t dim = p->dim;
    int rc = fc::check_spans({matrix(x, n, dim, ldx, p->residual, false), matrix(b, n, dim, ldb, p->dtype, false),
                              matrix(dy, n, dim, lddy, p->dtype, false), matrix(dout, n, dim, lddout, p->residual, false),
                              gate_span(gate, n, dim, ldgate, p->dtype, FC_F32, vector, false), matrix(weight, 1, dim, dim, FC_F32, false),
                              matrix(next, 1, dim, dim, FC_F32, false), matrix(dh, n, dim, lddh, p->residual, true),
                              matrix(db, n, dim, lddb, p->dtype, true), gate_span(dgate, n, dim, lddgate, p->dtype, dvec, vector, true),
                              matrix(dweight, 1, dim, dim, dvec, true), matrix(dnext, 1, dim, dim, dvec, true)});
    if (rc) return rc;
    bool note;
    rc = p->order.begin(s, note);
    if (rc) return rc;
    float* const sum1 = dweight || (dgate && vector) ? p->sum1 : nullptr;
    float* const sum2 = dnext ? p->sum2 : nullptr;
    const int64_t blocks = backward_blocks(p->shape, n);
    if (n) {
        const BackwardArgs a{x, before ? dy : nullptr, dout, after ? b : nullptr, gate, ldx, lddy, lddout, ldb, ldgate, weight, next, scale, p->eps,
                             p->kind, p->act, n, (int)dim, p->shape.lanes, dh, db, vector ? nullptr : dgate, lddh, lddb, lddgate, sum1, sum2, p->ldp};
        by_types(p, [&](auto t, auto r) { backward<decltype(t), decltype(r)>(p->shape, (unsigned)blocks, a, s); });
    }
    if (sum1 || sum2) {
        const FinishArgs f{sum1, sum2, (int)blocks, p->ldp, (int)dim, vector ? static_cast<const float*>(gate) : nullptr, weight, p->act, dweight, vector ? dgate : nullptr, dnext,
                           dvec, accumulate};
        finish_kernel<<<dim3((unsigned)fc::ceil_div(dim, 32), 2), 1024, 0, s>>>(f);
    }
    rc = fc::hip_code(hipGetLastError());
    p->order.done(s, note);
    return rc;
}

}  // namespace

extern "C" {

int fc_norm_create(fc_norm** plan, int64_t dim, int64_t max_tokens, int dtype, int residual_dtype, int kind, float eps, int gate) {
    if (!plan) return FC_EINVAL;
    *plan = nullptr;
    if (dim < 1 || dim > DIM_LIMIT || max_tokens < 0 || max_tokens >= TOKENS_LIMIT || !fc::dtype_bytes(dtype) ||
        (residual_dtype != dtype && residual_dtype != FC_F32) || (kind != FC_NORM_RMS && kind != FC_NORM_LAYER) || !(eps > 0) ||
        !(eps < __builtin_inff()) || gate < FC_GATE_NONE || gate > FC_GATE_SILU)
        return FC_EINVAL;
    return fc::no_throw([&] {
        fc_norm* p = new fc_norm;
        p->dim = dim;
        p->max_tokens = max_tokens;
        p->dtype = dtype;
        p->residual = residual_dtype;
        p->kind = kind;
        p->act = gate;
        p->eps = eps;
        p->shape = shape_of(dim);
        p->ldp = (int)fc::ceil_div(dim, 8) * 8;
        fc::Layout at;
        const uint64_t each = (uint64_t)backward_blocks(p->shape, max_tokens) * p->ldp * 4;
        const uint64_t o1 = at.take(each), o2 = at.take(each);
        int rc = p->order.create();
        if (!rc && p->shape.vectors > 1) by_types(p, [&](auto t, auto r) { rc = fc::hip_code(prepare<decltype(t), decltype(r)>()); });
        if (!rc) rc = p->block.create(at.size);
        if (rc) {
            fc_norm_destroy(p);
            return rc;
        }
        p->sum1 = reinterpret_cast<float*>(p->block.p + o1);
        p->sum2 = reinterpret_cast<float*>(p->block.p + o2);
        *plan = p;
        return FC_OK;
    });
}

void fc_norm_destroy(fc_norm* p) {
    if (!p) return;
    p->block.destroy();
    p->order.destroy();
    delete p;
}

int fc_norm_before(fc_norm* p, const void* x, int64_t ld_x, int64_t n, const float* weight, void* y, int64_t ld_y, void* stream) {
    return fc::no_throw([&] {
        return call_forward(p, x, ld_x, nullptr, 0, n, nullptr, 0, nullptr, weight, 0.f, nullptr, 0, y, ld_y, false, true,
                            static_cast<hipStream_t>(stream));
    });
}

int fc_norm_after(fc_norm* p, const void* h, int64_t ld_h, const void* b, int64_t ld_b, int64_t n, const void* gate, int64_t ld_gate,
                  const float* weight, float scale, void* out, int64_t ld_out, void* stream) {
    return fc::no_throw([&] {
        return call_forward(p, h, ld_h, b, ld_b, n, gate, ld_gate, weight, nullptr, scale, out, ld_out, nullptr, 0, true, false,
                            static_cast<hipStream_t>(stream));
    });
}

int fc_norm_between(fc_norm* p, const void* h, int64_t ld_h, const void* b, int64_t ld_b, int64_t n, const void* gate, int64_t ld_gate,
                    const float* weight, const float* next_weight, float scale, void* out, int64_t ld_out, void* y, int64_t ld_y,
                    void* stream) {
    return fc::no_throw([&] {
        return call_forward(p, h, ld_h, b, ld_b, n, gate, ld_gate, weight, next_weight, scale, out, ld_out, y, ld_y, true, true,
                            static_cast<hipStream_t>(stream));
    });
}

int fc_norm_before_grad(fc_norm* p, const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, const void* dout, int64_t ld_dout, int64_t n,
                        const float* weight, void* dx, int64_t ld_dx, void* dweight, int dvec_dtype, int accumulate,
                        void* stream) {
    return fc::no_throw([&] {
        return call_backward(p, x, ld_x, nullptr, 0, dy, ld_dy, dout, ld_dout, n, nullptr, 0, nullptr, weight, 0.f, dx, ld_dx, nullptr, 0,
                             nullptr, 0, nullptr, dweight, dvec_dtype, accumulate, false, true, static_cast<hipStream_t>(stream));
    });
}

int fc_norm_after_grad(fc_norm* p, const void* b, int64_t ld_b, const void* dout, int64_t ld_dout, int64_t n, const void* gate,
                       int64_t ld_gate, const float* weight, float scale, void* db, int64_t ld_db, void* dgate,
                       int64_t ld_dgate, void* dweight, int dvec_dtype, int accumulate, void* stream) {
    return fc::no_throw([&] {
        return call_backward(p, nullptr, 0, b, ld_b, nullptr, 0, dout, ld_dout, n, gate, ld_gate, weight, nullptr, scale, nullptr, 0, db,
                             ld_db, dgate, ld_dgate, dweight, nullptr, dvec_dtype, accumulate, true, false, static_cast<hipStream_t>(stream));
    });
}

int fc_norm_between_grad(fc_norm* p, const void* out, int64_t ld_out, const void* b, int64_t ld_b, const void* dy, int64_t ld_dy,
                         const void* dout, int64_t ld_dout, int64_t n, const void* gate, int64_t ld_gate, const float* weight,
                         const float* next_weight, float scale, void* dh, int64_t ld_dh, void* db, int64_t ld_db, void* dgate,
                         int64_t ld_dgate, void* dweight, void* dnext, int dvec_dtype, int accumulate, void* stream) {
    return fc::no_throw([&] {
        return call_backward(p, out, ld_out, b, ld_b, dy, ld_dy, dout, ld_dout, n, gate, ld_gate, weight, next_weight, scale, dh, ld_dh, db,
                             ld_db, dgate, ld_dgate, dweight, dnext, dvec_dtype, accumulate, true, true, static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
