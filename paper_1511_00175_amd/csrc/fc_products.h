// What the operators' products of two 16-bit matrices share beside fc_gemm.h: results
// with a scale, added up over parts of k or calls, the joins of these parts, and copies of
// operands that lie otherwise than the products need.
#pragma once

#include "fc_choice.h"
#include "fc_eight.h"
#include "fc_gemm.h"
#include "fc_lm_host.h"

using fc::Operand;
using fc::f32x2;
using fc::f32x4;
using fc::Half;

namespace {

typedef _Float16 f16;
typedef __bf16 bf16;

static_assert(STEP == fc::GEMM_BK, "the estimates are of the products' steps");

extern __shared__ __align__(1024) char lds[];

__device__ __forceinline__ int64_t target_of(const void* p, int bytes, int64_t t) {
    return bytes == 8 ? static_cast<const int64_t*>(p)[t] : static_cast<const int32_t*>(p)[t];
}

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

__device__ __forceinline__ float load_one(const void* p, int dt, int64_t at) {
    return dt == FC_F32 ? static_cast<const float*>(p)[at] : dt == FC_F16 ? (float)static_cast<const f16*>(p)[at] : (float)static_cast<const bf16*>(p)[at];
}

// O: of the operands, fc::Operand or another that P::run takes.
template <typename O> struct ResultArgs {
    O a, b;
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

typedef ResultArgs<Operand> GradArgs;

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

// Results of one call, or one part of k, straight from registers: two neighbouring fragments'
// 4 neighbours of a lane become 8 neighbours of one fragment by an exchange with the lane 16
// away, so that 16 rows get 32 or 64 bytes each in one store.  Against the strips above,
// which also hold sums over calls and padding: 256 x 256 tiles of 16-bit results that all
// end at once took 11 us for them, 4 so.
template <typename P, bool ADD, typename T, typename O>
__device__ __forceinline__ void store_tile_as(const ResultArgs<O>& a, const P& p, T* out, int64_t ld, float scale, int m0, int n0) {
    const int g = (threadIdx.x & 63) >> 4;
#pragma unroll
    for (int i = 0; i < P::FM; ++i) {
        const int m = m0 + P::row(i);
        const bool live = m < a.m;
        T* const row = out + (int64_t)m * ld;
#pragma unroll
        for (int j = 0; j + 1 < P::FN; j += 2) {
            fc::f32x8 v;
#pragma unroll
            for (int e = 0; e < 4; ++e) {
                const float x = p.acc[i][j][e], y = p.acc[i][j + 1][e];
                const auto both = __builtin_amdgcn_permlane16_swap(__builtin_bit_cast(uint32_t, x), __builtin_bit_cast(uint32_t, y), false, false);
                const uint32_t lo = both[0], hi = both[1];
                v[e] = __builtin_bit_cast(float, lo);
                v[e + 4] = __builtin_bit_cast(float, hi);
            }
            const int n = n0 + P::col(0) - 4 * g + 16 * (j + (g & 1)) + 8 * (g >> 1), left = a.n - n;
            v = v * scale;
            if (!live || left <= 0) continue;
            if constexpr (ADD) v += fc::load8(row + n, left);
            fc::store8(row + n, left, v);
        }
        if constexpr (P::FN % 2) {
            const int n = n0 + P::col(P::FN - 1), left = a.n - n;
#pragma unroll
            for (int e = 0; e < 4; ++e)
                if (live && e < left) row[n + e] = (T)(p.acc[i][P::FN - 1][e] * scale + (ADD ? (float)row[n + e] : 0.f));
        }
    }
}

// ADD: to what `out` holds.
template <typename P, bool ADD, typename O> __global__ __launch_bounds__(P::THREADS, P::THREADS / 256) void result_kernel(ResultArgs<O> a) {
    int ti, tj;
    fc::tile_place(fc::xcd_order(blockIdx.x, a.tm * a.tn), a.tm, a.tn, 8, ti, tj);
    const int kb = blockIdx.y * a.kper, ke = min(a.k, kb + a.kper);
    P p;
    p.run(lds, a.a, a.b, ti * P::BM, tj * P::BN, kb, ke, a.parts);
    if (a.sum) store_tile_as<P, false, float>(a, p, a.sum + (int64_t)blockIdx.y * a.m * a.n, a.n, 1.f, ti * P::BM, tj * P::BN);
    else if (a.dt == FC_F32) store_tile_as<P, ADD, float>(a, p, static_cast<float*>(a.out), a.ld, a.scale, ti * P::BM, tj * P::BN);
    else if (a.dt == FC_F16) store_tile_as<P, ADD, f16>(a, p, static_cast<f16*>(a.out), a.ld, a.scale, ti * P::BM, tj * P::BN);
    else store_tile_as<P, ADD, bf16>(a, p, static_cast<bf16*>(a.out), a.ld, a.scale, ti * P::BM, tj * P::BN);
}

struct SplitArgs {
    const float* sum;
    int splits, m, n;
    float scale;
    const int* row;
    void* out;
    int dt;
    int64_t ld;
    bool add;
    int64_t from;            // of this launch, in elements of a part
};

// The splits of a product added in order: 4 to 7 us, a launch's latency and one
// trip to memory.
__global__ __launch_bounds__(256) void split_kernel(SplitArgs a) {
    const int64_t i = a.from + (int64_t)blockIdx.x * 256 + threadIdx.x, total = (int64_t)a.m * a.n;
    if (i >= total) return;
    const int m = (int)(i / a.n), n = (int)(i % a.n);
    float v = 0.f;
#pragma unroll 8
    for (int s = 0; s < a.splits; ++s) v += a.sum[s * total + i];
    v = a.row && a.row[m] < 0 ? 0.f : v * a.scale;
    const int64_t to = (int64_t)m * a.ld + n;
    if (a.add) v += load_one(a.out, a.dt, to);
    store_one(a.out, a.dt, to, v);
}

template <typename O> void join_splits(const ResultArgs<O>& g, int splits, bool add, hipStream_t s) {
    fc::by_launches((int64_t)g.m * g.n, 1, [&](int64_t from, int64_t count) {
        SplitArgs q{g.sum, splits, g.m, g.n, g.scale, g.row, g.out, g.dt, g.ld, add, from};
        split_kernel<<<(unsigned)fc::ceil_div(count, 256), 256, 0, s>>>(q);
    });
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

template <typename P> hipError_t prepare(const void* kernel) {
    return P::LDS > 64 * 1024 ? hipFuncSetAttribute(kernel, hipFuncAttributeMaxDynamicSharedMemorySize, P::LDS) : hipSuccess;
}

template <typename P> void launch_grad(GradArgs a, hipStream_t s) {
    a.tm = (int)fc::ceil_div(a.m, P::BM);
    a.tn = (int)fc::ceil_div(a.n, P::BN);
    grad_kernel<P><<<dim3(a.tm * a.tn, (unsigned)fc::ceil_div(a.k, a.kper)), P::THREADS, P::LDS, s>>>(a);
}

template <typename P, bool ADD, typename O> void launch_result(ResultArgs<O> a, hipStream_t s) {
    a.tm = (int)fc::ceil_div(a.m, P::BM);
    a.tn = (int)fc::ceil_div(a.n, P::BN);
    result_kernel<P, ADD, O><<<dim3(a.tm * a.tn, (unsigned)fc::ceil_div(a.k, a.kper)), P::THREADS, P::LDS, s>>>(a);
}

__global__ __launch_bounds__(256) void zero_kernel(void* p, int dt, int64_t rows, int64_t len, int64_t ld) {
    const int64_t i = (int64_t)blockIdx.x * 256 + threadIdx.x;
    if (i < rows * len) store_one(p, dt, i / len * ld + i % len, 0.f);
}

// Zeros for a gradient without tokens: m rows of n elements.
inline void zeros(void* p, int dt, int64_t m, int64_t n, int64_t ld, hipStream_t s) {
    fc::by_launches(m, n, [&](int64_t r0, int64_t count) {
        zero_kernel<<<(unsigned)fc::ceil_div(count * n, 256), 256, 0, s>>>(static_cast<char*>(p) + r0 * ld * fc::dtype_bytes(dt), dt, count, n, ld);
    });
}

}  // namespace
