// Blocks of 32 neighbours of a row that share a scale: the formats of fc_ckpt and fc_mxfp.
//
// A scale is a power of two, 2^(byte - 127), byte 255 a NaN (E8M0); an element is an
// integer of 8 bits, a float of 8 (e4m3, largest 448) or of 4 (e2m1, largest 6), times it.
// The scale is the smallest with which no element of the block rounds past the format's
// largest number: with p bits of significand the block's largest magnitude is rounded to
// these, ties to even, and the exponent of that, less the largest number's, is taken.  So
// nothing saturates, and a block's largest element keeps all of its p bits.  Products with
// powers of two are exact, so that an element is rounded once.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

#include "fc_eight.h"
#include "fc_lm_host.h"

namespace fc {

constexpr int BLOCK = 32;

// FC_BLOCK_* of fc_lm.h, and the 4-bit one.
constexpr int E2M1 = 2;

// What is added to a magnitude's bits so that the exponent of the sum is that of the
// rounded magnitude: 1.111111|1 (127.5 / 64), 1.111 (e4m3 has no 1.111 * 2^8, so 1.110|1 and
// the tie below it stay), 1.1|1 in binary round up to the next power.
template <int F> constexpr uint32_t ROUND_UP = F == FC_BLOCK_I8 ? 0x010000u : F == FC_BLOCK_E4M3 ? 0x17ffffu : 0x200000u;
// Exponent of the largest number.
template <int F> constexpr int TOP = F == FC_BLOCK_I8 ? 6 : F == FC_BLOCK_E4M3 ? 8 : 2;
// Bytes of 8 elements.
template <int F> constexpr int EIGHT_BYTES = F == E2M1 ? 4 : 8;

// The scale's byte for a block whose largest magnitude has these bits (sign off); 255
// for infinities and NaN.
template <int F> __device__ __forceinline__ uint32_t scale_byte(uint32_t most) {
    if (most >= 0x7f800000u) return 255;
    const int e = (int)((most + ROUND_UP<F>) >> 23) - TOP<F>;
    return e < 0 ? 0 : e;
}

__device__ __forceinline__ float scale_value(uint32_t byte) {
    return __builtin_bit_cast(float, byte == 255 ? 0x7fc00000u : byte == 0 ? 0x00400000u : byte << 23);
}

// 1 / scale_value(byte); 0 for NaN, with which every code is 0.
__device__ __forceinline__ float scale_inverse(uint32_t byte) { return byte == 255 ? 0.f : __builtin_bit_cast(float, (254 - byte) << 23); }

// Bits of the largest magnitude of 8 elements; those of infinities and NaN are above
// every number's.
__device__ __forceinline__ uint32_t most_of(f32x8 v) {
    uint32_t m = 0;
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        const float x = v[e];  // a bit cast of v[e] itself takes v[0]
        m = max(m, __builtin_bit_cast(uint32_t, x) & 0x7fffffffu);
    }
    return m;
}

// The most of 4 neighbouring lanes', for a block of 32: by a permutation of lanes, not by way of LDS.
__device__ __forceinline__ uint32_t most_of_four(uint32_t most) {
    most = max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0xb1, 0xf, 0xf, true));  // lanes 1, 0, 3, 2
    return max(most, (uint32_t)__builtin_amdgcn_update_dpp(0, (int)most, 0x4e, 0xf, 0xf, true));  // lanes 2, 3, 0, 1
}

struct Codes {
    uint32_t lo, hi;  // hi unused by the 4-bit format
};

// 8 elements' codes, the first lowest; `inv` is their scale's inverse.
template <int F> __device__ __forceinline__ Codes encode8(f32x8 v, float inv) {
    Codes c{0, 0};
    if (inv == 0.f) return c;
    v = v * inv;
    if constexpr (F == FC_BLOCK_I8) {
        uint32_t q[8];
#pragma unroll
        for (int e = 0; e < 8; ++e) q[e] = (uint32_t)(int)rintf(v[e]) & 255u;
        c.lo = q[0] | q[1] << 8 | q[2] << 16 | q[3] << 24;
        c.hi = q[4] | q[5] << 8 | q[6] << 16 | q[7] << 24;
    } else if constexpr (F == FC_BLOCK_E4M3) {
        c.lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[0], v[1], 0, false);
        c.lo = __builtin_amdgcn_cvt_pk_fp8_f32(v[2], v[3], c.lo, true);
        c.hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[4], v[5], 0, false);
        c.hi = __builtin_amdgcn_cvt_pk_fp8_f32(v[6], v[7], c.hi, true);
    } else {
        c.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c.lo, v[0], v[1], 1.f, 0);
        c.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c.lo, v[2], v[3], 1.f, 1);
        c.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c.lo, v[4], v[5], 1.f, 2);
        c.lo = __builtin_amdgcn_cvt_scalef32_pk_fp4_f32(c.lo, v[6], v[7], 1.f, 3);
    }
    return c;
}

// 8 codes as numbers, without their scale.
template <int F> __device__ __forceinline__ f32x8 decode8(Codes c) {
    f32x8 v;
    if constexpr (F == FC_BLOCK_I8) {
#pragma unroll
        for (int e = 0; e < 4; ++e) {
            v[e] = (float)(int8_t)(c.lo >> (8 * e));
            v[e + 4] = (float)(int8_t)(c.hi >> (8 * e));
        }
    } else if constexpr (F == FC_BLOCK_E4M3) {
        typedef float f32x2 __attribute__((ext_vector_type(2)));
        const f32x2 a = __builtin_amdgcn_cvt_pk_f32_fp8(c.lo, false), b = __builtin_amdgcn_cvt_pk_f32_fp8(c.lo, true);
        const f32x2 d = __builtin_amdgcn_cvt_pk_f32_fp8(c.hi, false), g = __builtin_amdgcn_cvt_pk_f32_fp8(c.hi, true);
        v = f32x8{a.x, a.y, b.x, b.y, d.x, d.y, g.x, g.y};
    } else {
        // twice the magnitude of a code: 0, 1, 2, 3, 4, 6, 8, 12
#pragma unroll
        for (int e = 0; e < 8; ++e) {
            const uint32_t q = c.lo >> (4 * e), m = q & 7;
            const uint32_t twice = m < 4 ? m : (2 + (m & 1)) << ((m >> 1) - 1);
            v[e] = (q & 8) ? -0.5f * (float)twice : 0.5f * (float)twice;
        }
    }
    return v;
}

// A block's numbers in a type: one past its largest becomes that (the largest of a
// block may have been rounded up to a power of two that the type lacks), a NaN stays.
template <typename T> __device__ __forceinline__ f32x8 in_range(f32x8 v) {
    constexpr float MOST = sizeof(T) == 4 ? 3.4028234663852886e38f : __is_same(T, __bf16) ? 3.3895313892515355e38f : 65504.f;
#pragma unroll
    for (int e = 0; e < 8; ++e) v[e] = v[e] > MOST ? MOST : v[e] < -MOST ? -MOST : v[e];
    return v;
}

// The largest scale's byte with which all of a format's numbers are in a type's range.
template <int F, typename T> constexpr uint32_t FITS = 127 + (sizeof(T) == 2 && !__is_same(T, __bf16) ? 15 : 127) - (F == FC_BLOCK_I8 ? 7 : F == FC_BLOCK_E4M3 ? 9 : 3);

// ---- rows to blocks and back -----------------------------------------------------

struct BlockRows {
    const void* x;           // rows of dim elements
    int64_t ldx;
    uint8_t* codes;
    int64_t ldc;
    uint8_t* scales;         // packing: a row's first 8 at r * lds, its next `group` on
    int64_t lds;
    int64_t rows;
    int dim, blocks, width;  // width: bytes of a row of scales, those past the blocks are zeros
    int64_t group;
};

// The i-th 8 elements; 4 threads to a block of 32.  (More than 8 elements to a thread, with as
// many loads on their way, is no faster: 32768 rows of 2048 fp16 to int8 45 us, 203 MB at 4.5
// TB/s, which is a copy's rate; 54 with four times as many to a thread.)
template <int F, typename T> __device__ __forceinline__ void pack_eight(const BlockRows& a, uint32_t i) {
    const uint32_t per = 4 * a.blocks, r = i / per, u = i % per;
    if (r >= a.rows) return;
    const f32x8 v = load8(static_cast<const T*>(a.x) + r * a.ldx + 8 * u, a.dim - 8 * (int)u);
    const uint32_t byte = scale_byte<F>(most_of_four(most_of(v)));
    const Codes c = encode8<F>(v, scale_inverse(byte));
    uint8_t* const to = a.codes + r * a.ldc + u * EIGHT_BYTES<F>;
    if constexpr (F == E2M1) *reinterpret_cast<uint32_t*>(to) = c.lo;
    else *reinterpret_cast<uint2*>(to) = uint2{c.lo, c.hi};
    if (u % 4 == 0) {
        const int b = (int)(u / 4);
        uint8_t* const s = a.scales + r * a.lds + (b >> 3) * a.group;
        s[b & 7] = (uint8_t)byte;
        if (b == a.blocks - 1)
            for (int k = a.blocks; k < a.width; ++k) s[k & 7] = 0;  // of the same 8
    }
}

template <int F, typename T> __global__ __launch_bounds__(256) void pack_rows_kernel(BlockRows a) { pack_eight<F, T>(a, blockIdx.x * 256 + threadIdx.x); }

// The i-th 8 elements of out, rows of `len` of T: dim or, with zeros past it, up to a
// multiple of 8.
template <int F, typename T> __device__ __forceinline__ void unpack_eight(const BlockRows& a, void* out, int64_t ldout, int len, uint32_t i) {
    const uint32_t per = (len + 7) / 8, r = i / per, u = i % per;
    if (r >= a.rows) return;
    const uint8_t* const from = a.codes + r * a.ldc + u * EIGHT_BYTES<F>;
    Codes c{0, 0};
    if constexpr (F == E2M1) {
        c.lo = *reinterpret_cast<const uint32_t*>(from);
    } else {
        const uint2 q = *reinterpret_cast<const uint2*>(from);
        c = Codes{q.x, q.y};
    }
    const float s = scale_value(a.scales[r * a.lds + u / 4]);
    store8(static_cast<T*>(out) + r * ldout + 8 * u, len - 8 * (int)u, in_range<T>(decode8<F>(c) * s));
}

template <int F, typename T> __global__ __launch_bounds__(256) void unpack_rows_kernel(BlockRows a, void* out, int64_t ldout, int len) {
    unpack_eight<F, T>(a, out, ldout, len, blockIdx.x * 256 + threadIdx.x);
}

// f(element type) of an fc_dtype.
template <typename G> inline void by_dtype(int dt, G&& f) {
    if (dt == FC_F32) f(float{});
    else if (dt == FC_F16) f((_Float16)0);
    else f((__bf16)0.f);
}

template <int F> inline void pack_rows(BlockRows a, int dt, hipStream_t s) {
    const int64_t ex = dtype_bytes(dt), all = a.rows;
    by_launches(all, 4 * a.blocks, [&](int64_t r0, int64_t count) {
        BlockRows b = a;
        b.x = static_cast<const char*>(a.x) + r0 * a.ldx * ex;
        b.codes += r0 * a.ldc;
        b.scales += r0 * a.lds;
        b.rows = count;
        by_dtype(dt, [&](auto t) { pack_rows_kernel<F, decltype(t)><<<(unsigned)ceil_div(count * 4 * a.blocks, 256), 256, 0, s>>>(b); });
    });
}

template <int F> inline void unpack_rows(BlockRows a, void* out, int dt, int64_t ldout, int len, hipStream_t s) {
    const int64_t ex = dtype_bytes(dt), per = ceil_div(len, 8);
    by_launches(a.rows, per, [&](int64_t r0, int64_t count) {
        BlockRows b = a;
        b.codes += r0 * a.ldc;
        b.scales += r0 * a.lds;
        b.rows = count;
        void* const to = static_cast<char*>(out) + r0 * ldout * ex;
        by_dtype(dt, [&](auto t) { unpack_rows_kernel<F, decltype(t)><<<(unsigned)ceil_div(count * per, 256), 256, 0, s>>>(b, to, ldout, len); });
    });
}

}  // namespace fc
