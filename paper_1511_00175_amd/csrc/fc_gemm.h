// The matrix product under the operators: C[m, n] = sum over k of A(m, k) B(n, k)
// for 16-bit operands (fp16 or bf16) on the matrix cores, sums in fp32.
//
// An operand's tile is R rows (of C's m or n) by 64 of k, and its memory runs
// either along k ("contiguous") or along the rows ("slow": k is the slow axis):
// products with a transposed operand need no transposed copy.  A tile goes from
// memory to LDS without passing through registers (buffer loads with the lds
// modifier, 16 bytes per lane), STAGES tiles ahead of the one being multiplied.
// The hardware writes a wave's 64 x 16 bytes to consecutive LDS addresses, so
// the order that keeps LDS reads free of bank conflicts is made on the side of
// the memory addresses:
//   contiguous: row r's 8 chunks of 16 bytes are stored in order c ^ (r & 7);
//               a fragment is one 16-byte read per lane.
//   slow:       k's row of R elements is stored in blocks of 16 elements, block
//               b at b ^ h(k), h(k) = (k & 3) | ((k >> 3) & 3) << 2 (R not a power of
//               2: at (b + ((k >> 3) & 3)) mod R / 16); a fragment is two transposing
//               reads (ds_read_b64_tr_b16), which hand each lane 4 values along k
//               from 4 rows of 16 elements.
// Rows and k beyond the operand read as zero (the buffer descriptor's bounds).
//
// C is computed transposed (B's fragment is the instruction's first operand),
// so that a lane holds 4 neighbouring n of one m:
//   acc[i][j][e]: m = 16 i + (lane & 15), n = 16 j + 4 (lane >> 4) + e.
//
// Bound by the matrix cores for large tiles: 8192^3 of fp16 in 256 x 256 tiles of 8
// waves runs at 1.23 to 1.28 PFLOP/s, both for contiguous operands and with one of
// them slow (a library's product: 1.43).  On the way: reading a half tile's
// fragments before its multiplications and loading a tile at its start, 1.17; 4
// waves of 128 x 128 (half the LDS reads, but a single wave per SIMD that nothing
// covers at the barrier), 1.06; 128 x 128 tiles, 1.05.  Small tiles are bound by the
// time from a load to its data: 64 x 64 tiles on a full chip take 0.49 us per 64 of
// k with 2 stages, 0.24 with 4.  Besides its k loop a tile costs 9.5 us at 256 x 256,
// 7 at 192 x 192, 4.5 at 128 x 128 and 3 at 64 x 64 (the first loads and the
// results' stores), which decides for small ones where k is short.
#pragma once

#include <hip/hip_runtime.h>
#include <stdint.h>

namespace fc {

typedef float f32x4 __attribute__((ext_vector_type(4)));
typedef float f32x2 __attribute__((ext_vector_type(2)));
typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef uint32_t u32x2 __attribute__((ext_vector_type(2)));
typedef _Float16 f16x4 __attribute__((ext_vector_type(4)));
typedef _Float16 f16x8 __attribute__((ext_vector_type(8)));
typedef __bf16 b16x4 __attribute__((ext_vector_type(4)));
typedef __bf16 b16x8 __attribute__((ext_vector_type(8)));
typedef short s16x4 __attribute__((ext_vector_type(4)));
// Wherever elements may start: global memory takes any alignment.
typedef f32x4 f32x4_any __attribute__((aligned(4)));
typedef f16x4 f16x4_any __attribute__((aligned(2)));
typedef b16x4 b16x4_any __attribute__((aligned(2)));

#define FC_LDS __attribute__((address_space(3)))

template <typename T> struct Half;
template <> struct Half<_Float16> {
    typedef f16x4 v4;
    typedef f16x8 v8;
    static __device__ __forceinline__ f32x4 mma(v8 a, v8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_f16(a, b, c, 0, 0, 0);
    }
};
template <> struct Half<__bf16> {
    typedef b16x4 v4;
    typedef b16x8 v8;
    static __device__ __forceinline__ f32x4 mma(v8 a, v8 b, f32x4 c) {
        return __builtin_amdgcn_mfma_f32_16x16x32_bf16(a, b, c, 0, 0, 0);
    }
};

// A matrix operand: element (row, k) at p + row * ld + k (contiguous) or
// p + k * ld + row (slow), in elements.  p is 16-byte aligned and ld a multiple
// of 8; a contiguous operand's k extent is a multiple of 8 and a slow one's rows
// are readable up to the next multiple of 8.  `ks` is its k extent: beyond it the
// operand is zero.  256 ld < 2^30: offsets within a tile are 32 bits.  `lo` is
// where the second half of a value kept as a sum of two 16-bit numbers lies,
// from p (products of 3 parts).
struct Operand {
    const void* p;
    int64_t ld;
    int rows;
    int ks;
    int64_t lo;
};

constexpr int GEMM_BK = 64;
constexpr uint32_t GEMM_OUTSIDE = 0x7ffffff0u;  // an offset past every descriptor's bound

// LDS address of a pointer into it.
__device__ __forceinline__ uint32_t lds_address(const void* p) {
    return (uint32_t)(uintptr_t)(FC_LDS const char*)p;
}

// 16 bytes per lane from memory to LDS at lds + 16 * lane.  In asm, because the
// compiler would wait for every such load before any LDS read it cannot tell
// apart; the waits are the caller's.  It has no result in registers.  ONCE: of
// what no other block reads: it displaces nothing in the caches.
template <bool ONCE> __device__ __forceinline__ void load_to_lds(u32x4 desc, uint32_t lds, uint32_t off) {
    if constexpr (ONCE)
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen nt lds" ::"s"(lds), "v"(off), "s"(desc)
                     : "memory", "m0");
    else
        asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dwordx4 %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(desc)
                     : "memory", "m0");
}

template <int N> __device__ __forceinline__ void wait_loads() {
    asm volatile("s_waitcnt vmcnt(%0)" ::"n"(N) : "memory");
}

// Where a slow operand's block b of 16 elements of k's row lies (at most 64 of k
// apart: k, k + 4 and k + 32 agree in what is used of them).
template <int R> __device__ __forceinline__ int slow_block(int b, int k) {
    if constexpr ((R & (R - 1)) == 0) return b ^ (((k & 3) | ((k >> 3) & 3) << 2) & (R / 16 - 1));
    else return (b + ((k >> 3) & 3)) % (R / 16);
}
// The block that lies there.
template <int R> __device__ __forceinline__ int slow_block_at(int at, int k) {
    if constexpr ((R & (R - 1)) == 0) return slow_block<R>(at, k);
    else return (at + R / 16 - ((k >> 3) & 3)) % (R / 16);
}

// One wave's loads of one operand's tiles of R rows; `waves` waves share a tile.
template <int R, bool SLOW, int WAVES, bool ONCE = false> struct TileLoads {
    static constexpr int COUNT = R / 8 / WAVES;  // 1 KiB per load
    static_assert(COUNT * 8 * WAVES == R, "a tile is whole loads of every wave");
    uint32_t off[COUNT];
    uint32_t kpart;  // contiguous: the lane's first k within the tile
    uint64_t base;   // of the operand's tile row, k = 0
    uint64_t ldb;
    int64_t lob;
    int ks;
    uint32_t span;   // bytes from a k's base to the end of the tile's last valid row, k extent apart
    uint32_t tail;   // slow: bytes of a row from the tile's first column to the operand's last

    __device__ __forceinline__ void init(const Operand& o, int row0, int wave, int lane) {
        ldb = 2 * (uint64_t)o.ld;
        lob = 2 * o.lo;
        ks = o.ks;
        const int left = o.rows - row0;
        if constexpr (!SLOW) {
            const int chunk = (lane & 7) ^ (lane >> 3);
            kpart = 8 * chunk;
            base = (uint64_t)o.p + (uint64_t)row0 * ldb;
            const int valid = left < R ? left : R;
            span = (uint32_t)((uint64_t)(valid - 1) * ldb);
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int r = (wave * COUNT + i) * 8 + (lane >> 3);
                off[i] = (uint32_t)((uint64_t)r * ldb) + 16u * chunk;
                if (r >= valid) off[i] = GEMM_OUTSIDE;
            }
        } else {
            constexpr int SLOTS = R / 8;      // 16-byte slots per k
            base = (uint64_t)o.p + 2 * (uint64_t)row0;
            const int cols = (left + 7) & ~7;
            tail = 2u * (cols < R ? cols : R);
#pragma unroll
            for (int i = 0; i < COUNT; ++i) {
                const int at = (wave * COUNT + i) * 64 + lane, k = at / SLOTS, slot = at % SLOTS;
                const int col = slow_block_at<R>(slot >> 1, k) * 16 + (slot & 1) * 8;
                off[i] = 2 * col < (int)tail ? (uint32_t)((uint64_t)k * ldb) + 2u * col : GEMM_OUTSIDE;
            }
        }
    }
    // The loads of one tile: where from, where to.
    struct Tile {
        u32x4 desc;
        uint32_t to;
        bool past;  // contiguous: the lane's k is past the operand's
    };
    // The tile at k0 (below ks) into LDS at `lds`; `low`: of the second halves;
    // not `live`: zeros, from nowhere.
    __device__ __forceinline__ Tile tile(uint32_t lds, int k0, bool low, bool live, int wave) const {
        uint64_t b = base + (low ? (uint64_t)lob : 0);
        uint32_t records;
        if constexpr (!SLOW) {
            b += 2 * (uint64_t)k0;
            records = span + 2u * (ks - k0);
        } else {
            b += (uint64_t)k0 * ldb;
            const int left = ks - k0;
            records = (uint32_t)((uint64_t)((left < GEMM_BK ? left : GEMM_BK) - 1) * ldb) + tail;
        }
        Tile t;
        t.desc.x = __builtin_amdgcn_readfirstlane((uint32_t)b);
        t.desc.y = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
        t.desc.z = __builtin_amdgcn_readfirstlane(live ? records : 0u);
        t.desc.w = 0x00020000u;
        t.to = __builtin_amdgcn_readfirstlane(lds + wave * COUNT * 1024);
        t.past = !SLOW && k0 + (int)kpart >= ks;
        return t;
    }
    __device__ __forceinline__ void load(const Tile& t, int i) const {
        load_to_lds<ONCE>(t.desc, t.to + i * 1024, t.past ? GEMM_OUTSIDE : off[i]);
    }
};

// A wave's fragments of one operand's tile: F of 16 rows by 32 of k.
template <typename T, int R, bool SLOW, int F> struct Fragments {
    typedef typename Half<T>::v8 v8;
    uint32_t at[SLOW ? F : 1];
    __device__ __forceinline__ void init(int row, int lane) {
        const int i = lane & 15, g = lane >> 4;
        if constexpr (!SLOW) {
            at[0] = (row + i) * 128 + ((g ^ (i & 7)) << 4);
        } else {
#pragma unroll
            for (int f = 0; f < F; ++f)
                at[f] = (8 * g + (i >> 2)) * (2 * R) + (slow_block<R>((row >> 4) + f, 8 * g + (i >> 2)) << 5) + (i & 3) * 8;
        }
    }
    // Fragment f of the tile at LDS address `tile`, k from 32 kk on.
    __device__ __forceinline__ v8 get(uint32_t tile, int f, int kk) const {
        if constexpr (!SLOW) {
            return *(FC_LDS const v8*)(uintptr_t)((tile + f * 2048) + (at[0] ^ (kk << 6)));
        } else {
            typedef FC_LDS s16x4* P;
            const uint32_t a = tile + at[f] + kk * (64 * R);
            union {
                s16x4 s[2];
                v8 v;
            } u;
            u.s[0] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)a);
            u.s[1] = __builtin_amdgcn_ds_read_tr16_b64_v4i16((P)(uintptr_t)(a + 8 * R));
            return u.v;
        }
    }
};

// The product of one block's BM x BN tile, WM x WN per wave.  RUN > 0: sums are
// taken over runs of RUN tiles of k and then added, so that a long sum's rounding
// error grows with the root of RUN + tiles / RUN instead of that of tiles.  ONCE:
// every tile of B is read by one block only.
template <typename T_, int BM_, int BN_, int WM_, int WN_, bool AS, bool BS, int STAGES = 2, int RUN = 0, bool ONCE = false> struct Product {
    typedef T_ T;
    typedef typename Half<T>::v8 v8;
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int WAVES = (BM / WM) * (BN / WN), THREADS = 64 * WAVES;
    static constexpr int FM = WM / 16, FN = WN / 16;
    static constexpr int STAGE = (BM + BN) * GEMM_BK * 2;
    static constexpr int LDS = STAGES * STAGE;
    static constexpr int LOADS = (BM + BN) / 8 / WAVES;

    f32x4 acc[FM][FN];

    // Parts: 1; 2 where A is kept as a sum of two 16-bit numbers: low by B, then high
    // by B; 3 where both are: high by low, low by high, then high by high (the small
    // terms first, while the sums are small; low by low is below the result's last bit).
    // k runs over [kb, ke), kb below both operands' extents, and ke - kb a multiple
    // of 64 unless one of them ends there.
    __device__ __forceinline__ void run(char* lds, const Operand& A, const Operand& B, int m0, int n0, int kb, int ke, int parts) {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t la = lds_address(lds), lb = la + BM * GEMM_BK * 2;
        TileLoads<BM, AS, WAVES> ta;
        TileLoads<BN, BS, WAVES, ONCE> tb;
        ta.init(A, m0, wave, lane);
        tb.init(B, n0, wave, lane);
        Fragments<T, BM, AS, FM> fa;
        Fragments<T, BN, BS, FN> fb;
        fa.init((wave / (BN / WN)) * WM, lane);
        fb.init((wave % (BN / WN)) * WN, lane);
#pragma unroll
        for (int i = 0; i < FM; ++i)
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};

        f32x4 total_of[RUN ? FM : 1][RUN ? FN : 1];
        if constexpr (RUN > 0) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) total_of[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
        }

        const int per = (ke - kb + GEMM_BK - 1) / GEMM_BK, total = per * parts;
        int part = 0, k = kb, issued = 0, into = 0;
        typename TileLoads<BM, AS, WAVES>::Tile ia;
        typename TileLoads<BN, BS, WAVES, ONCE>::Tile ib;
        auto prepare = [&]() {
            const bool live = issued < total;
            ia = ta.tile(la + into, k, part == parts - 2, live, wave);
            ib = tb.tile(lb + into, k, parts == 3 && part == 0, live, wave);
            into = into == (STAGES - 1) * STAGE ? 0 : into + STAGE;
            k += GEMM_BK;
            if (k >= ke) {
                k = kb;
                ++part;
            }
            ++issued;
        };
        auto load = [&](int l) {
            if (l < ta.COUNT)
                ta.load(ia, l);
            else
                tb.load(ib, l - ta.COUNT);
        };
        // The multiplications of one half tile of k run while the fragments of the
        // next are read: a row's A fragment is replaced as soon as its row is done.
        // Between the two halves of a tile the block meets: its last reads of the
        // tile are done, so the loads of the tile STAGES later may overwrite it, and
        // the next tile has arrived.  Those loads are spread over the second half's
        // rows.  Past the last tile they store zeros that nobody reads, so that the
        // count of loads in flight is always the same.
        for (int s = 0; s < STAGES; ++s) {
            prepare();
#pragma unroll
            for (int l = 0; l < LOADS; ++l) load(l);
        }
        wait_loads<(STAGES - 1) * LOADS>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        v8 a[FM], b[FN], next[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) b[j] = fb.get(lb, j, 0);
#pragma unroll
        for (int i = 0; i < FM; ++i) a[i] = fa.get(la, i, 0);
        constexpr int FIRST = FM >= 4 ? 2 : FM >= 2 ? 1 : 0;  // rows that cover the wait for the last reads
        constexpr int REST = FM - FIRST;
        constexpr int EACH = (FN + REST - 1) / REST, LEACH = (LOADS + REST - 1) / REST;  // B fragments and loads per row
        auto row_of = [&](int i) {
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = Half<T>::mma(b[j], a[i], acc[i][j]);
            __builtin_amdgcn_sched_barrier(0);
        };
        uint32_t at = 0;
        for (int t = 0; t < total; ++t) {
            const uint32_t then = at == (STAGES - 1) * STAGE ? 0 : at + STAGE;
            prepare();
#pragma unroll
            for (int i = 0; i < FM; ++i) {
                row_of(i);
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    if (j / EACH == i) next[j] = fb.get(lb + at, j, 1);
                a[i] = fa.get(la + at, i, 1);
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) b[j] = next[j];
#pragma unroll
            for (int i = 0; i < FIRST; ++i) row_of(i);
            asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
            wait_loads<(STAGES - 2) * LOADS>();
            __builtin_amdgcn_s_barrier();
            asm volatile("" ::: "memory");
#pragma unroll
            for (int i = 0; i < FIRST; ++i) a[i] = fa.get(la + then, i, 0);
#pragma unroll
            for (int i = FIRST; i < FM; ++i) {
#pragma unroll
                for (int j = 0; j < FN; ++j)
                    if (j / EACH == i - FIRST) next[j] = fb.get(lb + then, j, 0);
                row_of(i);
                a[i] = fa.get(la + then, i, 0);
#pragma unroll
                for (int l = 0; l < LOADS; ++l)
                    if (l / LEACH == i - FIRST) load(l);
            }
#pragma unroll
            for (int j = 0; j < FN; ++j) b[j] = next[j];
            at = then;
            if constexpr (RUN > 0) {
                if (t % RUN == RUN - 1 || t == total - 1) {
                    const bool last = t == total - 1;
#pragma unroll
                    for (int i = 0; i < FM; ++i)
#pragma unroll
                        for (int j = 0; j < FN; ++j) {
                            total_of[i][j] += acc[i][j];
                            acc[i][j] = last ? total_of[i][j] : f32x4{0.f, 0.f, 0.f, 0.f};
                        }
                }
            }
        }
        wait_loads<0>();  // no store to LDS is left behind
    }
    // m and n of acc[i][j][0] within the block's tile.
    static __device__ __forceinline__ int row(int i) {
        return ((threadIdx.x >> 6) / (BN / WN)) * WM + 16 * i + (threadIdx.x & 15);
    }
    static __device__ __forceinline__ int col(int j) {
        return ((threadIdx.x >> 6) % (BN / WN)) * WN + 16 * j + 4 * ((threadIdx.x & 63) >> 4);
    }
};

// Block b of a launch of `count` tiles -> tile index such that every XCD (blocks
// b mod 8) works on neighbouring tiles, which then share its L2.
__device__ __forceinline__ int xcd_order(int b, int count) {
    const int x = b & 7, q = count >> 3, r = count & 7;
    return x * q + (x < r ? x : r) + (b >> 3);
}

// Tile index -> (tile row, tile column): groups of G rows, down the rows first.
__device__ __forceinline__ void tile_place(int t, int tm, int tn, int G, int& i, int& j) {
    const int g = t / (G * tn), first = g * G;
    const int h = tm - first < G ? tm - first : G;
    const int u = t - g * G * tn;
    i = first + u % h;
    j = u / h;
}

}  // namespace fc
