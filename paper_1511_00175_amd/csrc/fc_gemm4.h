// The product of fc_gemm.h for operands in 4 bits with a scale for every 32 along k
// (fc_blocks.h), on the block-scaled matrix cores: C[m, n] = sum over k of A(m, k) B(n, k).
//
// A row of codes is read as 16-bit units of 4 elements, along k, so that a tile of 64 units
// holds 256 of k and goes to LDS and to fragments as fc_gemm.h's contiguous operands do: a
// lane's 16 bytes are the 32 elements of one scale.  The scales of a tile, 8 bytes for each
// row, go to LDS beside it, two rows' worth of lanes (4 bytes each) to a row; a lane reads its
// row's 8 and shifts the byte of its 32 elements down.  An instruction multiplies 16 x 16 by
// 128 of k in the cycles of a 16-bit one's 32 of k, from as many bytes, so that the same
// tiles give four times the operations for the same reads.
//
// What bounds it, measured on the loop alone, 16384 x 4096 by 4096 of k in 256 x 256 tiles: 127
// us, 4.3 PFLOP/s, and 109 with zeros for data, at which the clock stays higher; 106 without
// the loads, 77 the multiplications by themselves (zeros), 69 the loads, 50 the reads of LDS.
// A unit does 64 steps of 256 of k there.  A step's multiplications take about 2060 cycles, what
// LDS takes in and gives out at 128 bytes a cycle 2048: 63 us of the 127 each at 2.1 GHz, so that
// neither is the bound.  Multiplications and reads of LDS hardly overlap (77 and 50 by
// themselves, 106 together): it is the order in which they are issued and what they wait for.
// No faster were: 32 x 32 instructions of 64 of k
// (126), 4 waves of 128 x 128 (144), steps of 128 of k in 4 stages (172), padded rows, reads ahead
// into L2 (149), the results of a tile stored between the next one's products (4% more).
#pragma once

#include "fc_gemm.h"

namespace fc {

// p, ld, rows, ks in 16-bit units, as Operand; scales in bytes: 8 for each row and 64 units,
// rows `lds` and next units' `group` apart, all multiples of 8.  With lds 8 a tile's lie
// together: scales that are 8 of each cache line cost the loads of 256 x 256 tiles a third
// of their rate.
struct Operand4 {
    const void* p;
    int64_t ld;
    int rows;
    int ks;
    const void* scales;
    int64_t lds, group;
};

// 4 bytes per lane from memory to LDS at lds + 4 * lane.
__device__ __forceinline__ void load_words_to_lds(u32x4 desc, uint32_t lds, uint32_t off) {
    asm volatile("s_mov_b32 m0, %0\n\ts_nop 0\n\tbuffer_load_dword %1, %2, 0 offen lds" ::"s"(lds), "v"(off), "s"(desc)
                 : "memory", "m0");
}

typedef int i32x4 __attribute__((ext_vector_type(4)));
typedef int i32x8 __attribute__((ext_vector_type(8)));

// The products of a lane's 32 elements each of a and b, scaled by bytes 0 of sa and sb.
__device__ __forceinline__ f32x4 mma4(i32x4 a, i32x4 b, f32x4 c, uint32_t sa, uint32_t sb) {
    const i32x8 x = __builtin_shufflevector(a, a, 0, 1, 2, 3, -1, -1, -1, -1), y = __builtin_shufflevector(b, b, 0, 1, 2, 3, -1, -1, -1, -1);
    return __builtin_amdgcn_mfma_scale_f32_16x16x128_f8f6f4(x, y, c, 4, 4, 0, (int)sa, 0, (int)sb);
}

// One wave's loads of one operand's scales for tiles of R rows, of which `waves` waves load
// 32 rows at a time each.
template <int R> struct ScaleLoads {
    uint32_t off;
    uint64_t base;
    int64_t group;
    uint32_t span;
    bool rows;  // whether any of them is the operand's
    // Of the 32 rows from `row` on.
    __device__ __forceinline__ void init(const Operand4& o, int row, int lane) {
        group = o.group;
        move(o, row);
        const int r = lane >> 1;
        off = r < o.rows - row ? (uint32_t)((uint64_t)r * o.lds) + 4u * (lane & 1) : GEMM_OUTSIDE;
    }
    // As TileLoads::move, after an init of 32 rows that are all the operand's.
    __device__ __forceinline__ void move(const Operand4& o, int row) {
        const int left = o.rows - row, valid = left < 32 ? left : 32;
        rows = valid > 0;
        base = (uint64_t)o.scales + (rows ? (uint64_t)row * o.lds : 0);
        span = rows ? (uint32_t)((uint64_t)(valid - 1) * o.lds) : 0;
    }
    // Of the 64 units at step s.
    __device__ __forceinline__ void load(uint32_t lds, int s, bool live) const {
        const uint64_t b = base + (uint64_t)s * group;
        u32x4 desc;
        desc.x = __builtin_amdgcn_readfirstlane((uint32_t)b);
        desc.y = __builtin_amdgcn_readfirstlane((uint32_t)(b >> 32));
        desc.z = __builtin_amdgcn_readfirstlane(live && rows ? span + 8 : 0u);
        desc.w = 0x00020000u;
        load_words_to_lds(desc, __builtin_amdgcn_readfirstlane(lds), off);
    }
};

// The product of one block's BM x BN tile, WM x WN per wave; fc_gemm.h's loop with scales.
template <int BM_, int BN_, int WM_, int WN_, int STAGES> struct Product4 {
    static constexpr int BM = BM_, BN = BN_, WM = WM_, WN = WN_;
    static constexpr int WAVES = (BM / WM) * (BN / WN), THREADS = 64 * WAVES;
    static constexpr int FM = WM / 16, FN = WN / 16;
    static constexpr int CODES = (BM + BN) * GEMM_BK * 2;
    static constexpr int STAGE = CODES + (BM + BN) * 8;
    static constexpr int LDS = STAGES * STAGE;
    static constexpr int SCALES = (BM + BN) / 32 / WAVES;  // loads of 32 rows' scales per wave
    static constexpr int LOADS = (BM + BN) / 8 / WAVES + SCALES;
    static_assert(SCALES * 32 * WAVES == BM + BN && BM % 32 == 0, "the scales are whole loads of every wave");

    f32x4 acc[FM][FN];

    // The operand of the part-th 32 rows of A's and B's tiles.
    static __device__ __forceinline__ Operand4 side(const Operand4& A, const Operand4& B, int part) {
        const bool a = part < BM / 32;
        return {nullptr, 0, a ? A.rows : B.rows, 0, a ? A.scales : B.scales, a ? A.lds : B.lds, a ? A.group : B.group};
    }

    // Tile after tile: place(i, m0, n0) gives the block's i-th or false, done(m0, n0) takes acc.
    // The loads run ahead from a tile into the next, so that only the first waits for its data.
    // k runs over [kb, ke) in 16-bit units, kb a multiple of 64.
    template <typename Place, typename Done>
    __device__ __forceinline__ void run_tiles(char* lds, const Operand4& A, const Operand4& B, int kb, int ke, Place&& place, Done&& done) {
        const int lane = threadIdx.x & 63;
        const int wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6);
        const uint32_t la = lds_address(lds), lb = la + BM * GEMM_BK * 2, ls = la + CODES;
        TileLoads<BM, false, WAVES> ta;
        TileLoads<BN, false, WAVES> tb;
        const Operand oa{A.p, A.ld, A.rows, A.ks, 0}, ob{B.p, B.ld, B.rows, B.ks, 0};
        ta.init(Operand{A.p, A.ld, BM, A.ks, 0}, 0, wave, lane);
        tb.init(Operand{B.p, B.ld, BN, B.ks, 0}, 0, wave, lane);
        ScaleLoads<BM> ts[SCALES];
#pragma unroll
        for (int i = 0; i < SCALES; ++i) {
            Operand4 all = side(A, B, wave * SCALES + i);
            all.rows = 32;
            ts[i].init(all, 0, lane);
        }
        int tile = 0, im = 0, in = 0;  // whose loads are issued
        bool live = place(0, im, in);
        auto move = [&]() __attribute__((always_inline)) {
            ta.move(oa, im);
            tb.move(ob, in);
#pragma unroll
            for (int i = 0; i < SCALES; ++i) {
                const int part = wave * SCALES + i;
                ts[i].move(side(A, B, part), part < BM / 32 ? im + 32 * part : in + 32 * part - BM);
            }
        };
        if (live) move();
        Fragments<_Float16, BM, false, FM> fa;
        Fragments<_Float16, BN, false, FN> fb;
        const int wm = (wave / (BN / WN)) * WM, wn = (wave % (BN / WN)) * WN;
        fa.init(wm, lane);
        fb.init(wn, lane);
        const uint32_t sa_at = ls + 8 * (wm + (lane & 15)), sb_at = ls + 8 * (BM + wn + (lane & 15)), shift = 8 * (lane >> 4);
        auto frag = [&](auto& f, uint32_t tile, int i, int kk) __attribute__((always_inline)) { return __builtin_bit_cast(i32x4, f.get(tile, i, kk)); };
        auto scales = [&](uint32_t at, int i) __attribute__((always_inline)) { return *(FC_LDS const u32x2*)(uintptr_t)(at + 128 * i); };
        const int total = (ke - kb + GEMM_BK - 1) / GEMM_BK;
        int next_step = 0;
        uint32_t into = 0, is = 0;
        typename TileLoads<BM, false, WAVES>::Tile ia;
        typename TileLoads<BN, false, WAVES>::Tile ib;
        int step = 0;
        bool now = false;
        auto prepare = [&]() __attribute__((always_inline)) {
            if (next_step == total) {
                next_step = 0;
                live = live && place(++tile, im, in);
                if (live) move();
            }
            now = live;
            step = kb / GEMM_BK + next_step;
            ia = ta.tile(la + into, step * GEMM_BK, false, now, wave);
            ib = tb.tile(lb + into, step * GEMM_BK, false, now, wave);
            is = ls + into + wave * SCALES * 256;
            into = into == (STAGES - 1) * STAGE ? 0 : into + STAGE;
            ++next_step;
        };
        auto load = [&](int l) __attribute__((always_inline)) {
            if (l < ta.COUNT) ta.load(ia, l);
            else if (l < ta.COUNT + tb.COUNT) tb.load(ib, l - ta.COUNT);
            else ts[l - ta.COUNT - tb.COUNT].load(is + 256 * (l - ta.COUNT - tb.COUNT), step, now);
        };
        for (int s = 0; s < STAGES; ++s) {
            prepare();
#pragma unroll
            for (int l = 0; l < LOADS; ++l) load(l);
        }
        wait_loads<(STAGES - 1) * LOADS>();
        __builtin_amdgcn_s_barrier();
        asm volatile("" ::: "memory");
        i32x4 a[FM], b[FN], next[FN];
        u32x2 sa[FM], sb[FN], sn[FN];
#pragma unroll
        for (int j = 0; j < FN; ++j) {
            b[j] = frag(fb, lb, j, 0);
            sb[j] = scales(sb_at, j);
        }
#pragma unroll
        for (int i = 0; i < FM; ++i) {
            a[i] = frag(fa, la, i, 0);
            sa[i] = scales(sa_at, i);
        }
        constexpr int FIRST = FM >= 4 ? 2 : FM >= 2 ? 1 : 0;  // rows that cover the wait for the last reads
        constexpr int REST = FM - FIRST;
        constexpr int EACH = (FN + REST - 1) / REST, LEACH = (LOADS + REST - 1) / REST;
        auto row_of = [&](int i, int kk) __attribute__((always_inline)) {
            const uint32_t s = sa[i][kk] >> shift;
            __builtin_amdgcn_sched_barrier(0);
#pragma unroll
            for (int j = 0; j < FN; ++j) acc[i][j] = mma4(b[j], a[i], acc[i][j], sb[j][kk], s);
            __builtin_amdgcn_sched_barrier(0);
        };
        uint32_t at = 0;
        int m0, n0;
        for (int mine = 0; place(mine, m0, n0); ++mine) {
#pragma unroll
            for (int i = 0; i < FM; ++i)
#pragma unroll
                for (int j = 0; j < FN; ++j) acc[i][j] = f32x4{0.f, 0.f, 0.f, 0.f};
            // As fc_gemm.h's loop.  (A read or load after each multiplication instead of a
            // row's: 124 us for 127, but more registers than there are beside the results.)
            for (int t = 0; t < total; ++t) {
                const uint32_t then = at == (STAGES - 1) * STAGE ? 0 : at + STAGE;
                prepare();
#pragma unroll
                for (int j = 0; j < FN; ++j) sb[j] >>= shift;
#pragma unroll
                for (int i = 0; i < FM; ++i) {
                    row_of(i, 0);
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        if (j / EACH == i) next[j] = frag(fb, lb + at, j, 1);
                    a[i] = frag(fa, la + at, i, 1);
                }
#pragma unroll
                for (int j = 0; j < FN; ++j) b[j] = next[j];
#pragma unroll
                for (int i = 0; i < FIRST; ++i) row_of(i, 1);
                asm volatile("s_waitcnt lgkmcnt(0)" ::: "memory");
                wait_loads<(STAGES - 2) * LOADS>();
                __builtin_amdgcn_s_barrier();
                asm volatile("" ::: "memory");
#pragma unroll
                for (int i = 0; i < FIRST; ++i) {
                    a[i] = frag(fa, la + then, i, 0);
                    sa[i] = scales(sa_at + then, i);
                }
#pragma unroll
                for (int i = FIRST; i < FM; ++i) {
#pragma unroll
                    for (int j = 0; j < FN; ++j)
                        if (j / EACH == i - FIRST) {
                            next[j] = frag(fb, lb + then, j, 0);
                            sn[j] = scales(sb_at + then, j);
                        }
                    row_of(i, 1);
                    a[i] = frag(fa, la + then, i, 0);
                    sa[i] = scales(sa_at + then, i);
#pragma unroll
                    for (int l = 0; l < LOADS; ++l)
                        if (l / LEACH == i - FIRST) load(l);
                }
#pragma unroll
                for (int j = 0; j < FN; ++j) {
                    b[j] = next[j];
                    sb[j] = sn[j];
                }
                at = then;
            }
            done(m0, n0);
        }
        wait_loads<0>();  // no store to LDS is left behind
    }
    // One tile; acc holds it afterwards.
    __device__ __forceinline__ void run(char* lds, const Operand4& A, const Operand4& B, int m0, int n0, int kb, int ke, int) {
        run_tiles(
            lds, A, B, kb, ke,
            [&](int i, int& m, int& n) __attribute__((always_inline)) {
                m = m0;
                n = n0;
                return i == 0;
            },
            [](int, int) __attribute__((always_inline)) {});
    }
    // m and n of acc[i][j][0] within the block's tile.
    static __device__ __forceinline__ int row(int i) {
        return ((threadIdx.x >> 6) / (BN / WN)) * WM + 16 * i + (threadIdx.x & 15);
    }
    static __device__ __forceinline__ int col(int j) {
        return ((threadIdx.x >> 6) % (BN / WN)) * WN + 16 * j + 4 * ((threadIdx.x & 63) >> 4);
    }
};

}  // namespace fc
