// Matrices in microscaled 4-bit floating point, and products of them (fc_lm.h; the format
// is described in fc_blocks.h, the product in fc_gemm4.h).
//
//   out[t, r] (+)= scale sum over k of a[t, k] b[r, k]
//
// 2 tokens rows dim operations on the block-scaled matrix cores, from 0.53 bytes an element;
// packing is bound by memory, and a large product by the matrix cores (fc_gemm4.h).  In us:
// 8192 tokens, 8192 x 2048, bf16: the weight 15.8, the inputs with both operands' scales
// brought in order 12.5 (44 MB, 3.6 TB/s), the product 81 (3.4 PFLOP/s; its 134 MB of results
// alone take 19 to 28); 16384 tokens, 4096 x 4096, fp16: the weight by its columns 14, the inputs
// 42 (177 MB, 4.2 TB/s), the product 136 to 156 by card and pass (3.5 to 4.0 PFLOP/s).
#include "fc_blocks.h"
#include "fc_gemm4.h"
#include "fc_products.h"

namespace {

using fc::Operand4;

constexpr int64_t LD_LIMIT = 1 << 21, TOKENS_LIMIT = (int64_t)1 << 31;
constexpr int64_t CHUNK = MXFP_CHUNK;

// ---- columns to blocks ---------------------------------------------------------------

// A block's tile is 256 of x's rows (a packed row's elements) by 128 of its columns (packed
// rows).  A thread holds 8 columns of 8 rows, four threads a block of the format for each of
// the columns; the codes go through LDS, so that a packed row's 128 bytes are stored together.
struct ColumnArgs {
    const void* x;
    int64_t ldx;
    uint8_t* codes;
    int64_t ldc;
    uint8_t* scales;
    int64_t lds;
    int rows, dim, blocks;   // packed rows
};

constexpr int COLUMNS = 128;

template <typename T> __global__ __launch_bounds__(512) void pack_columns_kernel(ColumnArgs a) {
    __shared__ __align__(16) uint32_t tile[COLUMNS][33];  // codes of 256 elements of a packed row
    __shared__ uint8_t scale[COLUMNS][8];
    const int lane = threadIdx.x & 63, kb = threadIdx.x >> 6, sub = lane >> 4, c = 8 * (lane & 15);
    const int k0 = blockIdx.x * 256 + 32 * kb + 8 * sub, r0 = blockIdx.y * COLUMNS, left = a.rows - r0 - c;
    const T* const p = static_cast<const T*>(a.x) + (int64_t)k0 * a.ldx + r0 + c;
    typename fc::Eight<T>::vec v[8];
#pragma unroll
    for (int e = 0; e < 8; ++e) {
        v[e] = typename fc::Eight<T>::vec{};
        if (k0 + e >= a.dim) continue;
        if (left >= 8) {
            v[e] = fc::raw8(p + e * a.ldx);
        } else {
#pragma unroll
            for (int q = 0; q < 7; ++q)
                if (q < left) v[e][q] = p[e * a.ldx + q];
        }
    }
#pragma unroll
    for (int q = 0; q < 8; ++q) {
        fc::f32x8 x;
#pragma unroll
        for (int e = 0; e < 8; ++e) x[e] = (float)v[e][q];
        uint32_t most = fc::most_of(x);
        most = max(most, (uint32_t)__shfl_xor((int)most, 16));
        most = max(most, (uint32_t)__shfl_xor((int)most, 32));
        const uint32_t byte = fc::scale_byte<fc::E2M1>(most);
        tile[c + q][4 * kb + sub] = fc::encode8<fc::E2M1>(x, fc::scale_inverse(byte)).lo;
        if (sub == 0) scale[c + q][kb] = (uint8_t)byte;
    }
    __syncthreads();
    const int first = blockIdx.x * 8;  // block of the format
#pragma unroll
    for (int i = 0; i < 2; ++i) {
        const int at = threadIdx.x + 512 * i, r = at >> 3, b = at & 7;  // 16 bytes each
        if (r0 + r >= a.rows) continue;
        if (first + b < a.blocks)
            *reinterpret_cast<uint4*>(a.codes + (int64_t)(r0 + r) * a.ldc + 16 * (first + b)) =
                uint4{tile[r][4 * b], tile[r][4 * b + 1], tile[r][4 * b + 2], tile[r][4 * b + 3]};
        a.scales[(int64_t)(r0 + r) * a.lds + first + b] = first + b < a.blocks ? scale[r][b] : 0;
    }
}

// Scales of a packed matrix in the order in which 256 x 256 tiles read them: all rows' first 8,
// all rows' next 8.
struct ScaleArgs {
    const uint8_t* from;
    int64_t lds;
    uint64_t* to;
    int64_t rows;
    int groups;
};

__device__ __forceinline__ void reorder_scales(const ScaleArgs& a, int64_t i) {
    const int64_t r = i % a.rows, g = i / a.rows;
    if (g < a.groups) a.to[i] = *reinterpret_cast<const uint64_t*>(a.from + r * a.lds + 8 * g);
}

__global__ __launch_bounds__(256) void scales_kernel(ScaleArgs a) { reorder_scales(a, (int64_t)blockIdx.x * 256 + threadIdx.x); }

// A product's inputs packed and its weight's scales reordered, in one launch: the first
// blocks pack.
template <typename T> __global__ __launch_bounds__(256) void inputs_kernel(fc::BlockRows a, unsigned packing, ScaleArgs b) {
    if (blockIdx.x < packing) fc::pack_eight<fc::E2M1, T>(a, blockIdx.x * 256 + threadIdx.x);
    else reorder_scales(b, (int64_t)(blockIdx.x - packing) * 256 + threadIdx.x);
}

// ---- the product ------------------------------------------------------------------------

using Wide4 = fc::Product4<256, 256, 128, 64, 2>;
using Half4 = fc::Product4<128, 128, 64, 64, 2>;
using Small4 = fc::Product4<64, 64, 32, 32, 4>;

// A block goes through every gridDim.x-th tile, in the order of result_kernel's.
template <typename P, typename T> __global__ __launch_bounds__(P::THREADS, P::THREADS / 256) void tiles_kernel(ResultArgs<Operand4> a) {
    const int count = a.tm * a.tn;
    P p;
    p.run_tiles(
        lds, a.a, a.b, 0, a.k,
        [&](int i, int& m0, int& n0) __attribute__((always_inline)) {
            const int at = blockIdx.x + i * gridDim.x;
            if (at >= count) return false;
            fc::tile_place(fc::xcd_order(at, count), a.tm, a.tn, 8, m0, n0);
            m0 *= P::BM;
            n0 *= P::BN;
            return true;
        },
        [&](int m0, int n0) __attribute__((always_inline)) { store_tile_as<P, false, T>(a, p, static_cast<T*>(a.out), a.ld, a.scale, m0, n0); });
}

template <typename P> void launch_tiles(ResultArgs<Operand4> a, hipStream_t s) {
    a.tm = (int)fc::ceil_div(a.m, P::BM);
    a.tn = (int)fc::ceil_div(a.n, P::BN);
    const unsigned grid = (unsigned)std::min<int64_t>(CUS, (int64_t)a.tm * a.tn);
    fc::by_dtype(a.dt, [&](auto t) { tiles_kernel<P, decltype(t)><<<grid, P::THREADS, P::LDS, s>>>(a); });
}

template <typename P> hipError_t prepare_tiles() {
    for (hipError_t e : {prepare<P>((const void*)tiles_kernel<P, float>), prepare<P>((const void*)tiles_kernel<P, f16>),
                         prepare<P>((const void*)tiles_kernel<P, bf16>)})
        if (e != hipSuccess) return e;
    return hipSuccess;
}

// ---- few tokens ---------------------------------------------------------------------------

// Up to 16 tokens by 16 rows of b to a block, whose waves share k in steps of 256 and add up
// through LDS.  b's elements are read once, so they go from memory to registers: a lane's 16
// bytes are its row's 32 elements of one scale.  The tokens are packed into LDS by every
// block, while its first steps of b are on their way; the other steps' loads wait until it is
// done, so that one token of 9216 takes twice what reading the weight does.  One token, fp16, us, other weights in
// the caches: 4096 x 9216 (20 MB) 8.5, 8192 x 2048 5.6, 65536 x 2048 (71 MB) 20.
struct FewArgs {
    Operand4 b;
    const void* x;
    int64_t ldx;
    int n, dim, blocks, width;
    float scale;
    void* out;
    int dt;
    int64_t ld;
    bool add;
};

// `tokens` rows of x packed into LDS by all threads of a block, rows of codes and of scales
// `row` and `scale_row` bytes apart; `after` rows of x follow them.  4 loads of a thread are on
// their way at a time, whole vectors but at the end of the last row.
template <typename X>
__device__ __forceinline__ void pack_tokens(const X* x, int64_t ldx, int tokens, int after, int dim, int blocks, char* codes, int row, char* scales, int scale_row) {
    typedef typename fc::Eight<X>::vec V;
    const uint32_t per = 4 * blocks, all = tokens * per;
    for (uint32_t i0 = threadIdx.x; i0 < all; i0 += 4 * blockDim.x) {
        V v[4];
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t i = i0 + q * blockDim.x, t = i / per, u = i - t * per;
            const int left = dim - 8 * (int)u;
            v[q] = V{};
            if (i >= all || left <= 0) continue;
            const X* const p = x + t * ldx + 8 * u;
            if (left >= 8 || (tokens + after - 1 - (int)t) * ldx + left >= 8) {
                v[q] = fc::raw8(p);
            } else {
#pragma unroll
                for (int e = 0; e < 7; ++e)
                    if (e < left) v[q][e] = p[e];
            }
        }
#pragma unroll
        for (int q = 0; q < 4; ++q) {
            const uint32_t i = i0 + q * blockDim.x, t = i / per, u = i - t * per;
            if (i >= all) break;  // the same for the 4 threads of a block of the format
            const int left = dim - 8 * (int)u;
            fc::f32x8 f = __builtin_convertvector(v[q], fc::f32x8);
            if (left < 8) {
#pragma unroll
                for (int e = 0; e < 8; ++e) f[e] = e < left ? f[e] : 0.f;
            }
            const uint32_t byte = fc::scale_byte<fc::E2M1>(fc::most_of_four(fc::most_of(f)));
            *reinterpret_cast<uint32_t*>(codes + t * row + 4 * u) = fc::encode8<fc::E2M1>(f, fc::scale_inverse(byte)).lo;
            if (u % 4 == 0) scales[t * scale_row + u / 4] = (char)byte;
        }
    }
}

constexpr int AHEAD = 3;     // steps of a wave on their way at a time

template <typename X> __global__ __launch_bounds__(1024) void few_kernel(FewArgs a) {
    typedef fc::i32x4 V;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), waves = blockDim.x >> 6, r = lane & 15, g = lane >> 4;
    const int r0 = blockIdx.x * 16, steps = a.width / 8;
    struct Step {
        V code[2];
        uint32_t scale[2];
    };
    // A row's codes and scales at step s; zeros past its blocks.
    auto fetch = [&](const char* codes, const char* scales, int s) __attribute__((always_inline)) {
        Step q{};
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            const int block = 8 * s + 4 * h + g;
            if (block < a.blocks) {
                q.code[h] = *reinterpret_cast<const V*>(codes + 16 * block);
                q.scale[h] = *reinterpret_cast<const uint8_t*>(scales + block);
            }
        }
        return q;
    };
    const int row = min(r0 + r, a.b.rows - 1);
    const char* const bc = static_cast<const char*>(a.b.p) + (int64_t)row * 2 * a.b.ld;
    const char* const bs = static_cast<const char*>(a.b.scales) + (int64_t)row * a.b.lds;
    Step b[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) b[u] = wave + u * waves < steps ? fetch(bc, bs, wave + u * waves) : Step{};
    const int codes = 16 * a.blocks;                        // bytes of a token's
    char* const xc = lds;                                   // [token][codes]
    char* const xs = lds + a.n * codes;                     // [token][width]
    pack_tokens(static_cast<const X*>(a.x), a.ldx, a.n, 0, a.dim, a.blocks, xc, codes, xs, a.width);
    __syncthreads();
    fc::f32x4 acc{0.f, 0.f, 0.f, 0.f};
    for (int s0 = wave; s0 < steps; s0 += AHEAD * waves) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int s = s0 + u * waves;
            if (s >= steps) break;
            const Step x = r < a.n ? fetch(xc + r * codes, xs + r * a.width, s) : Step{};
#pragma unroll
            for (int h = 0; h < 2; ++h) acc = fc::mma4(b[u].code[h], x.code[h], acc, b[u].scale[h], x.scale[h]);
            const int then = s + AHEAD * waves;
            b[u] = then < steps ? fetch(bc, bs, then) : Step{};
        }
    }
    __syncthreads();  // the packed tokens are done with
    // acc[e]: row 4 g + e of b, token r
    float(*const part)[16][16 + 1] = reinterpret_cast<float(*)[16][16 + 1]>(lds);  // [wave][token][row]
#pragma unroll
    for (int e = 0; e < 4; ++e) part[wave][r][4 * g + e] = acc[e];
    __syncthreads();
    const int t = threadIdx.x >> 4, c = threadIdx.x & 15;
    if (t >= a.n || r0 + c >= a.b.rows) return;
    float v = 0.f;
    for (int w = 0; w < waves; ++w) v += part[w][t][c];
    v *= a.scale;
    const int64_t at = (int64_t)t * a.ld + r0 + c;
    if (a.add) v += load_one(a.out, a.dt, at);
    store_one(a.out, a.dt, at, v);
}

template <typename X> void launch_few(const FewArgs& a, hipStream_t s) {
    const int blocks = (int)fc::ceil_div(a.b.rows, 16);
    int waves = 16;  // as many as the chip holds of all blocks at once, 24 to a compute unit, at least 4 and at most a step each
    while (waves > 4 && (waves * blocks > 24 * CUS || waves > a.width / 8)) waves /= 2;
    const int bytes = std::max<int>(waves * 16 * 17 * 4, a.n * (16 * a.blocks + a.width));
    few_kernel<X><<<blocks, 64 * waves, bytes, s>>>(a);
}

// ---- few tiles ----------------------------------------------------------------------------

// 64 tokens by 64 rows of b to a block, in one launch: the block packs its tokens into LDS, and
// its waves, 32 x 32 of the tile each, share k in steps of 128 by fours and add up through LDS.
// b's elements go from memory to registers as few_kernel's do.  What bounds it is the packing,
// done again for every 64 rows of b.
constexpr int SMALL = MXFP_SMALL, PARTS = 4, SMALL_WAVES = 4 * PARTS, SMALL_AHEAD = 2;
constexpr int SMALL_LDS = PARTS * SMALL * (SMALL + 4) * 4;  // the parts' sums

// LDS of a token's codes: an odd number of 16 bytes, so that 16 rows' lie in different banks.
__host__ __device__ constexpr int small_row(int blocks) { return 16 * (blocks | 1); }
static_assert(SMALL * (small_row(MXFP_SMALL_DIM / fc::BLOCK) + MXFP_SMALL_DIM / fc::BLOCK + 3) <= SMALL_LDS, "the packed tokens fit");

template <typename X> __global__ __launch_bounds__(64 * SMALL_WAVES) void small_kernel(FewArgs a, int tm, int tn) {
    typedef fc::i32x4 V;
    const int lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), part = wave >> 2, r = lane & 15, g = lane >> 4;
    int ti, tj;
    fc::tile_place(fc::xcd_order(blockIdx.x, tm * tn), tm, tn, 8, ti, tj);
    const int t0 = ti * SMALL, r0 = tj * SMALL, wm = 32 * ((wave >> 1) & 1), wn = 32 * (wave & 1);
    const int steps = (a.blocks + 3) / 4, tokens = min(SMALL, a.n - t0);
    struct Rows {
        V code[2];
        uint32_t scale[2];
    };
    const char *bc[2], *bs[2];
#pragma unroll
    for (int j = 0; j < 2; ++j) {
        const int row = min(r0 + wn + 16 * j + r, a.b.rows - 1);
        bc[j] = static_cast<const char*>(a.b.p) + (int64_t)row * 2 * a.b.ld;
        bs[j] = static_cast<const char*>(a.b.scales) + (int64_t)row * a.b.lds;
    }
    auto fetch = [&](int s) __attribute__((always_inline)) {
        Rows q{};
        const int block = 4 * s + g;
        if (s < steps && block < a.blocks) {
#pragma unroll
            for (int j = 0; j < 2; ++j) {
                q.code[j] = *reinterpret_cast<const V*>(bc[j] + 16 * block);
                q.scale[j] = *reinterpret_cast<const uint8_t*>(bs[j] + block);
            }
        }
        return q;
    };
    Rows b[SMALL_AHEAD];
#pragma unroll
    for (int u = 0; u < SMALL_AHEAD; ++u) b[u] = fetch(part + PARTS * u);
    const int row = small_row(a.blocks), scales = (a.blocks + 3) / 4 * 4;
    char* const xc = lds;                                   // [token][row]
    char* const xs = lds + SMALL * row;                     // [token][scales]
    pack_tokens(static_cast<const X*>(a.x) + t0 * a.ldx, a.ldx, tokens, a.n - t0 - tokens, a.dim, a.blocks, xc, row, xs, scales);
    __syncthreads();
    fc::f32x4 acc[2][2]{};
    for (int s0 = part; s0 < steps; s0 += PARTS * SMALL_AHEAD) {
#pragma unroll
        for (int u = 0; u < SMALL_AHEAD; ++u) {
            const int s = s0 + PARTS * u;
            if (s >= steps) break;
            const int block = 4 * s + g;
#pragma unroll
            for (int i = 0; i < 2; ++i) {
                const int t = wm + 16 * i + r;
                V code{};
                uint32_t scale = 0;
                if (block < a.blocks && t < tokens) {
                    code = *reinterpret_cast<const V*>(xc + t * row + 16 * block);
                    scale = *reinterpret_cast<const uint8_t*>(xs + t * scales + block);
                }
#pragma unroll
                for (int j = 0; j < 2; ++j) acc[i][j] = fc::mma4(b[u].code[j], code, acc[i][j], b[u].scale[j], scale);
            }
            b[u] = fetch(s + PARTS * SMALL_AHEAD);
        }
    }
    __syncthreads();  // the packed tokens are done with
    float(*const sums)[SMALL][SMALL + 4] = reinterpret_cast<float(*)[SMALL][SMALL + 4]>(lds);  // [part][token][row]
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) *reinterpret_cast<fc::f32x4*>(&sums[part][wm + 16 * i + r][wn + 16 * j + 4 * g]) = acc[i][j];
    __syncthreads();
    const int t = threadIdx.x >> 4, c = 4 * (threadIdx.x & 15), left = a.b.rows - r0 - c;
    if (t >= tokens || left <= 0) return;
    fc::f32x4 v{};
#pragma unroll
    for (int q = 0; q < PARTS; ++q) v += *reinterpret_cast<const fc::f32x4*>(&sums[q][t][c]);
    v = v * a.scale;
    const int64_t to = (int64_t)(t0 + t) * a.ld + r0 + c;
    if (a.add) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) v[e] += load_one(a.out, a.dt, to + e);
    }
    store_four(a.out, a.dt, to, v, left);
}

hipError_t prepare_small() {
    for (const void* k : {(const void*)small_kernel<float>, (const void*)small_kernel<f16>, (const void*)small_kernel<bf16>}) {
        const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, SMALL_LDS);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

template <typename X> void launch_small(const FewArgs& a, hipStream_t s) {
    const int tm = (int)fc::ceil_div(a.n, SMALL), tn = (int)fc::ceil_div(a.b.rows, SMALL);
    small_kernel<X><<<tm * tn, 64 * SMALL_WAVES, SMALL_LDS, s>>>(a, tm, tn);
}

template <bool ADD> hipError_t prepare_all() {
    for (hipError_t e : {prepare<Wide4>((const void*)result_kernel<Wide4, ADD, Operand4>), prepare<Half4>((const void*)result_kernel<Half4, ADD, Operand4>),
                         prepare<Small4>((const void*)result_kernel<Small4, ADD, Operand4>), prepare_tiles<Wide4>(), prepare_small()})
        if (e != hipSuccess) return e;
    return hipSuccess;
}

template <bool ADD> void launch(int kind, const ResultArgs<Operand4>& g, hipStream_t s) {
    if constexpr (!ADD) {  // with it the registers do not hold the next tile's first fragments beside the results
        if (kind == WIDE4 && !g.sum) return launch_tiles<Wide4>(g, s);
    }
    if (kind == WIDE4) launch_result<Wide4, ADD, Operand4>(g, s);
    else if (kind == HALF4) launch_result<Half4, ADD, Operand4>(g, s);
    else launch_result<Small4, ADD, Operand4>(g, s);
}

}  // namespace

struct fc_mxfp {
    fc::CallOrder order;
    fc::DeviceBlock block;
    int64_t rows = 0, dim = 0, max_tokens = 0;
    int blocks = 0, width = 0;   // of a row: scales, bytes of scales
    int64_t sums = 0;            // mxfp_limit, of which mxfp_room floats are made
    uint8_t* codes = nullptr;    // linear's packed inputs
    uint8_t* scales = nullptr;   // theirs, or those of a product's, reordered
    uint8_t* b_scales = nullptr; // the weight's, reordered
    float* sum = nullptr;
};

namespace {

// A packed matrix of a call.
struct Packed {
    const void* codes;
    int64_t ldc;
    const void* scales;
    int64_t lds;
    int64_t rows;
    int64_t group = 8;  // from 8 scales of a row to its next
};

fc::Span codes_span(const fc_mxfp* p, const Packed& m, bool written) { return {m.codes, m.rows, 16 * (int64_t)p->blocks, m.ldc, 1, written}; }
fc::Span scales_span(const fc_mxfp* p, const Packed& m, bool written) { return {m.scales, m.rows, p->width, m.lds, 1, written}; }

// What check_spans does not look at.
int check_packed(const Packed& m) {
    if (m.ldc > LD_LIMIT || m.lds > LD_LIMIT) return FC_EINVAL;
    if (m.ldc % 16 || reinterpret_cast<uintptr_t>(m.codes) % 16 || m.lds % 8 || reinterpret_cast<uintptr_t>(m.scales) % 8) return FC_EALIGN;
    return FC_OK;
}

fc::BlockRows rows_of(const fc_mxfp* p, const void* x, int64_t ldx, const Packed& m) {
    return {x, ldx, static_cast<uint8_t*>(const_cast<void*>(m.codes)), m.ldc, static_cast<uint8_t*>(const_cast<void*>(m.scales)), m.lds, m.rows, (int)p->dim,
            p->blocks, p->width, m.group};
}

Operand4 operand(const fc_mxfp* p, const Packed& m, int64_t r0, int64_t count) {
    return {static_cast<const uint8_t*>(m.codes) + r0 * m.ldc, m.ldc / 2, (int)count, 8 * p->blocks, static_cast<const uint8_t*>(m.scales) + r0 * m.lds, m.lds, m.group};
}

Choice choice(const fc_mxfp* p, int64_t n) { return mxfp_choice(n, p->rows, p->dim, p->sums); }

// Whether scales go to the product in the order of its tiles.
bool reorders(const fc_mxfp* p, int64_t n) { return choice(p, n).kind == WIDE4; }

ScaleArgs reordered(const fc_mxfp* p, Packed& m, uint8_t* to) {
    const ScaleArgs a{static_cast<const uint8_t*>(m.scales), m.lds, reinterpret_cast<uint64_t*>(to), m.rows, p->width / 8};
    m.scales = to;
    m.lds = 8;
    m.group = 8 * m.rows;
    return a;
}

unsigned blocks_of(const ScaleArgs& a) { return (unsigned)fc::ceil_div(a.rows * a.groups, 256); }

// At most CHUNK rows of a.
void product(fc_mxfp* p, const Packed& a, const Packed& b, float scale, void* out, int dt, int64_t ld, bool add, hipStream_t s) {
    const Operand4 oa = operand(p, a, 0, a.rows), ob = operand(p, b, 0, b.rows);
    const Choice c = choice(p, a.rows);
    const bool split = c.splits > 1;
    ResultArgs<Operand4> g{};
    g.a = oa;
    g.b = ob;
    g.m = (int)a.rows;
    g.n = (int)b.rows;
    g.k = oa.ks;
    g.parts = 1;
    g.kper = c.steps * fc::GEMM_BK;
    g.scale = scale;
    g.out = out;
    g.dt = dt;
    g.ld = ld;
    g.sum = split ? p->sum : nullptr;
    if (add && !split) launch<true>(c.kind, g, s);
    else launch<false>(c.kind, g, s);
    if (split) join_splits(g, c.splits, add, s);
}

}  // namespace

extern "C" {

int fc_mxfp_create(fc_mxfp** plan, int64_t rows, int64_t dim, int64_t max_tokens) {
    if (!plan) return FC_EINVAL;
    *plan = nullptr;
    if (rows < 1 || rows > LD_LIMIT || dim < 1 || dim > LD_LIMIT || max_tokens < 0 || max_tokens >= TOKENS_LIMIT) return FC_EINVAL;
    return fc::no_throw([&] {
        fc_mxfp* p = new fc_mxfp;
        p->rows = rows;
        p->dim = dim;
        p->max_tokens = max_tokens;
        p->blocks = (int)fc::ceil_div(dim, fc::BLOCK);
        p->width = 8 * (int)fc::ceil_div(dim, 256);
        const int64_t c = std::min(max_tokens, CHUNK);
        p->sums = mxfp_limit(max_tokens, rows);
        fc::Layout at;
        const uint64_t o_codes = at.take(c * 16 * p->blocks), o_scales = at.take(c * p->width), o_b = at.take(rows * p->width), o_sum = at.take(mxfp_room(max_tokens, rows, dim) * 4);
        int rc = p->order.create();
        if (!rc) rc = fc::hip_code(prepare_all<false>());
        if (!rc) rc = fc::hip_code(prepare_all<true>());
        if (!rc) rc = p->block.create(at.size);
        if (rc) {
            fc_mxfp_destroy(p);
            return rc;
        }
        p->codes = reinterpret_cast<uint8_t*>(p->block.p + o_codes);
        p->scales = reinterpret_cast<uint8_t*>(p->block.p + o_scales);
        p->b_scales = reinterpret_cast<uint8_t*>(p->block.p + o_b);
        p->sum = reinterpret_cast<float*>(p->block.p + o_sum);
        *plan = p;
        return FC_OK;
    });
}

void fc_mxfp_destroy(fc_mxfp* p) {
    if (!p) return;
    p->block.destroy();
    p->order.destroy();
    delete p;
}

int fc_mxfp_pack(fc_mxfp* p, const void* x, int x_dtype, int64_t ld_x, int64_t rows, int transpose, void* codes, int64_t ld_codes, void* scales,
                 int64_t ld_scales, void* stream) {
    return fc::no_throw([&]() -> int {
        if (!p || rows < 0 || rows >= TOKENS_LIMIT) return FC_EINVAL;
        const Packed m{codes, ld_codes, scales, ld_scales, rows};
        const int bytes = fc::dtype_bytes(x_dtype);
        int rc = fc::check_spans({transpose ? fc::Span{x, p->dim, rows, ld_x, bytes, false} : fc::Span{x, rows, p->dim, ld_x, bytes, false}, codes_span(p, m, true),
                                  scales_span(p, m, true)});
        if (!rc) rc = check_packed(m);
        if (rc) return rc;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        bool note;
        rc = p->order.begin(s, note);
        if (rc) return rc;
        if (!transpose) {
            fc::pack_rows<fc::E2M1>(rows_of(p, x, ld_x, m), x_dtype, s);
        } else {
            const int64_t groups = fc::ceil_div(p->dim, 256), most = (int64_t)COLUMNS * 32768;  // a launch's blocks along y
            for (int64_t r0 = 0; r0 < rows; r0 += most) {
                const int64_t count = std::min(most, rows - r0);
                const ColumnArgs a{static_cast<const char*>(x) + r0 * bytes, ld_x, static_cast<uint8_t*>(codes) + r0 * ld_codes, ld_codes,
                                   static_cast<uint8_t*>(scales) + r0 * ld_scales, ld_scales, (int)count, (int)p->dim, p->blocks};
                const dim3 grid((unsigned)groups, (unsigned)fc::ceil_div(count, COLUMNS));
                fc::by_dtype(x_dtype, [&](auto t) { pack_columns_kernel<decltype(t)><<<grid, 512, 0, s>>>(a); });
            }
        }
        rc = fc::hip_code(hipGetLastError());
        p->order.done(s, note);
        return rc;
    });
}

int fc_mxfp_unpack(fc_mxfp* p, const void* codes, int64_t ld_codes, const void* scales, int64_t ld_scales, int64_t rows, void* out, int out_dtype,
                   int64_t ld_out, void* stream) {
    return fc::no_throw([&]() -> int {
        if (!p || rows < 0 || rows >= TOKENS_LIMIT) return FC_EINVAL;
        const Packed m{codes, ld_codes, scales, ld_scales, rows};
        int rc = fc::check_spans({codes_span(p, m, false), scales_span(p, m, false), {out, rows, p->dim, ld_out, fc::dtype_bytes(out_dtype), true}});
        if (!rc) rc = check_packed(m);
        if (rc) return rc;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        bool note;
        rc = p->order.begin(s, note);
        if (rc) return rc;
        fc::unpack_rows<fc::E2M1>(rows_of(p, nullptr, 0, m), out, out_dtype, ld_out, (int)p->dim, s);
        rc = fc::hip_code(hipGetLastError());
        p->order.done(s, note);
        return rc;
    });
}

int fc_mxfp_product(fc_mxfp* p, const void* a_codes, int64_t ld_a_codes, const void* a_scales, int64_t ld_a_scales, int64_t n, const void* b_codes,
                    int64_t ld_b_codes, const void* b_scales, int64_t ld_b_scales, float scale, void* out, int out_dtype, int64_t ld_out, int accumulate,
                    void* stream) {
    return fc::no_throw([&]() -> int {
        if (!p || n < 0 || n > p->max_tokens) return FC_EINVAL;
        const Packed a{a_codes, ld_a_codes, a_scales, ld_a_scales, n}, b{b_codes, ld_b_codes, b_scales, ld_b_scales, p->rows};
        const int bytes = fc::dtype_bytes(out_dtype);
        int rc = fc::check_spans({codes_span(p, a, false), scales_span(p, a, false), codes_span(p, b, false), scales_span(p, b, false),
                                  {out, n, p->rows, ld_out, bytes, true}});
        if (!rc) rc = check_packed(a);
        if (!rc) rc = check_packed(b);
        if (rc) return rc;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        bool note;
        rc = p->order.begin(s, note);
        if (rc) return rc;
        for (int64_t t0 = 0; t0 < n; t0 += CHUNK) {
            Packed at{static_cast<const char*>(a_codes) + t0 * ld_a_codes, ld_a_codes, static_cast<const char*>(a_scales) + t0 * ld_a_scales, ld_a_scales, std::min(CHUNK, n - t0)};
            Packed bt = b;
            if (reorders(p, at.rows)) {
                const ScaleArgs sa = reordered(p, at, p->scales), sb = reordered(p, bt, p->b_scales);
                scales_kernel<<<blocks_of(sa), 256, 0, s>>>(sa);
                scales_kernel<<<blocks_of(sb), 256, 0, s>>>(sb);
            }
            product(p, at, bt, scale, static_cast<char*>(out) + t0 * ld_out * bytes, out_dtype, ld_out, accumulate != 0, s);
        }
        rc = fc::hip_code(hipGetLastError());
        p->order.done(s, note);
        return rc;
    });
}

int fc_mxfp_linear(fc_mxfp* p, const void* x, int x_dtype, int64_t ld_x, int64_t n, const void* b_codes, int64_t ld_b_codes, const void* b_scales,
                   int64_t ld_b_scales, float scale, void* out, int out_dtype, int64_t ld_out, int accumulate, void* stream) {
    return fc::no_throw([&]() -> int {
        if (!p || n < 0 || n > p->max_tokens) return FC_EINVAL;
        const Packed b{b_codes, ld_b_codes, b_scales, ld_b_scales, p->rows};
        const int bytes = fc::dtype_bytes(out_dtype), xbytes = fc::dtype_bytes(x_dtype);
        int rc = fc::check_spans({{x, n, p->dim, ld_x, xbytes, false}, codes_span(p, b, false), scales_span(p, b, false), {out, n, p->rows, ld_out, bytes, true}});
        if (!rc) rc = check_packed(b);
        if (rc) return rc;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        bool note;
        rc = p->order.begin(s, note);
        if (rc) return rc;
        const bool few = mxfp_few(n, p->rows, p->dim);
        if (n && (few || mxfp_small(n, p->rows, p->dim))) {
            const FewArgs f{operand(p, b, 0, p->rows), x, ld_x, (int)n, (int)p->dim, p->blocks, p->width, scale, out, out_dtype, ld_out, accumulate != 0};
            fc::by_dtype(x_dtype, [&](auto t) { few ? launch_few<decltype(t)>(f, s) : launch_small<decltype(t)>(f, s); });
            n = 0;
        }
        for (int64_t t0 = 0; t0 < n; t0 += CHUNK) {
            Packed a{p->codes, 16 * (int64_t)p->blocks, p->scales, p->width, std::min(CHUNK, n - t0)}, bt = b;
            const void* const xt = static_cast<const char*>(x) + t0 * ld_x * xbytes;
            const int64_t eights = a.rows * 4 * p->blocks;
            if (reorders(p, a.rows)) {
                a.lds = 8;
                a.group = 8 * a.rows;
                const ScaleArgs sb = reordered(p, bt, p->b_scales);
                if (eights < fc::LAUNCH_THREADS) {
                    const unsigned packing = (unsigned)fc::ceil_div(eights, 256);
                    fc::by_dtype(x_dtype, [&](auto t) { inputs_kernel<decltype(t)><<<packing + blocks_of(sb), 256, 0, s>>>(rows_of(p, xt, ld_x, a), packing, sb); });
                } else {
                    fc::pack_rows<fc::E2M1>(rows_of(p, xt, ld_x, a), x_dtype, s);
                    scales_kernel<<<blocks_of(sb), 256, 0, s>>>(sb);
                }
            } else {
                fc::pack_rows<fc::E2M1>(rows_of(p, xt, ld_x, a), x_dtype, s);
            }
            product(p, a, bt, scale, static_cast<char*>(out) + t0 * ld_out * bytes, out_dtype, ld_out, accumulate != 0, s);
        }
        rc = fc::hip_code(hipGetLastError());
        p->order.done(s, note);
        return rc;
    });
}

}  // extern "C"
