// Activations kept in 8 bits, and a weight's gradient from them (fc_lm.h; the formats are
// described in fc_blocks.h).
//
//   dw[o, i] (+)= scale sum over t of dy[t, o] x[t, i]
//
// Packing and unpacking are bound by memory: 32768 rows of 2048, fp16 and int8, 203 MB each way,
// 45 us (4.5 TB/s) and 31 (the codes, 71 MB, come from the caches after packing).
//
// The gradient is 2 tokens outs dim operations.  x is first unpacked to dy's type, in which
// its numbers are exact (but for what is out of fp16's range), and the product then takes
// both operands across their rows (fc_gemm.h), so that neither is transposed in memory.
// Unpacking is 12 us of 240 at 8192 tokens, 8192 x 2048, where 32 tiles read every part of x;
// the product is 228 to 264 by card and pass, 1.0 to 1.2 PFLOP/s, the matrix cores busy 59% of the
// cycles at 2.09 GHz.  Few tiles take one launch (small_kernel).
#include "fc_blocks.h"
#include "fc_products.h"

namespace {

constexpr int64_t ROWS_LIMIT = 1 << 21, LD_LIMIT = 1 << 21, TOKENS_LIMIT = (int64_t)1 << 31;
constexpr int64_t GRAD_TOKENS = (int64_t)1 << 30;  // a product's k, up to a multiple of 64, is a 32-bit number

// ---- operands --------------------------------------------------------------------

// x unpacked and, where dy lies otherwise than the product reads it, dy copied, in one
// launch: the first blocks unpack.
struct OperandArgs {
    fc::BlockRows kept;
    void* x;
    int64_t ldx;
    unsigned unpacking;      // blocks
    const void* dy;          // or null
    int64_t lddy;
    void* copy;
    int64_t ldcopy;          // a multiple of 8
    int outs;
};

template <int F, typename T> __global__ __launch_bounds__(256) void operands_kernel(OperandArgs a) {
    if (blockIdx.x < a.unpacking) {
        fc::unpack_eight<F, T>(a.kept, a.x, a.ldx, (int)a.ldx, blockIdx.x * 256 + threadIdx.x);
        return;
    }
    const uint32_t per = (uint32_t)(a.ldcopy / 8), i = (blockIdx.x - a.unpacking) * 256 + threadIdx.x, r = i / per, u = i % per;
    if (r >= a.kept.rows) return;
    typedef typename fc::Eight<T>::vec V;
    const T* const from = static_cast<const T*>(a.dy) + r * a.lddy + 8 * u;
    const int left = a.outs - 8 * (int)u;
    V v{};
    if (left >= 8) {
        v = *reinterpret_cast<const typename fc::Eight<T>::any*>(from);
    } else {
#pragma unroll
        for (int e = 0; e < 7; ++e)
            if (e < left) v[e] = from[e];
    }
    *reinterpret_cast<V*>(static_cast<T*>(a.copy) + r * a.ldcopy + 8 * u) = v;
}

// ---- the product --------------------------------------------------------------------

// TINY of fc_choice.h.
template <typename T> using Tiny = fc::Product<T, 64, 64, 32, 32, true, true, 4>;

template <typename T, bool ADD> hipError_t prepare_all() {
    for (hipError_t e : {prepare<Large<T, true, true>>((const void*)result_kernel<Large<T, true, true>, ADD, Operand>),
                         prepare<Broad<T, true, true>>((const void*)result_kernel<Broad<T, true, true>, ADD, Operand>),
                         prepare<Middle<T, true, true>>((const void*)result_kernel<Middle<T, true, true>, ADD, Operand>),
                         prepare<Tiny<T>>((const void*)result_kernel<Tiny<T>, ADD, Operand>)})
        if (e != hipSuccess) return e;
    return hipSuccess;
}

template <typename T, bool ADD> void launch(int kind, const GradArgs& g, hipStream_t s) {
    if (kind == LARGE) launch_result<Large<T, true, true>, ADD, Operand>(g, s);
    else if (kind == BROAD) launch_result<Broad<T, true, true>, ADD, Operand>(g, s);
    else if (kind == MIDDLE) launch_result<Middle<T, true, true>, ADD, Operand>(g, s);
    else launch_result<Tiny<T>, ADD, Operand>(g, s);
}

// ---- gradients of few tiles -------------------------------------------------------------

// One launch, 64 x 64 of dw to a block: 4 groups of 4 waves go through every 4th step of 64
// tokens, each with its own buffers, and their sums are added in order at the end.  Both
// operands pass registers, where x is unpacked and dy may lie on any element.  Four
// steps take 1.4 us, of which 0.64 are what LDS takes in and gives out for 32 x 32 of a wave (192
// KB): the unpacking, done again by every block of a column, and what it waits for are the rest.  In graphs, us, against the operands' launch and the tiles': 1 to 256
// tokens, 1024 x 1024 5.3 to 5.5, 6.2 to 7.6; 1003 tokens, 1001 x 520 9.8, 11.7; 1003, 2048 x
// 1024 17.9, 17.2; 4096, 1024 x 1024 27, 30; 4096, 256 x 512, where k is split 22.7, 14.1.
struct SmallArgs {
    fc::BlockRows kept;
    const void* dy;
    int64_t lddy;
    int outs;
    float scale;
    void* out;
    int dt;
    int64_t ld;
    bool add;
    int tm, tn;
};

constexpr int AHEAD = 3;      // steps of a group on their way at a time
constexpr int SMALL = CKPT_SMALL, GROUPS = CKPT_GROUPS, SMALL_THREADS = GROUPS * 256;
constexpr int SMALL_TILE = SMALL * SMALL * 2;             // bytes of an operand's
constexpr int SMALL_LDS = GROUPS * 2 * 2 * SMALL_TILE;    // 2 buffers of both

template <int F, typename T> __global__ __launch_bounds__(SMALL_THREADS) void small_kernel(SmallArgs a) {
    typedef typename fc::Eight<T>::vec V;
    int ti, tj;
    fc::tile_place(fc::xcd_order(blockIdx.x, a.tm * a.tn), a.tm, a.tn, 8, ti, tj);
    const int m0 = ti * SMALL, n0 = tj * SMALL, lane = threadIdx.x & 63, wave = __builtin_amdgcn_readfirstlane(threadIdx.x >> 6), g = wave >> 2;
    const int k = (threadIdx.x & 255) >> 2, c = 16 * (threadIdx.x & 3);  // a thread brings 16 columns of a step's token k
    const int steps = (int)((a.kept.rows + SMALL - 1) / SMALL);
    const uint32_t base = fc::lds_address(lds) + g * 4 * SMALL_TILE, to = k * 2 * SMALL + (fc::slow_block<SMALL>(c >> 4, k) << 5);
    struct Data {
        V dy[2];
        fc::Codes x[2];
        uint32_t scale;
    };
    // This thread's next step.
    int64_t t = (int64_t)g * SMALL + k;
    const T* dy = static_cast<const T*>(a.dy) + t * a.lddy + m0 + c;
    const uint8_t *codes = a.kept.codes + t * a.kept.ldc + n0 + c, *scales = a.kept.scales + t * a.kept.lds + (n0 + c) / fc::BLOCK;
    const int there = a.outs - m0 - c;
    const bool kept = (n0 + c) / fc::BLOCK < a.kept.blocks;
    auto fetch = [&]() __attribute__((always_inline)) {
        Data d{};
        if (t < a.kept.rows) {
            // past a row's end anything does: what is made of it is not stored
            if (there > 0 && (there >= 16 || (a.kept.rows - 1 - t) * a.lddy + there >= 16)) {
                d.dy[0] = fc::raw8(dy);
                d.dy[1] = fc::raw8(dy + 8);
            } else {
#pragma unroll
                for (int e = 0; e < 15; ++e)
                    if (e < there) d.dy[e / 8][e % 8] = dy[e];
            }
            if (kept) {
                const uint4 q = *reinterpret_cast<const uint4*>(codes);
                d.x[0] = fc::Codes{q.x, q.y};
                d.x[1] = fc::Codes{q.z, q.w};
                d.scale = *scales;
            }
        }
        t += GROUPS * SMALL;
        dy += GROUPS * SMALL * a.lddy;
        codes += GROUPS * SMALL * a.kept.ldc;
        scales += GROUPS * SMALL * a.kept.lds;
        return d;
    };
    auto put = [&](const Data& d, uint32_t at) __attribute__((always_inline)) {
        const float s = fc::scale_value(d.scale);
        fc::f32x8 x[2] = {fc::decode8<F>(d.x[0]) * s, fc::decode8<F>(d.x[1]) * s};
        if (d.scale > fc::FITS<F, T>) {  // seldom
            x[0] = fc::in_range<T>(x[0]);
            x[1] = fc::in_range<T>(x[1]);
        }
#pragma unroll
        for (int h = 0; h < 2; ++h) {
            *(FC_LDS V*)(uintptr_t)(at + to + 16 * h) = d.dy[h];
            *(FC_LDS V*)(uintptr_t)(at + SMALL_TILE + to + 16 * h) = __builtin_convertvector(x[h], V);
        }
    };
    const int wm = 32 * ((wave >> 1) & 1), wn = 32 * (wave & 1);
    fc::Fragments<T, SMALL, true, 2> fa, fb;
    fa.init(wm, lane);
    fb.init(wn, lane);
    f32x4 acc[2][2]{};
    Data d[AHEAD];
#pragma unroll
    for (int u = 0; u < AHEAD; ++u) d[u] = fetch();
    for (int s0 = 0, turn = 0; s0 < steps; s0 += AHEAD * GROUPS) {
#pragma unroll
        for (int u = 0; u < AHEAD; ++u) {
            const int s = s0 + u * GROUPS;
            if (s >= steps) break;
            const uint32_t at = base + turn * 2 * SMALL_TILE;
            turn ^= 1;
            put(d[u], at);
            __syncthreads();
            d[u] = fetch();
#pragma unroll
            for (int kk = 0; kk < 2; ++kk)
#pragma unroll
                for (int i = 0; i < 2; ++i)
#pragma unroll
                    for (int j = 0; j < 2; ++j) acc[i][j] = Half<T>::mma(fb.get(at + SMALL_TILE, j, kk), fa.get(at, i, kk), acc[i][j]);
        }
    }
    __syncthreads();  // the tiles are done with
    float(*const part)[SMALL][SMALL + 4] = reinterpret_cast<float(*)[SMALL][SMALL + 4]>(lds);
    static_assert(sizeof(float) * GROUPS * SMALL * (SMALL + 4) <= SMALL_LDS, "the groups' sums fit");
#pragma unroll
    for (int i = 0; i < 2; ++i)
#pragma unroll
        for (int j = 0; j < 2; ++j) *reinterpret_cast<f32x4*>(&part[g][wm + 16 * i + (lane & 15)][wn + 16 * j + 4 * (lane >> 4)]) = acc[i][j];
    __syncthreads();
    const int m = threadIdx.x >> 4, n = 4 * (threadIdx.x & 15), left = a.kept.dim - n0 - n;
    if (m0 + m >= a.outs || left <= 0) return;
    f32x4 v{};
#pragma unroll
    for (int q = 0; q < GROUPS; ++q) v += *reinterpret_cast<const f32x4*>(&part[q][m][n]);
    v = v * a.scale;
    const int64_t at = (int64_t)(m0 + m) * a.ld + n0 + n;
    if (a.add) {
#pragma unroll
        for (int e = 0; e < 4; ++e)
            if (e < left) v[e] += load_one(a.out, a.dt, at + e);
    }
    store_four(a.out, a.dt, at, v, left);
}

template <int F, typename T> void launch_small(SmallArgs a, hipStream_t s) {
    a.tm = (int)fc::ceil_div(a.outs, SMALL);
    a.tn = (int)fc::ceil_div(a.kept.dim, SMALL);
    small_kernel<F, T><<<a.tm * a.tn, SMALL_THREADS, SMALL_LDS, s>>>(a);
}

template <typename T> hipError_t prepare_small() {
    for (const void* k : {(const void*)small_kernel<FC_BLOCK_I8, T>, (const void*)small_kernel<FC_BLOCK_E4M3, T>}) {
        const hipError_t e = hipFuncSetAttribute(k, hipFuncAttributeMaxDynamicSharedMemorySize, SMALL_LDS);
        if (e != hipSuccess) return e;
    }
    return hipSuccess;
}

}  // namespace

struct fc_ckpt {
    fc::CallOrder order;
    fc::DeviceBlock block;
    int64_t dim = 0, max_tokens = 0, max_outs = 0;
    int dtype = FC_F16, format = FC_BLOCK_I8, blocks = 0;
    int64_t sums = 0;        // ckpt_limit, of which ckpt_room floats are made
    char* x = nullptr;       // unpacked
    char* dy = nullptr;      // copied
    float* sum = nullptr;
};

namespace {

fc::BlockRows rows_of(const fc_ckpt* p, const void* x, int64_t ldx, const void* codes, int64_t ldc, const void* scales, int64_t lds, int64_t n) {
    return {x, ldx, static_cast<uint8_t*>(const_cast<void*>(codes)), ldc, static_cast<uint8_t*>(const_cast<void*>(scales)), lds, n, (int)p->dim, p->blocks,
            p->blocks, 8};
}

fc::Span codes_span(const fc_ckpt* p, const void* codes, int64_t ldc, int64_t n, bool written) { return {codes, n, 32 * (int64_t)p->blocks, ldc, 1, written}; }
fc::Span scales_span(const fc_ckpt* p, const void* scales, int64_t lds, int64_t n, bool written) { return {scales, n, p->blocks, lds, 1, written}; }

bool aligned(const void* codes, int64_t ldc) { return ldc % 16 == 0 && reinterpret_cast<uintptr_t>(codes) % 16 == 0; }

template <typename T>
void grad(fc_ckpt* p, const void* dy, int64_t lddy, const fc::BlockRows& kept, int64_t outs, float scale, void* dw, int dwt, int64_t lddw, bool add,
          hipStream_t s) {
    const int64_t n = kept.rows, ldx = fc::ceil_div(p->dim, 8) * 8;
    const Choice c = ckpt_choice(n, outs, p->dim, p->sums);
    if (ckpt_small(c, n, outs, p->dim)) {
        const SmallArgs q{kept, dy, lddy, (int)outs, scale, dw, dwt, lddw, add};
        if (p->format == FC_BLOCK_I8) launch_small<FC_BLOCK_I8, T>(q, s);
        else launch_small<FC_BLOCK_E4M3, T>(q, s);
        return;
    }
    const bool copy = lddy % 8 || reinterpret_cast<uintptr_t>(dy) % 16;
    const int64_t ld = fc::ceil_div(outs, 8) * 8, per = ldx / 8, per_dy = copy ? ld / 8 : 0;
    fc::by_launches(n, per + per_dy, [&](int64_t r0, int64_t count) {
        OperandArgs a{kept, p->x + r0 * ldx * 2, ldx, (unsigned)fc::ceil_div(count * per, 256), static_cast<const char*>(dy) + r0 * lddy * 2, lddy,
                      p->dy + r0 * ld * 2, ld, (int)outs};
        a.kept.codes += r0 * kept.ldc;
        a.kept.scales += r0 * kept.lds;
        a.kept.rows = count;
        const unsigned grid = a.unpacking + (unsigned)fc::ceil_div(count * per_dy, 256);
        if (p->format == FC_BLOCK_I8) operands_kernel<FC_BLOCK_I8, T><<<grid, 256, 0, s>>>(a);
        else operands_kernel<FC_BLOCK_E4M3, T><<<grid, 256, 0, s>>>(a);
    });
    if (copy) {
        dy = p->dy;
        lddy = ld;
    }
    GradArgs g{};
    g.a = Operand{dy, lddy, (int)outs, (int)n, 0};
    g.b = Operand{p->x, ldx, (int)p->dim, (int)n, 0};
    g.m = (int)outs;
    g.n = (int)p->dim;
    g.k = (int)n;
    g.parts = 1;
    const bool split = c.splits > 1;
    g.kper = c.steps * fc::GEMM_BK;
    g.scale = scale;
    g.out = dw;
    g.dt = dwt;
    g.ld = lddw;
    g.sum = split ? p->sum : nullptr;
    if (add && !split) launch<T, true>(c.kind, g, s);
    else launch<T, false>(c.kind, g, s);
    if (split) join_splits(g, c.splits, add, s);
}

}  // namespace

extern "C" {

int fc_ckpt_create(fc_ckpt** plan, int64_t dim, int64_t max_tokens, int64_t max_outs, int dtype, int format) {
    if (!plan) return FC_EINVAL;
    *plan = nullptr;
    if (dim < 1 || dim > LD_LIMIT || max_tokens < 0 || max_tokens > GRAD_TOKENS || max_outs < 0 || max_outs > ROWS_LIMIT ||
        (dtype != FC_F16 && dtype != FC_BF16) || (format != FC_BLOCK_I8 && format != FC_BLOCK_E4M3))
        return FC_EINVAL;
    return fc::no_throw([&] {
        fc_ckpt* p = new fc_ckpt;
        p->dim = dim;
        p->max_tokens = max_tokens;
        p->max_outs = max_outs;
        p->dtype = dtype;
        p->format = format;
        p->blocks = (int)fc::ceil_div(dim, fc::BLOCK);
        fc::Layout at;
        const bool grads = max_outs > 0;
        p->sums = ckpt_limit(max_outs, dim);
        const uint64_t o_x = at.take(grads ? max_tokens * fc::ceil_div(dim, 8) * 16 : 0),
                       o_dy = at.take(max_outs % 8 ? max_tokens * fc::ceil_div(max_outs, 8) * 16 : 0), o_sum = at.take(ckpt_room(max_tokens, max_outs, dim) * 4);
        int rc = p->order.create();
        if (!rc) rc = fc::hip_code(dtype == FC_F16 ? prepare_all<f16, false>() : prepare_all<bf16, false>());
        if (!rc) rc = fc::hip_code(dtype == FC_F16 ? prepare_all<f16, true>() : prepare_all<bf16, true>());
        if (!rc) rc = fc::hip_code(dtype == FC_F16 ? prepare_small<f16>() : prepare_small<bf16>());
        if (!rc) rc = p->block.create(at.size);
        if (rc) {
            fc_ckpt_destroy(p);
            return rc;
        }
        p->x = p->block.p + o_x;
        p->dy = p->block.p + o_dy;
        p->sum = reinterpret_cast<float*>(p->block.p + o_sum);
        *plan = p;
        return FC_OK;
    });
}

void fc_ckpt_destroy(fc_ckpt* p) {
    if (!p) return;
    p->block.destroy();
    p->order.destroy();
    delete p;
}

int fc_ckpt_pack(fc_ckpt* p, const void* x, int x_dtype, int64_t ld_x, int64_t n, void* codes, int64_t ld_codes, void* scales, int64_t ld_scales,
                 void* stream) {
    return fc::no_throw([&]() -> int {
        if (!p || n < 0 || n >= TOKENS_LIMIT) return FC_EINVAL;
        int rc = fc::check_spans({{x, n, p->dim, ld_x, fc::dtype_bytes(x_dtype), false}, codes_span(p, codes, ld_codes, n, true), scales_span(p, scales, ld_scales, n, true)});
        if (rc) return rc;
        if (!aligned(codes, ld_codes)) return FC_EALIGN;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        bool note;
        rc = p->order.begin(s, note);
        if (rc) return rc;
        const fc::BlockRows a = rows_of(p, x, ld_x, codes, ld_codes, scales, ld_scales, n);
        if (p->format == FC_BLOCK_I8) fc::pack_rows<FC_BLOCK_I8>(a, x_dtype, s);
        else fc::pack_rows<FC_BLOCK_E4M3>(a, x_dtype, s);
        rc = fc::hip_code(hipGetLastError());
        p->order.done(s, note);
        return rc;
    });
}

int fc_ckpt_unpack(fc_ckpt* p, const void* codes, int64_t ld_codes, const void* scales, int64_t ld_scales, int64_t n, void* out, int out_dtype,
                   int64_t ld_out, void* stream) {
    return fc::no_throw([&]() -> int {
        if (!p || n < 0 || n >= TOKENS_LIMIT) return FC_EINVAL;
        int rc = fc::check_spans({codes_span(p, codes, ld_codes, n, false), scales_span(p, scales, ld_scales, n, false),
                                  {out, n, p->dim, ld_out, fc::dtype_bytes(out_dtype), true}});
        if (rc) return rc;
        if (!aligned(codes, ld_codes)) return FC_EALIGN;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        bool note;
        rc = p->order.begin(s, note);
        if (rc) return rc;
        const fc::BlockRows a = rows_of(p, nullptr, 0, codes, ld_codes, scales, ld_scales, n);
        if (p->format == FC_BLOCK_I8) fc::unpack_rows<FC_BLOCK_I8>(a, out, out_dtype, ld_out, (int)p->dim, s);
        else fc::unpack_rows<FC_BLOCK_E4M3>(a, out, out_dtype, ld_out, (int)p->dim, s);
        rc = fc::hip_code(hipGetLastError());
        p->order.done(s, note);
        return rc;
    });
}

int fc_ckpt_grad(fc_ckpt* p, const void* dy, int64_t ld_dy, const void* codes, int64_t ld_codes, const void* scales, int64_t ld_scales, int64_t n,
                 int64_t outs, float scale, void* dw, int dw_dtype, int64_t ld_dw, int accumulate, void* stream) {
    return fc::no_throw([&]() -> int {
        if (!p || n < 0 || n > p->max_tokens || outs < 0 || outs > p->max_outs || ld_dy > LD_LIMIT) return FC_EINVAL;
        int rc = fc::check_spans({{dy, n, outs, ld_dy, 2, false}, codes_span(p, codes, ld_codes, n, false), scales_span(p, scales, ld_scales, n, false),
                                  {dw, outs, p->dim, ld_dw, fc::dtype_bytes(dw_dtype), true}});
        if (rc) return rc;
        if (!aligned(codes, ld_codes)) return FC_EALIGN;
        if (n && outs && p->max_outs % 8 == 0 && (ld_dy % 8 || reinterpret_cast<uintptr_t>(dy) % 16)) return FC_EALIGN;
        const hipStream_t s = static_cast<hipStream_t>(stream);
        bool note;
        rc = p->order.begin(s, note);
        if (rc) return rc;
        const fc::BlockRows a = rows_of(p, nullptr, 0, codes, ld_codes, scales, ld_scales, n);
        if (n == 0) {
            if (!accumulate && outs) zeros(dw, dw_dtype, outs, p->dim, ld_dw, s);
        } else if (outs) {
            if (p->dtype == FC_F16) grad<f16>(p, dy, ld_dy, a, outs, scale, dw, dw_dtype, ld_dw, accumulate != 0, s);
            else grad<bf16>(p, dy, ld_dy, a, outs, scale, dw, dw_dtype, ld_dw, accumulate != 0, s);
        }
        rc = fc::hip_code(hipGetLastError());
        p->order.done(s, note);
        return rc;
    });
}

}  // extern "C"
