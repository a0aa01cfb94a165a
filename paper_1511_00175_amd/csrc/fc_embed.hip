// Embedding rows and their gradient (fc_lm.h).
//
// lookup: out[t] = scale * table[token[t]].  One pass; bounded by the bytes of
//   the rows read and written: 32768 rows of 2048 fp16 take 48 us (5.6 TB/s), 5001 odd
//   rows of 1001 from bf16 to fp32 7 us (4.3 TB/s), one row 1.8 (an empty launch's
//   time; 6.2 with the host's part of a call).
// grad: dtable[r] = scale * sum of dy[t] over token[t] == r.  The tokens are
//   sorted by a stable radix sort on their (row, t) pairs; then the sorted list
//   is cut into chunks of 8 or 32 entries, each summed by its own threads in order.
//   A row whose entries lie in one chunk is written there; the parts of a row
//   that runs over chunks go to a workspace and are added in a fixed order by a second
//   kernel.  No atomics on sums: the same inputs give the same bits.  Bounded by
//   the bytes of dy and of the whole table's gradient, of which the rows without
//   a token are most: the zeros are stored by blocks that run beside the sort's
//   few ones, a share in each of its launches.  32768 tokens of 2048 fp16 into
//   65536 rows of fp32 take 168 us: 87 of sort and zeros (537 MB, 6.2 TB/s), 74 of
//   sums and 8 of joins; in all 671 MB at 4.0 TB/s, where a large copy has 4.8.  256
//   tokens of 1001 fp32 into 1000 rows: 12 us, three launches one after the other.
//   Every block of a sort's second launch adds up all blocks' counts, so that very
//   long lists are bound by that: rows of 1024 fp16, 2^20 tokens 0.92 ms, 2^22 3.6, 2^24
//   24.6 (2.6, 2.5 and 1.4 TB/s).
#include <algorithm>

#include "fc_lm_host.h"

namespace {

typedef _Float16 f16;
typedef __bf16 bf16;

// V neighbours of a row, which may start at any element: global memory takes any
// alignment.  A row's last V overlap those before them where its length is no multiple
// of V.  Measured against vectors as wide as every row's alignment allows, us: 32768
// rows of 2047 looked up, fp16 41 / 71, fp32 87 / 147; their gradient into 65536 rows,
// fp16 119 / 195, fp32 241 / 313 (rows of 2048: 38, 81, 121, 214).
template <typename T, int V> struct Vec {
    T x[V];
    __device__ __forceinline__ void load(const T* p) { __builtin_memcpy(x, p, sizeof(x)); }
    __device__ __forceinline__ void store(T* p) const { __builtin_memcpy(p, x, sizeof(x)); }
};

constexpr int BITS = 9;                  // of a radix digit
constexpr int BINS = 1 << BITS;
constexpr int SORT_THREADS = 1024;
constexpr int SORT_WAVES = SORT_THREADS / 64;
constexpr int PER_THREAD = 4;
constexpr int PER_BLOCK = SORT_THREADS * PER_THREAD;

struct Tokens {
    const void* p;
    int bytes;
    int n;
    uint32_t rows;
    // The sort key of token t: its row, or `rows` where it names none.
    __device__ __forceinline__ uint32_t key(int t) const {
        const int64_t v = bytes == 8 ? static_cast<const int64_t*>(p)[t] : static_cast<const int32_t*>(p)[t];
        return v >= 0 && v < (int64_t)rows ? (uint32_t)v : rows;
    }
};

// Zeros for the rows of a gradient: `part` of `parts` equal shares.
struct Fill {
    char* p;
    int64_t ld_bytes;
    int64_t row_bytes;
    int64_t rows;
    int part, parts;
    int blocks;     // that fill
};

// Zeros, 16 bytes a store but for the ends (any even address and length).
__device__ __forceinline__ void fill_run(char* p, int64_t bytes) {
    const int64_t head = min(bytes, (int64_t)(-(uintptr_t)p & 15)), whole = (bytes - head) / 16, tail = bytes - head - 16 * whole;
    for (int64_t i = threadIdx.x; i < whole; i += blockDim.x) *reinterpret_cast<uint4*>(p + head + 16 * i) = uint4{};
    const int i = threadIdx.x;
    if (2 * i < head) reinterpret_cast<uint16_t*>(p)[i] = 0;
    if (2 * i < tail) reinterpret_cast<uint16_t*>(p + head + 16 * whole)[i] = 0;
}

__device__ __forceinline__ void fill_rows(const Fill& f, int64_t block) {
    const int64_t r0 = f.rows * f.part / f.parts, r1 = f.rows * (f.part + 1) / f.parts;
    const int64_t lo = r0 + (r1 - r0) * block / f.blocks, hi = r0 + (r1 - r0) * (block + 1) / f.blocks;
    if (f.row_bytes == f.ld_bytes) return fill_run(f.p + lo * f.ld_bytes, (hi - lo) * f.row_bytes);
    for (int64_t r = lo; r < hi; ++r) fill_run(f.p + r * f.ld_bytes, f.row_bytes);
}

struct SortPass {
    Tokens tokens;
    const uint2* in;      // (key, t), or null: the tokens themselves
    uint2* out;
    uint32_t* hist;       // per block, BINS counts of the pass's digit
    int shift;
    int blocks;           // that sort; the launch's others fill
    Fill fill;
};

__device__ __forceinline__ uint2 sort_item(const SortPass& a, int i) {
    return a.in ? a.in[i] : make_uint2(a.tokens.key(i), (uint32_t)i);
}

// Counts of every digit among a block's items.  21647 tokens: 4.3 us, a launch's
// latency, as the pass after it, 9.2, is bound by its scan over the bins.
__global__ __launch_bounds__(SORT_THREADS) void sort_count_kernel(SortPass a) {
    if ((int)blockIdx.x >= a.blocks) return fill_rows(a.fill, blockIdx.x - a.blocks);
    __shared__ uint32_t count[BINS];
    for (int d = threadIdx.x; d < BINS; d += SORT_THREADS) count[d] = 0;
    __syncthreads();
    const int first = blockIdx.x * PER_BLOCK;
    for (int i = threadIdx.x; i < PER_BLOCK && first + i < a.tokens.n; i += SORT_THREADS)
        atomicAdd(&count[(sort_item(a, first + i).x >> a.shift) & (BINS - 1)], 1u);
    __syncthreads();
    for (int d = threadIdx.x; d < BINS; d += SORT_THREADS) a.hist[(int64_t)blockIdx.x * BINS + d] = count[d];
}

// One pass over the items of block `b` of `blocks`: each wave counts its digits
// in the order of its items, the waves' and blocks' counts before it give every
// item its place.
__global__ __launch_bounds__(SORT_THREADS) void sort_scatter_kernel(SortPass a) {
    if ((int)blockIdx.x >= a.blocks) return fill_rows(a.fill, blockIdx.x - a.blocks);
    __shared__ uint32_t count[SORT_WAVES][BINS];
    __shared__ uint32_t scan[SORT_WAVES];
    const int b = blockIdx.x;
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int first = b * PER_BLOCK + wave * (64 * PER_THREAD);
    for (int d = lane; d < BINS; d += 64) count[wave][d] = 0;
    __syncthreads();
    uint2 item[PER_THREAD];
    uint32_t rank[PER_THREAD];
#pragma unroll
    for (int q = 0; q < PER_THREAD; ++q) {
        const int i = first + 64 * q + lane;
        const bool live = i < a.tokens.n;
        item[q] = live ? sort_item(a, i) : make_uint2(0xffffffffu, 0);
        const uint32_t digit = (item[q].x >> a.shift) & (BINS - 1);
        uint64_t same = __ballot(live);
#pragma unroll
        for (int k = 0; k < BITS; ++k) {
            const uint64_t set = __ballot((digit >> k) & 1);
            same &= (digit >> k) & 1 ? set : ~set;
        }
        const uint32_t before = __popcll(same & ((1ull << lane) - 1));
        if (live) rank[q] = count[wave][digit] + before;
        __builtin_amdgcn_wave_barrier();
        if (live && before == 0) count[wave][digit] += __popcll(same);
        __builtin_amdgcn_wave_barrier();
    }
    __syncthreads();
    // per digit: the block's waves in order, and the items of earlier blocks
    const int d = threadIdx.x;
    uint32_t total = 0, earlier = 0;
    if (d < BINS) {
        uint32_t sum = 0;
        for (int w = 0; w < SORT_WAVES; ++w) {
            const uint32_t c = count[w][d];
            count[w][d] = sum;
            sum += c;
        }
        for (int k = 0; k < a.blocks; ++k) {
            const uint32_t c = a.hist[(int64_t)k * BINS + d];
            earlier += k < b ? c : 0;
            total += c;
        }
    }
    // exclusive sum of the totals over the digits: within waves, then over waves
    uint32_t inc = total;
#pragma unroll
    for (int k = 1; k < 64; k *= 2) {
        const uint32_t up = __shfl_up(inc, k);
        if (lane >= k) inc += up;
    }
    if (d < BINS && lane == 63) scan[wave] = inc;
    __syncthreads();
    if (d < BINS) {
        uint32_t before = inc - total + earlier;
        for (int w = 0; w < wave; ++w) before += scan[w];
        for (int w = 0; w < SORT_WAVES; ++w) count[w][d] += before;
    }
    __syncthreads();
#pragma unroll
    for (int q = 0; q < PER_THREAD; ++q) {
        const int i = first + 64 * q + lane;
        if (i < a.tokens.n) a.out[count[wave][(item[q].x >> a.shift) & (BINS - 1)] + rank[q]] = item[q];
    }
}

// Lists of up to FEW tokens are sorted in one launch: a block has 64 tokens, and
// each of its 16 waves counts for them which of a sixteenth of the list come before.
// A whole gradient of 1000 rows of 1024, us, with the passes by digits in one block /
// with this: 256 tokens 17.1 / 11.2, 1024 tokens 18.0 / 12.4, 4096 tokens 23.8 / 19.2;
// of 500 rows (one pass) 13.3 / 11.2, 14.0 / 11.8, 18.9 / 18.9.
constexpr int FEW = 4096;

__global__ __launch_bounds__(SORT_THREADS) void sort_few_kernel(SortPass a) {
    if ((int)blockIdx.x >= a.blocks) return fill_rows(a.fill, blockIdx.x - a.blocks);
    __shared__ __align__(16) uint64_t keys[FEW];  // a row, then a place in the list: no two are the same
    __shared__ uint32_t before[SORT_WAVES][64];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int per = (a.tokens.n + 8 * SORT_WAVES - 1) / (8 * SORT_WAVES) * 8;  // of a wave
    for (int t = threadIdx.x; t < per * SORT_WAVES; t += SORT_THREADS)
        keys[t] = t < a.tokens.n ? (uint64_t)a.tokens.key(t) << 32 | (uint32_t)t : ~0ull;
    __syncthreads();
    const int t = min((int)blockIdx.x * 64 + lane, a.tokens.n - 1);
    const uint64_t mine = keys[t];
    uint32_t count = 0;
    for (int k = wave * per; k < (wave + 1) * per; k += 8) {
#pragma unroll
        for (int u = 0; u < 8; ++u) count += keys[k + u] < mine;
    }
    before[wave][lane] = count;
    __syncthreads();
    if (wave || (int)blockIdx.x * 64 + lane >= a.tokens.n) return;
#pragma unroll
    for (int q = 1; q < SORT_WAVES; ++q) count += before[q][lane];
    a.out[count] = make_uint2((uint32_t)(mine >> 32), (uint32_t)mine);
}

struct SumArgs {
    const uint2* sorted;     // (row, t) by row, then t; rows of `rows` name none
    int n;
    uint32_t rows;
    int chunk;
    const void* dy;
    int64_t ld_dy;
    int dim;
    void* out;
    int64_t ld_out;
    float scale;
    int accumulate;
    int first;               // chunk of the launch's first block
    float* parts;            // per chunk: the sum that goes on from the chunk before, and the one that goes on into the next
};

// The columns before `own` are another thread's as well: it adds to them.
template <typename TO, int V> __device__ __forceinline__ void store_row(const SumArgs& a, uint32_t row, int col, int own, const float* sum) {
    TO* const p = static_cast<TO*>(a.out) + (int64_t)row * a.ld_out + col;
    Vec<TO, V> o;
    if (a.accumulate && own > col) {
#pragma unroll
        for (int e = 0; e < V; ++e)
            if (col + e >= own) p[e] = (TO)((float)p[e] + a.scale * sum[e]);
        return;
    }
    if (a.accumulate) {
        o.load(p);
#pragma unroll
        for (int e = 0; e < V; ++e) o.x[e] = (TO)((float)o.x[e] + a.scale * sum[e]);
    } else {
#pragma unroll
        for (int e = 0; e < V; ++e) o.x[e] = (TO)(a.scale * sum[e]);
    }
    o.store(p);
}

// Sums of one chunk of the sorted list; a thread holds V columns.  The entries
// are the same for every thread of a block, so keys and branches are uniform;
// UNROLL rows are loaded before the first is added: a row alone would wait for
// each load.  Bound by reading dy and writing rows (74 us for 32768 tokens of 2048
// fp16, 402 MB at most: the rows written again after their zeros among them);
// 4 or 16 rows ahead, narrower vectors and other chunks were no faster.
template <typename TI, typename TO, int V> __global__ __launch_bounds__(256) void sum_kernel(SumArgs a) {
    constexpr int UNROLL = 8;
    typedef Vec<TI, V> I;
    const int own = (blockIdx.y * 256 + threadIdx.x) * V, col = min(own, a.dim - V);
    const int c = a.first + blockIdx.x, lo = c * a.chunk, hi = min(lo + a.chunk, a.n);
    uint32_t row = a.sorted[lo].x;
    if (row >= a.rows || own >= a.dim) return;
    bool from_before = c > 0 && a.sorted[lo - 1].x == row;
    float* const head = a.parts + (int64_t)(2 * c) * a.dim + col;
    float* const tail = head + a.dim;
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.f;
    const TI* dy = static_cast<const TI*>(a.dy) + col;
    auto finish = [&]() {
        if (from_before) {
#pragma unroll
            for (int e = 0; e < V; ++e) head[e] = sum[e];
        } else {
            store_row<TO, V>(a, row, col, own, sum);
        }
    };
    for (int i = lo; i < hi; i += UNROLL) {
        uint2 e[UNROLL];
        I x[UNROLL];
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            e[u] = a.sorted[min(i + u, hi - 1)];
            e[u].x = __builtin_amdgcn_readfirstlane(e[u].x);
            e[u].y = __builtin_amdgcn_readfirstlane(e[u].y);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {  // an entry that names no row has a place in dy as well
            x[u].load(dy + (int64_t)e[u].y * a.ld_dy);
        }
#pragma unroll
        for (int u = 0; u < UNROLL; ++u) {
            if (i + u >= hi) break;
            if (e[u].x != row) {
                finish();
                if (e[u].x >= a.rows) return;  // the rest names no row
                row = e[u].x;
                from_before = false;
#pragma unroll
                for (int k = 0; k < V; ++k) sum[k] = 0.f;
            }
#pragma unroll
            for (int k = 0; k < V; ++k) sum[k] += (float)x[u].x[k];
        }
    }
    if (!from_before && hi < a.n && a.sorted[hi].x == row) {
#pragma unroll
        for (int e = 0; e < V; ++e) tail[e] = sum[e];
    } else {
        finish();
    }
}

// The rows that run over chunks: the block of the chunk where a row begins adds
// its parts, each of 4 waves every fourth one, then the waves' sums in order.
// Bound by its chain of loads (a search, then parts): 3.3 to 8 us.
template <typename TO, int V> __global__ __launch_bounds__(256) void join_kernel(SumArgs a) {
    constexpr int UNROLL = 4;
    __shared__ float part[4][64 * V];
    const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
    const int own = (blockIdx.y * 64 + lane) * V, col = min(own, a.dim - V);
    const int c = a.first + blockIdx.x, chunks = (a.n + a.chunk - 1) / a.chunk;
    const int hi = (c + 1) * a.chunk;
    if (hi >= a.n) return;
    const uint32_t row = a.sorted[hi].x;
    if (row >= a.rows || a.sorted[hi - 1].x != row) return;
    // the whole chunk is one row from before: its owner is an earlier chunk
    if (c > 0 && a.sorted[c * a.chunk].x == row && a.sorted[c * a.chunk - 1].x == row) return;
    int end = c + 1;
    {  // the last chunk that begins with this row
        int lo = c + 1, up = chunks - 1;
        while (lo < up) {
            const int mid = (lo + up + 1) / 2;
            if (a.sorted[(int64_t)mid * a.chunk].x == row) lo = mid;
            else up = mid - 1;
        }
        end = lo;
    }
    const bool live = own < a.dim;
    float sum[V];
#pragma unroll
    for (int e = 0; e < V; ++e) sum[e] = 0.f;
    if (live) {
        if (wave == 0) {
            const float* p = a.parts + (int64_t)(2 * c + 1) * a.dim + col;
#pragma unroll
            for (int e = 0; e < V; ++e) sum[e] = p[e];
        }
        for (int k = c + 1 + wave; k <= end; k += 4 * UNROLL) {
            float x[UNROLL][V];
#pragma unroll
            for (int u = 0; u < UNROLL; ++u) {
                const float* p = a.parts + (int64_t)(2 * min(k + 4 * u, end)) * a.dim + col;
#pragma unroll
                for (int e = 0; e < V; ++e) x[u][e] = p[e];
            }
#pragma unroll
            for (int u = 0; u < UNROLL; ++u)
#pragma unroll
                for (int e = 0; e < V; ++e) sum[e] += k + 4 * u <= end ? x[u][e] : 0.f;
        }
#pragma unroll
        for (int e = 0; e < V; ++e) part[wave][lane * V + e] = sum[e];
    }
    __syncthreads();
    if (wave || !live) return;
#pragma unroll
    for (int w = 1; w < 4; ++w)
#pragma unroll
        for (int e = 0; e < V; ++e) sum[e] += part[w][lane * V + e];
    store_row<TO, V>(a, row, col, own, sum);
}

struct LookupArgs {
    const void* table;
    int64_t ld_table;
    Tokens tokens;
    void* out;
    int64_t ld_out;
    int dim;
    float scale;
    int per_row;   // threads per row, a power of two
};

template <typename TI, typename TO, int V> __global__ __launch_bounds__(256) void lookup_kernel(LookupArgs a) {
    const int rows_per_block = 256 / a.per_row;
    const int64_t t = (int64_t)blockIdx.x * rows_per_block + threadIdx.x / a.per_row;
    if (t >= a.tokens.n) return;
    const uint32_t row = a.tokens.key((int)t);
    const TI* in = static_cast<const TI*>(a.table) + (int64_t)row * a.ld_table;
    TO* out = static_cast<TO*>(a.out) + t * a.ld_out;
    for (int own = (threadIdx.x & (a.per_row - 1)) * V; own < a.dim; own += a.per_row * V) {
        const int col = min(own, a.dim - V);
        Vec<TO, V> o;
        if (row < a.tokens.rows) {
            Vec<TI, V> x;
            x.load(in + col);
#pragma unroll
            for (int e = 0; e < V; ++e) o.x[e] = (TO)(a.scale * (float)x.x[e]);
        } else {
#pragma unroll
            for (int e = 0; e < V; ++e) o.x[e] = (TO)0.f;
        }
        o.store(out + col);
    }
}

// f(pointer to a value of the storage type) for an fc_dtype value.
template <typename F> void with_type(int dt, F&& f) {
    if (dt == FC_F32) f(static_cast<float*>(nullptr));
    else if (dt == FC_F16) f(static_cast<f16*>(nullptr));
    else f(static_cast<bf16*>(nullptr));
}

template <int N> struct Width {
    static constexpr int value = N;
};

template <typename F> void with_width(int v, F&& f) {
    if (v == 8) f(Width<8>{});
    else if (v == 4) f(Width<4>{});
    else if (v == 2) f(Width<2>{});
    else f(Width<1>{});
}

int pow2_at_least(int64_t n, int most) {
    int p = 1;
    while (p < n && p < most) p *= 2;
    return p;
}

}  // namespace

struct fc_embed {
    fc::CallOrder order;
    fc::DeviceBlock block;
    int64_t rows = 0, dim = 0, max_tokens = 0;
    int passes = 0;
    uint2* pairs[2] = {nullptr, nullptr};
    uint32_t* hist = nullptr;
    float* parts = nullptr;
};

namespace {

constexpr int64_t LIMIT = (int64_t)1 << 31;
// Tokens of a gradient: places in the sorted list, and the ends of its chunks, are
// 32-bit numbers (above 2^31 - 32 tokens the last chunk's end would not be).
constexpr int64_t TOKENS_LIMIT = (int64_t)1 << 30;
constexpr int64_t DIM_LIMIT = (int64_t)1 << 20;  // column blocks of a launch

// Entries of the sorted list per chunk: enough chunks to fill the chip, long
// enough that a row's parts are few.
int chunk_of(int64_t n) { return n <= 4096 ? 8 : 32; }

// Neighbours per thread: of 16 bytes, or as many as a row has.
int vector_of(int most, int64_t dim) {
    while (most > dim) most /= 2;
    return most;
}

int64_t most_chunks(int64_t n) { return std::max(fc::ceil_div(std::min<int64_t>(n, 4096), 8), fc::ceil_div(n, 32)); }

int lookup_body(fc_embed* p, const void* table, int tdt, int64_t ld_table, const void* tokens, int token_bytes, int64_t n,
                float scale, void* out, int odt, int64_t ld_out, hipStream_t s) {
    if (!p || n < 0 || n >= LIMIT || (token_bytes != 4 && token_bytes != 8)) return FC_EINVAL;
    const fc::Span st{table, p->rows, p->dim, ld_table, fc::dtype_bytes(tdt), false};
    const fc::Span so{out, n, p->dim, ld_out, fc::dtype_bytes(odt), true};
    int rc = fc::check_spans({st, so, {tokens, 1, n, n, token_bytes, false}});
    if (rc || n == 0) return rc;
    const int v = vector_of(16 / std::min(st.bytes, so.bytes), p->dim);
    LookupArgs a{table, ld_table, {tokens, token_bytes, (int)n, (uint32_t)p->rows}, out, ld_out, (int)p->dim, scale, 0};
    a.per_row = pow2_at_least(fc::ceil_div(p->dim, v), 256);
    bool note;
    rc = p->order.begin(s, note);
    if (rc) return rc;
    with_type(tdt, [&](auto* ti) {
        with_type(odt, [&](auto* to) {
            with_width(v, [&](auto w) {
                typedef std::remove_pointer_t<decltype(ti)> TI;
                typedef std::remove_pointer_t<decltype(to)> TO;
                fc::by_launches(n, a.per_row, [&](int64_t t0, int64_t count) {
                    LookupArgs b = a;
                    b.tokens.p = static_cast<const char*>(tokens) + t0 * token_bytes;
                    b.tokens.n = (int)count;
                    b.out = static_cast<char*>(out) + t0 * ld_out * so.bytes;
                    lookup_kernel<TI, TO, decltype(w)::value><<<(unsigned)fc::ceil_div(count, 256 / a.per_row), 256, 0, s>>>(b);
                });
            });
        });
    });
    rc = fc::hip_code(hipGetLastError());
    p->order.done(s, note);
    return rc;
}

int grad_body(fc_embed* p, const void* dy, int ydt, int64_t ld_dy, const void* tokens, int token_bytes, int64_t n, float scale,
              void* out, int odt, int64_t ld_out, int accumulate, hipStream_t s) {
    if (!p || n < 0 || n > p->max_tokens || (token_bytes != 4 && token_bytes != 8)) return FC_EINVAL;
    const fc::Span sy{dy, n, p->dim, ld_dy, fc::dtype_bytes(ydt), false};
    const fc::Span so{out, p->rows, p->dim, ld_out, fc::dtype_bytes(odt), true};
    int rc = fc::check_spans({sy, so, {tokens, 1, n, n, token_bytes, false}});
    if (rc) return rc;
    bool note;
    rc = p->order.begin(s, note);
    if (rc) return rc;

    // launches of the sort, each with a share of the zeros
    const bool few = n <= FEW;
    const int blocks = (int)fc::ceil_div(n, few ? 64 : PER_BLOCK);
    const int launches = few ? 1 : 2 * p->passes;
    Fill fill{static_cast<char*>(out), ld_out * so.bytes, p->dim * so.bytes, p->rows, 0, launches, 0};
    if (!accumulate) {
        // blocks of 1024 threads with about 16 stores each
        const int64_t units = fill.row_bytes * fill.rows / launches / 16;
        fill.blocks = (int)std::min<int64_t>(std::max<int64_t>(1, fc::ceil_div(units, 16 * SORT_THREADS)),
                                             std::max<int64_t>(1, p->rows / launches));
    }
    const Tokens t{tokens, token_bytes, (int)n, (uint32_t)p->rows};
    const uint2* sorted = nullptr;
    if (few) {
        SortPass a{t, nullptr, p->pairs[0], nullptr, 0, blocks, fill};
        if (blocks + fill.blocks > 0) sort_few_kernel<<<blocks + fill.blocks, SORT_THREADS, 0, s>>>(a);
        sorted = p->pairs[0];
    } else {
        SortPass a{t, nullptr, nullptr, p->hist, 0, blocks, fill};
        for (int k = 0; k < p->passes; ++k) {
            a.shift = k * BITS;
            a.out = p->pairs[k & 1];
            a.fill.part = 2 * k;
            sort_count_kernel<<<blocks + fill.blocks, SORT_THREADS, 0, s>>>(a);
            a.fill.part = 2 * k + 1;
            sort_scatter_kernel<<<blocks + fill.blocks, SORT_THREADS, 0, s>>>(a);
            a.in = a.out;
        }
        sorted = a.in;
    }
    rc = fc::hip_code(hipGetLastError());
    if (!rc && n > 0) {
        const int chunk = chunk_of(n);
        SumArgs a{sorted, (int)n, (uint32_t)p->rows, chunk, dy, ld_dy, (int)p->dim, out, ld_out, scale, accumulate, 0, p->parts};
        const int v = vector_of(16 / sy.bytes, p->dim);
        const int chunks = (int)fc::ceil_div(n, chunk);
        with_type(odt, [&](auto* to) {
            typedef std::remove_pointer_t<decltype(to)> TO;
            with_width(v, [&](auto w) {
                constexpr int V = decltype(w)::value;
                fc::by_launches(chunks, 256, [&](int64_t first, int64_t count) {
                    a.first = (int)first;
                    const dim3 grid((unsigned)count, (unsigned)fc::ceil_div(p->dim, 256 * V));
                    with_type(ydt, [&](auto* ti) {
                        typedef std::remove_pointer_t<decltype(ti)> TI;
                        sum_kernel<TI, TO, V><<<grid, 256, 0, s>>>(a);
                    });
                });
                fc::by_launches(chunks - 1, 256, [&](int64_t first, int64_t count) {
                    a.first = (int)first;
                    join_kernel<TO, V><<<dim3((unsigned)count, (unsigned)fc::ceil_div(p->dim, 64 * V)), 256, 0, s>>>(a);
                });
            });
        });
        rc = fc::hip_code(hipGetLastError());
    }
    p->order.done(s, note);
    return rc;
}

}  // namespace

extern "C" {

int fc_embed_create(fc_embed** plan, int64_t rows, int64_t dim, int64_t max_tokens) {
    if (!plan) return FC_EINVAL;
    *plan = nullptr;
    if (rows < 1 || dim < 1 || max_tokens < 0 || rows >= LIMIT || dim > DIM_LIMIT || max_tokens > TOKENS_LIMIT) return FC_EINVAL;
    return fc::no_throw([&] {
        fc_embed* p = new fc_embed;
        p->rows = rows;
        p->dim = dim;
        p->max_tokens = max_tokens;
        for (int64_t top = rows; top > 0; top >>= BITS) ++p->passes;  // keys are 0 .. rows
        fc::Layout at;
        const uint64_t a = at.take(max_tokens * sizeof(uint2)), b = at.take(max_tokens * sizeof(uint2));
        const uint64_t h = at.take(fc::ceil_div(max_tokens, PER_BLOCK) * BINS * sizeof(uint32_t));
        const uint64_t q = at.take(2 * most_chunks(max_tokens) * dim * sizeof(float));
        int rc = p->order.create();
        if (!rc) rc = p->block.create(at.size);
        if (rc) {
            fc_embed_destroy(p);
            return rc;
        }
        p->pairs[0] = reinterpret_cast<uint2*>(p->block.p + a);
        p->pairs[1] = reinterpret_cast<uint2*>(p->block.p + b);
        p->hist = reinterpret_cast<uint32_t*>(p->block.p + h);
        p->parts = reinterpret_cast<float*>(p->block.p + q);
        *plan = p;
        return FC_OK;
    });
}

void fc_embed_destroy(fc_embed* p) {
    if (!p) return;
    p->block.destroy();
    p->order.destroy();
    delete p;
}

int fc_embed_lookup(fc_embed* p, const void* table, int table_dtype, int64_t ld_table, const void* tokens, int token_bytes,
                    int64_t n, float scale, void* out, int out_dtype, int64_t ld_out, void* stream) {
    return fc::no_throw([&] {
        return lookup_body(p, table, table_dtype, ld_table, tokens, token_bytes, n, scale, out, out_dtype, ld_out,
                           static_cast<hipStream_t>(stream));
    });
}

int fc_embed_grad(fc_embed* p, const void* dy, int dy_dtype, int64_t ld_dy, const void* tokens, int token_bytes, int64_t n,
                  float scale, void* dtable, int dtable_dtype, int64_t ld_dtable, int accumulate, void* stream) {
    return fc::no_throw([&] {
        return grad_body(p, dy, dy_dtype, ld_dy, tokens, token_bytes, n, scale, dtable, dtable_dtype, ld_dtable, accumulate,
                         static_cast<hipStream_t>(stream));
    });
}

}  // extern "C"
