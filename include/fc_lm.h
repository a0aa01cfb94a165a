/*
 * fc_lm.h -- C ABI of the operators at the ends of a language model, within its
 * blocks and of its matrix update, for MI355X (gfx950): what produces the gradients
 * that fc.h aggregates, and what else may consume their sum.
 *   fc_embed : scaled rows of a table for a list of tokens, and the table's
 *              gradient, summed token by token in sorted order
 *   fc_xent  : softmax cross entropy over a vocabulary, computed in pieces of
 *              the vocabulary without storing the logits, with both gradients
 *              (for which 16-bit exponentials are kept, see fc_xent_create)
 *   fc_muon  : momentum updates made orthogonal by Newton-Schulz products,
 *              for every matrix of a flat parameter vector at once
 *   fc_norm  : the norms before and after a block with its gate and residual
 *              scale, and their gradients
 *   fc_ckpt  : activations kept in 8 bits, and a weight's gradient from them
 *   fc_mxfp  : matrices in microscaled 4-bit floating point, and their products
 *
 * Conventions for every entry point, as in fc.h:
 *   - Buffers are device pointers owned by the caller.  A plan owns its tables
 *     and workspaces (hipMalloc on the device current when it is created) and
 *     nothing of a call is kept for the next.
 *   - Pointers are aligned to their element type (FC_EALIGN otherwise); the
 *     flat vectors of fc_muon to 16 bytes, as in fc.h.  A row stride `ld` is in
 *     elements and at least the row's length; 16-byte aligned rows are the
 *     fast case.
 *   - Calls are asynchronous on `stream` and validate before they enqueue.
 *     Calls on one plan take effect in the order they are made, whatever their
 *     streams (a call on another stream than the previous one makes its stream
 *     wait, on the device).  They must not run concurrently from several host
 *     threads.
 *   - Every call enqueues kernel launches only (no copies, memsets or
 *     allocations), so it may be captured in a HIP graph; a captured call
 *     neither waits for the plan's previous call nor becomes it.  Graphs that
 *     hold calls of one plan share its workspace: they run one after the other.
 *   - A written buffer may not overlap any other buffer of the call
 *     (FC_EALIAS).
 *   - Results do not depend on timing: sums are taken in a fixed order, so the
 *     same inputs give the same bits.
 *   - Token and target lists hold int32 or int64 (`token_bytes` 4 or 8).  An
 *     entry outside [0, rows) -- below zero is the usual padding -- names no
 *     row: its looked-up row is zeros, it has loss 0 and no gradient, whatever
 *     its inputs hold (infinities and NaN included).
 *   - Return value: FC_OK or a negative code of fc.h (fc_strerror names it).
 */
#ifndef FC_LM_H
#define FC_LM_H

#include <stdint.h>

#include "fc.h"

#ifdef __cplusplus
extern "C" {
#endif

/* Storage types are fc.h's fc_dtype values and this one. */
#define FC_BF16 2

/* ---- embedding ---------------------------------------------------------- */

typedef struct fc_embed fc_embed;

/* A plan for tables of `rows` rows of `dim` elements and up to `max_tokens`
 * tokens a gradient (1 <= rows < 2^31, 1 <= dim <= 2^20, 0 <= max_tokens <= 2^30).
 * Its workspace holds the sorted tokens and partial sums: 16 + dim / 4 bytes per
 * token (dim for the first 4096). */
int fc_embed_create(fc_embed** plan, int64_t rows, int64_t dim, int64_t max_tokens);
void fc_embed_destroy(fc_embed* plan);

/* out[t, :] = scale * table[tokens[t], :] for t < n, computed in fp32 and
 * rounded once to the output's type.  n < 2^31. */
int fc_embed_lookup(fc_embed* plan, const void* table, int table_dtype, int64_t ld_table, const void* tokens,
                    int token_bytes, int64_t n, float scale, void* out, int out_dtype, int64_t ld_out, void* stream);

/* dtable[r, :] = (accumulate ? dtable[r, :] : 0) + scale * sum of dy[t, :] over
 * the t with tokens[t] == r, for every row of the table, in fp32, rounded once to
 * the output's type.  The tokens are sorted (stable) and the sorted list is cut into
 * chunks of a fixed length, wherever rows begin in it: within a chunk a row's terms
 * are added in ascending t; of a row that runs over chunks every fourth chunk's sum is
 * added to one of four, and these in order.  The same list and inputs give the same
 * bits; a row's last bits may depend on how many tokens other rows have.
 * n <= max_tokens (FC_EINVAL). */
int fc_embed_grad(fc_embed* plan, const void* dy, int dy_dtype, int64_t ld_dy, const void* tokens, int token_bytes,
                  int64_t n, float scale, void* dtable, int dtable_dtype, int64_t ld_dtable, int accumulate,
                  void* stream);

/* ---- cross entropy ------------------------------------------------------ */

typedef struct fc_xent fc_xent;

/* A plan for a vocabulary of `rows` rows of `dim` elements and up to
 * `max_tokens` tokens a call; x and w are of `dtype`, FC_F16 or FC_BF16.
 * 1 <= rows, dim <= 2^21, 0 <= max_tokens < 2^31.  `chunk_tokens` tokens go through
 * together (0: as many as the exponentials below fit in 4 GiB, at least 256; at most
 * 2^18 in any case).  The workspace, all of it made here whatever calls follow:
 *   16 bits per row and token of a chunk (64 for the first 64) for exp(l - a maximum),
 *   which fc_xent_loss does not use; 8 bytes per token and 128 rows (32 rows for the
 *   first 64); a 16-bit copy of a chunk's x, and of w where dim is no multiple of 8;
 *   partial sums of products that are split along k, up to 512 MiB; and for plans of
 *   more tokens than a chunk's 4 bytes per element of dw. */
int fc_xent_create(fc_xent** plan, int64_t rows, int64_t dim, int64_t max_tokens, int dtype, int64_t chunk_tokens);
void fc_xent_destroy(fc_xent* plan);

/* loss[t] = log sum over r of exp(l[t, r]) - l[t, targets[t]], l[t, r] = the sum
 * over d of x[t, d] w[r, d], for t < n <= max_tokens.  Products, logits,
 * maxima, sums and the loss are fp32.  Unless dim is not a multiple of 8 (x and
 * w are then copied), ld_x and ld_w are multiples of 8 and x and w 16-byte
 * aligned (FC_EALIGN); both strides are at most 2^21. */
int fc_xent_loss(fc_xent* plan, const void* x, int64_t ld_x, const void* w, int64_t ld_w, const void* targets,
                 int token_bytes, int64_t n, float* loss, void* stream);

/* The same, with the gradients of scale * the sum of the losses:
 *   dx[t, :] = scale * sum over r of d[t, r] w[r, :]
 *   dw[r, :] = scale * sum over t of d[t, r] x[t, :]
 *   d[t, r] = exp(l[t, r] - lse[t]) - (r == targets[t])
 * d is rounded to x's type for the products, and the exponential it is formed from
 * once before (both times 2^15 for fp16, so that 2^-29 of the largest keeps all its
 * bits); the products' sums are fp32 and rounded once to the output's type.  An fp32
 * output thus carries the two roundings of every d, 2^-11 (fp16) or 2^-8 (bf16) each at
 * most.  A chunk of at most 64 tokens keeps d to twice that type's bits: so does a plan
 * of chunk_tokens <= 64 for any number of tokens, reading w for each chunk (1003 tokens,
 * 50001 rows of 520, bf16: 2.2 ms instead of 0.36).  Either output may be null.  Without
 * tokens dw is zeros. */
int fc_xent_loss_grad(fc_xent* plan, const void* x, int64_t ld_x, const void* w, int64_t ld_w, const void* targets,
                      int token_bytes, int64_t n, float scale, float* loss, void* dx, int dx_dtype, int64_t ld_dx,
                      void* dw, int dw_dtype, int64_t ld_dw, void* stream);

/* ---- orthogonal updates ------------------------------------------------- */

/* A matrix within the flat vectors of fc.h: element (r, c) is at
 * offset + r * cols + c.  Offsets are multiples of 4 (FC_EALIGN); matrices are
 * sorted by offset and do not overlap.  The multipliers scale lr and wd, as
 * fc_segment's do. */
typedef struct {
    uint64_t offset;
    uint64_t rows, cols; /* 1 to 2^20 each */
    float lr_mult;
    float decay_mult;
} fc_matrix;

typedef struct fc_muon fc_muon;

/* A plan for n matrices (n may be 0) and `steps` (1 to 64) Newton-Schulz steps
 *   X = D / |D|_F;  X <- a X + (b A + c A A) X, A = X X^T, `steps` times
 * (a matrix of more rows than columns is transposed before and after; a matrix
 * of zeros stays zeros; |D|_F is taken in 64 bits).
 *   coefficients : a, b, c, or null for 3.4445, -4.7750, 2.0315, which bring
 *                  every singular value above about 0.001 near 1 in 5 steps.
 *                  Others must keep singular values in [0, 2] (FC_EINVAL).
 *   dtype        : of the result.  FC_BF16: products of 11-bit numbers (fp16,
 *                  scaled), sums in fp32, and X's own term at 22 bits; the error is
 *                  below bf16's rounding.  FC_F16, FC_F32: every product from 22-bit
 *                  operands, for 3 times the work; about fp32's accuracy (below that
 *                  of plain fp32 products for large matrices, a few 2^-22 of the norm
 *                  for those of a few rows).
 *   nesterov     : for fc_muon_step.
 * The workspace holds 8 bytes per element and 4 (FC_BF16) or 8 per element of
 * the shorter side's square. */
int fc_muon_create(fc_muon** plan, const fc_matrix* matrices, int n, int dtype, int steps, const double* coefficients,
                   int nesterov);
void fc_muon_destroy(fc_muon* plan);

/* out = the steps above of g, matrix by matrix; elements of no matrix are not
 * written.  g is of any type, out of the plan's. */
int fc_muon_orthogonalize(fc_muon* plan, const void* g, int g_dtype, void* out, void* stream);

/* One momentum step from a raw sum g (as fc_sgd_step takes it), for the plan's
 * matrices:
 *   ga = g * (1 / batch),  v' = mu * v + ga
 *   D  = nesterov ? ga + mu * v' : v',  O = the steps above of D
 *   w' = w - lr_j * (sqrt(max(1, rows / cols)) * O + wd_j * w)
 * O at the plan's accuracy (the plan's dtype), all else fp32. */
int fc_muon_step(fc_muon* plan, float* w, float* v, const float* g, float lr, float mu, float wd, int batch, void* stream);

/* ---- norms around a block ------------------------------------------------ */

/* N(x) of a row x of D = `dim` elements: (x - m) / sqrt(mean((x - m)^2) + eps), m
 * the row's mean (FC_NORM_LAYER) or 0 (FC_NORM_RMS). */
#define FC_NORM_RMS 0
#define FC_NORM_LAYER 1

/* What a gate g multiplies by: a(g) = g, 1 / (1 + exp(-g)) or g / (1 + exp(-g)).  The
 * sigmoid s and 1 - s, of which the slopes are made, are off by less than 2^-20 of
 * themselves (2^-16 of a 16-bit gate), however far g is from 0 (0 where exp(-|g|) is below
 * 2^-126). */
#define FC_GATE_NONE 0
#define FC_GATE_SIGMOID 1
#define FC_GATE_SILU 2

typedef struct fc_norm fc_norm;

/* A plan for rows of `dim` elements (1 to 16384) and gradients of up to `max_tokens`
 * of them (0 to 2^31 - 1).
 *   dtype          : of the block's side: b, y, a gate per token and their gradients
 *   residual_dtype : of the residual's side: h, x, out and their gradients; `dtype`
 *                    or FC_F32
 *   kind, gate     : as above; eps > 0
 * Per-channel vectors (weights, a gate that is one) are dim contiguous fp32 elements, as
 * the flat vectors of fc.h hold them; their gradients are of a type that the call names.
 * A weight may be null: 1.  Everything is computed in fp32 and rounded once, statistics
 * included: the squares of a row must not run past its range.  Sums over tokens are
 * fp32, in an order that depends on n and dim alone.  The workspace holds up to 1280
 * rows of partial sums of two vectors, 8 bytes per element of a row (2048 rows where dim is
 * below 8). */
int fc_norm_create(fc_norm** plan, int64_t dim, int64_t max_tokens, int dtype, int residual_dtype, int kind, float eps,
                   int gate);
void fc_norm_destroy(fc_norm* plan);

/* Before a block: y[t, :] = weight * N(x[t, :]), t < n < 2^31. */
int fc_norm_before(fc_norm* plan, const void* x, int64_t ld_x, int64_t n, const float* weight, void* y,
                   int64_t ld_y, void* stream);

/* After it: out[t, :] = h[t, :] + scale * a(gate) * weight * N(b[t, :]).  gate is null
 * (a = 1), a vector (ld_gate 0) or n rows of the plan's dtype, ld_gate apart. */
int fc_norm_after(fc_norm* plan, const void* h, int64_t ld_h, const void* b, int64_t ld_b, int64_t n, const void* gate,
                  int64_t ld_gate, const float* weight, float scale, void* out, int64_t ld_out, void* stream);

/* Between two blocks: out as fc_norm_after's, y[t, :] = next_weight * N(out[t, :]) of out as
 * it is stored, in one pass. */
int fc_norm_between(fc_norm* plan, const void* h, int64_t ld_h, const void* b, int64_t ld_b, int64_t n, const void* gate,
                    int64_t ld_gate, const float* weight, const float* next_weight, float scale, void* out,
                    int64_t ld_out, void* y, int64_t ld_y, void* stream);

/* The gradients of fc_norm_before: dx = dout + N's of weight * dy (dout, the gradient
 * that comes by the residual, may be null: 0), and dweight = (accumulate ? dweight : 0) +
 * the sum over t of dy * N(x) (may be null: not wanted).  n <= max_tokens here and below. */
int fc_norm_before_grad(fc_norm* plan, const void* x, int64_t ld_x, const void* dy, int64_t ld_dy, const void* dout,
                        int64_t ld_dout, int64_t n, const float* weight, void* dx, int64_t ld_dx, void* dweight,
                        int dvec_dtype, int accumulate, void* stream);

/* The gradients of fc_norm_after (that of h is dout itself): db; dgate, a vector where the
 * gate is one (accumulate: added to) and else n rows of the plan's dtype ld_dgate apart
 * (written), may be null; dweight may be null. */
int fc_norm_after_grad(fc_norm* plan, const void* b, int64_t ld_b, const void* dout, int64_t ld_dout, int64_t n,
                       const void* gate, int64_t ld_gate, const float* weight, float scale, void* db,
                       int64_t ld_db, void* dgate, int64_t ld_dgate, void* dweight, int dvec_dtype, int accumulate,
                       void* stream);

/* The gradients of fc_norm_between, of both outputs (dout may be null: 0): dh, which is
 * out's whole gradient, as well; dnext is next_weight's. */
int fc_norm_between_grad(fc_norm* plan, const void* out, int64_t ld_out, const void* b, int64_t ld_b, const void* dy,
                         int64_t ld_dy, const void* dout, int64_t ld_dout, int64_t n, const void* gate, int64_t ld_gate,
                         const float* weight, const float* next_weight, float scale, void* dh, int64_t ld_dh,
                         void* db, int64_t ld_db, void* dgate, int64_t ld_dgate, void* dweight, void* dnext, int dvec_dtype,
                         int accumulate, void* stream);

/* ---- activations in 8 bits ------------------------------------------------- */

/* Rows in blocks of 32 neighbours that share a scale, a power of two 2^(byte - 127) (E8M0;
 * byte 255 is a NaN): the smallest, from 2^-127 on, with which no element of the block rounds
 * past the format's largest number.  An element is kept as an integer of 8 bits times it
 * (FC_BLOCK_I8, 127 the largest: steps of 1/63 to 1/128 of the block's largest magnitude), or
 * as an e4m3 float times it (FC_BLOCK_E4M3, 448 the largest: 4 bits of every element down to
 * 2^-14 of the block's largest), rounded to the nearest, ties to even.  A block that holds an
 * infinity or NaN is kept as NaN.
 *   codes  : `rows` rows of 32 * ceil(dim / 32) bytes (zeros past dim), ld_codes apart, a
 *            multiple of 16, on 16 bytes (FC_EALIGN)
 *   scales : `rows` rows of ceil(dim / 32) bytes, ld_scales apart */
#define FC_BLOCK_I8 0
#define FC_BLOCK_E4M3 1

typedef struct fc_ckpt fc_ckpt;

/* A plan for activations of `dim` elements (1 to 2^21) and gradients of weights of up to
 * max_outs rows (0 to 2^21) from up to max_tokens tokens (0 to 2^30) and a dy of `dtype`,
 * FC_F16 or FC_BF16.  The workspace, made here (none where max_outs is 0): 2 bytes per
 * element of max_tokens activations; 2 per element of dy where max_outs is no multiple of 8;
 * partial sums of products that are split along the tokens, up to 128 MiB and at most one part
 * for every 128 of max_tokens.  Layers of one dim can share a plan (of the largest max_outs), whose
 * calls run one after the other; a plan for each costs twice their checkpoints' memory. */
int fc_ckpt_create(fc_ckpt** plan, int64_t dim, int64_t max_tokens, int64_t max_outs, int dtype, int format);
void fc_ckpt_destroy(fc_ckpt* plan);

/* n rows x of any type to codes and scales; n < 2^31, here and in fc_ckpt_unpack. */
int fc_ckpt_pack(fc_ckpt* plan, const void* x, int x_dtype, int64_t ld_x, int64_t n, void* codes, int64_t ld_codes,
                 void* scales, int64_t ld_scales, void* stream);

/* out[t, :] = the numbers kept, rounded to out's type; one past its largest (a block's
 * largest element may have been rounded up to a power of two beyond) becomes that. */
int fc_ckpt_unpack(fc_ckpt* plan, const void* codes, int64_t ld_codes, const void* scales, int64_t ld_scales, int64_t n,
                   void* out, int out_dtype, int64_t ld_out, void* stream);

/* The gradient of a weight (outs, dim) whose layer's inputs x are kept so and whose outputs'
 * gradient is dy (n, outs): dw[o, :] = (accumulate ? dw[o, :] : 0) + scale * the sum over t of
 * dy[t, o] x[t, :], with x as unpacked to dy's type (exact but for what is out of fp16's range:
 * past 65504 that, below 2^-14 whole steps of 2^-24, so that less than 2^-25 is lost), products
 * and sums fp32, in whose roundings a factor of fp16 below 2^-14 counts as 2^-14, rounded once to
 * dw's type.  n <= max_tokens, outs <= max_outs (FC_EINVAL).  dy lies on 16 bytes with ld_dy a
 * multiple of 8 and is read by whole 16 bytes (of the last row, too, up to the next 8 elements), or
 * is copied, for which plans whose max_outs is no multiple of 8 have room (others: FC_EALIGN);
 * ld_dy is at most 2^21. */
int fc_ckpt_grad(fc_ckpt* plan, const void* dy, int64_t ld_dy, const void* codes, int64_t ld_codes, const void* scales,
                 int64_t ld_scales, int64_t n, int64_t outs, float scale, void* dw, int dw_dtype, int64_t ld_dw,
                 int accumulate, void* stream);

/* ---- matrices in 4 bits ------------------------------------------------------ */

/* Rows in blocks of 32 with a scale as above, of e2m1 numbers (0, 0.5, 1, 1.5, 2, 3, 4, 6 and
 * their negatives; MXFP4), and products along them on the block-scaled matrix cores.
 *   codes  : rows of 16 * ceil(dim / 32) bytes, the even element in a byte's low half (zeros
 *            past dim), ld_codes apart, a multiple of 16 and at most 2^21, on 16 bytes
 *   scales : rows of 8 * ceil(dim / 256) bytes, zeros past the blocks, ld_scales apart, a
 *            multiple of 8 and at most 2^21, on 8 bytes (FC_EALIGN, both) */
typedef struct fc_mxfp fc_mxfp;

/* A plan for products with a matrix of `rows` rows of `dim` elements (1 to 2^21 each) and up
 * to max_tokens rows (0 to 2^31 - 1).  The workspace: fc_mxfp_linear's packed inputs, 0.53
 * bytes per element of up to 2^18 tokens; the matrix's scales in another order; partial sums
 * of products that are split, up to 128 MiB and at most one part for every 512 of dim.  Any
 * number of matrices of these sizes can share a plan, whose calls run one after the other. */
int fc_mxfp_create(fc_mxfp** plan, int64_t rows, int64_t dim, int64_t max_tokens);
void fc_mxfp_destroy(fc_mxfp* plan);

/* `rows` rows (any number below 2^31) of dim elements of any type to codes and scales; with
 * `transpose` from x's columns: x has dim rows of `rows` elements. */
int fc_mxfp_pack(fc_mxfp* plan, const void* x, int x_dtype, int64_t ld_x, int64_t rows, int transpose, void* codes,
                 int64_t ld_codes, void* scales, int64_t ld_scales, void* stream);

/* The numbers kept, as fc_ckpt_unpack's. */
int fc_mxfp_unpack(fc_mxfp* plan, const void* codes, int64_t ld_codes, const void* scales, int64_t ld_scales, int64_t rows,
                   void* out, int out_dtype, int64_t ld_out, void* stream);

/* out[t, r] = (accumulate ? out[t, r] : 0) + scale * the sum over k of a[t, k] b[r, k], t < n <=
 * max_tokens, b of the plan's rows, both packed; the sum is fp32, rounded once to out's type. */
int fc_mxfp_product(fc_mxfp* plan, const void* a_codes, int64_t ld_a_codes, const void* a_scales, int64_t ld_a_scales,
                    int64_t n, const void* b_codes, int64_t ld_b_codes, const void* b_scales, int64_t ld_b_scales,
                    float scale, void* out, int out_dtype, int64_t ld_out, int accumulate, void* stream);

/* The same of n rows x of any type, packed on the way: a layer's outputs from its inputs and
 * packed weight. */
int fc_mxfp_linear(fc_mxfp* plan, const void* x, int x_dtype, int64_t ld_x, int64_t n, const void* b_codes,
                   int64_t ld_b_codes, const void* b_scales, int64_t ld_b_scales, float scale, void* out, int out_dtype,
                   int64_t ld_out, int accumulate, void* stream);

#ifdef __cplusplus
}
#endif

#endif /* FC_LM_H */
