/*
 * fc_lm.h -- C ABI of the operators at the ends of a language model and of its
 * matrix update, for MI355X (gfx950): what produces the gradients that fc.h
 * aggregates, and what else may consume their sum.
 *   fc_embed : scaled rows of a table for a list of tokens, and the table's
 *              gradient, summed token by token in sorted order
 *   fc_xent  : softmax cross entropy over a vocabulary, computed in pieces of
 *              the vocabulary without storing the logits, with both gradients
 *              (for which 16-bit exponentials are kept, see fc_xent_create)
 *   fc_muon  : momentum updates made orthogonal by Newton-Schulz products,
 *              for every matrix of a flat parameter vector at once
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
 *     neither waits for the plan's previous call nor becomes it.
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

#ifdef __cplusplus
}
#endif

#endif /* FC_LM_H */
