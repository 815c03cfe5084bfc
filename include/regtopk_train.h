/*
 * regtopk_train.h: C ABI of the training operators that stand beside the sparsification step of regtopk.h: dropout,
 * layer norm and products grouped by expert, with their gradients, for the tokens of N workers batched on one GPU.
 *
 * A round of regtopk.h begins with every worker's gradient in that worker's row.  The calls here produce such rows:
 * the tokens of all workers lie in one array, sorted by worker (by worker and expert for the products), and each
 * weight gradient is formed per group of tokens, in binary32, and written to, or added with a single
 * round-to-nearest addition per element to, rows with any stride, e.g. those of regtopk_accumulator.
 *
 * Conventions (where they differ from regtopk.h's: there is no context)
 *   - Every pointer is a DEVICE pointer.  The caller owns every buffer, workspaces included; the library allocates no
 *     device memory.  A workspace holds nothing between calls; two calls that may run at once need one each.
 *   - Matrices are row-major; a leading dimension counts elements from one row to the next, and a row's elements are
 *     contiguous.  Any alignment that the element type allows is accepted; 16-byte aligned rows are read fastest.
 *   - Outputs overlap neither inputs nor one another, except where a call says that they may.
 *   - Calls enqueue work on cuda_stream (a cudaStream_t of the current device, NULL = default stream) and return
 *     without synchronising.  Return value: REGTOPK_OK or a negative REGTOPK_ERR_* code of regtopk.h.  Nothing aborts,
 *     throws or traps.
 *   - Statistics, sums and weight gradients are binary32 (the products' say how), and each output is rounded once.  Results do not depend on
 *     the order in which blocks run: equal calls give equal bits.
 *   - offsets arrays are int64 on the device, `groups` + 1 ascending values: group g is the rows
 *     [offsets[g], offsets[g+1]), which may be none.  The values are the caller's data and not trusted: they are
 *     limited to [0, rows], and nothing outside the outputs is touched whatever they are.
 */
#ifndef REGTOPK_TRAIN_H_
#define REGTOPK_TRAIN_H_

#include <stddef.h>
#include <stdint.h>

#include "regtopk.h"

#ifdef __cplusplus
extern "C" {
#endif

/* element types */
enum { REGTOPK_TYPE_F32 = 0, REGTOPK_TYPE_BF16 = 1, REGTOPK_TYPE_F16 = 2 };

#define REGTOPK_NORM_MAX_COLS 16384   /* widest row of a layer norm */
#define REGTOPK_NORM_MAX_GROUPS 65535 /* most groups of one layer norm's weight gradients */
#define REGTOPK_MATMUL_MAX_GROUPS 2048 /* most groups of one grouped product */
#define REGTOPK_MATMUL_MAX_SIZE 0x7FF00000 /* its largest rows, k and m, 2^31 - 2^20 */

/* Dropout with a mask that is never stored.  t = 65536 p rounded to the nearest whole number; the element in column c
 * of row r is kept if its 16-bit number n(r, c) is at least t, and is then multiplied by 65536 / (65536 - t); it is +0
 * otherwise, whatever its value was (infinities and NaN too).  n(r, c) is part of the output of Philox4x32-10 (Salmon,
 * Moraes, Dror, Shaw: "Parallel random numbers: as easy as 1, 2, 3", SC 2011) for the counter
 * (c / 8, r mod 2^32, r / 2^32, subsequence) and the key (seed mod 2^32, seed / 2^32): its word (c mod 8) / 2, the
 * word's low half for even c and its high half for odd c.  The mask depends on the position alone, not on the type,
 * strides or address, so the same call on dy is the backward pass.
 *   drop = { p in [0, 1], seed, subsequence }; use another subsequence for every layer and step of one seed.       */
typedef struct {
  double p;
  uint64_t seed;
  uint32_t subsequence;
} regtopk_dropout_params;

/* y = dropout(x), both [rows][cols] of `type`; y may be x.  rows, cols >= 0; cols <= 2^34.
 * Errors: INVALID_ARG, NO_DEVICE, CUDA. */
int regtopk_dropout(const void* x, int64_t ldx, void* y, int64_t ldy, int64_t rows, int64_t cols, int32_t type,
                    const regtopk_dropout_params* drop, void* cuda_stream);

/* Layer norm, alone or as the end of a sublayer:
 *   h = residual + dropout(x)                     (residual NULL: h = dropout(x); drop NULL: no dropout)
 *   mean, rstd = mean(h), 1 / sqrt(mean((h - mean)^2) + eps) over each row, of h before it is rounded
 *   y = (h - mean) * rstd * weight + bias         (bias NULL: 0)
 * x, y [rows][cols] of `type`; residual, h [rows][cols] of `stream_type`, which is `type` or F32; h NULL: not written.
 * weight, bias [cols] and mean, rstd [rows] binary32.  1 <= cols <= REGTOPK_NORM_MAX_COLS, rows >= 0, eps >= 0.
 * Errors: INVALID_ARG, TOO_LARGE, NO_DEVICE, CUDA. */
int regtopk_layer_norm(const void* x, int64_t ldx, const void* residual, int64_t ld_residual, const float* weight,
                       const float* bias, float eps, void* y, int64_t ldy, void* h, int64_t ldh, float* mean,
                       float* rstd, int64_t rows, int64_t cols, int32_t type, int32_t stream_type,
                       const regtopk_dropout_params* drop, void* cuda_stream);

/* The gradients of regtopk_layer_norm, given h (x itself where it was not written), mean, rstd and weight:
 *   u = (h - mean) * rstd,  g = dy * weight
 *   dresidual = dh + rstd * (g - mean(g) - u * mean(g * u))    (dh, the gradient that reached h otherwise; NULL: 0)
 *   dx = dropout(dresidual), the mask of the forward pass
 *   dweight[n] (+)= sum of dy * u,  dbias[n] (+)= sum of dy,  over the rows of group n, each in row n of its array
 * dy, dx of `type`; h, dh, dresidual of `stream_type`; dresidual NULL: not written.  dweight, dbias binary32 with
 * leading dimensions of their own, NULL: not wanted.  offsets NULL: one group of all rows (groups is then 1);
 * 1 <= groups <= REGTOPK_NORM_MAX_GROUPS.
 * accumulate != 0 adds to what dweight and dbias hold.  Rows of no group get their dx and add to no weight gradient.
 * workspace: 16-byte aligned, at least regtopk_layer_norm_backward_workspace_bytes(rows, cols, groups) bytes; may be NULL
 * if neither dweight nor dbias is wanted.  Errors: as above, and WORKSPACE_TOO_SMALL. */
size_t regtopk_layer_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int32_t groups);
int regtopk_layer_norm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ldh, const float* mean,
                                const float* rstd, const float* weight, const void* dh, int64_t ld_dh, void* dx,
                                int64_t ld_dx, void* dresidual, int64_t ld_dresidual, float* dweight,
                                int64_t ld_dweight, float* dbias, int64_t ld_dbias, const int64_t* offsets,
                                int32_t groups, int32_t accumulate, int64_t rows, int64_t cols, int32_t type,
                                int32_t stream_type, const regtopk_dropout_params* drop, void* workspace,
                                size_t workspace_bytes, void* cuda_stream);

/* Products of rows with the matrix of their group (the tokens of each expert with that expert's weights):
 *   y[t] = w[g mod weights] x[t]   for the rows t of group g; a row of no group gets zeros.
 * x [rows][k] and y [rows][m] of `type`, which is BF16 or F16; w holds `weights` matrices, element (i, j) of matrix e at
 * w[e * w_stride + i * ldw + j].  transposed == 0: matrices [m][k], as a linear layer keeps them.  transposed != 0:
 * matrices [k][m], used as y[t] = x[t] w: with dy for x and the layer's own [m][k] matrices this is the gradient to the
 * tokens.  groups is a multiple of weights: groups sorted by (worker, expert) share the experts' matrices.
 * Products are exact and sums binary32 on the tensor cores, which cut the running sum off where an addition would round: sums of up to
 * 4,096 terms are some 3e-5 of the sum of magnitudes too small at most, and longer ones are joined from such by rounded additions.  y is
 * rounded once.  rows, k, m <= REGTOPK_MATMUL_MAX_SIZE; k == 0 gives zeros.
 * workspace: 16-byte aligned, at least regtopk_grouped_matmul_workspace_bytes(...) bytes, which hold a copy of
 * x or w where it has no 16-byte aligned rows (base and leading dimension; for w the stride between matrices too), and partial
 * sums where k is long and there are few rows; often 0.  Errors: INVALID_ARG, TOO_LARGE (groups), WORKSPACE_TOO_SMALL, NO_DEVICE, CUDA. */
size_t regtopk_grouped_matmul_workspace_bytes(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t w_stride,
                                              int32_t transposed, int32_t weights, int32_t groups, int64_t rows, int64_t k,
                                              int64_t m);
int regtopk_grouped_matmul(const void* x, int64_t ldx, const void* w, int64_t ldw, int64_t w_stride, int32_t transposed,
                           int32_t weights, void* y, int64_t ldy, const int64_t* offsets, int32_t groups, int64_t rows,
                           int64_t k, int64_t m, int32_t type, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* The gradient of such products to the matrices, for each group on its own:
 *   out[g] (+)= sum over the rows t of group g of dy[t] x[t]^T, an [m][k] matrix; a group without rows gives zeros.
 * dy [rows][m] and x [rows][k] of `type` (BF16 or F16); out binary32, element (i, j) of group g = n * inner + e at
 * out[n * outer_stride + e * inner_stride + i * ld_out + j]: with inner experts and groups sorted by (worker, expert) this is
 * each worker's own row of a flat gradient.  No two rows of out may overlap (INVALID_ARG: blocks write them at once).
 * accumulate != 0 adds to what out holds, one rounded addition per element.  The tensor cores' sums of up to 512 rows are joined by
 * rounded additions: 2 to 5e-7 of the result off.
 * workspace as above, by regtopk_grouped_matmul_dw_workspace_bytes.  Errors as above. */
size_t regtopk_grouped_matmul_dw_workspace_bytes(const void* dy, int64_t ld_dy, const void* x, int64_t ldx, int32_t groups,
                                                 int64_t rows, int64_t k, int64_t m);
int regtopk_grouped_matmul_dw(const void* dy, int64_t ld_dy, const void* x, int64_t ldx, float* out, int64_t ld_out,
                              int64_t inner_stride, int64_t outer_stride, int32_t inner, int32_t accumulate,
                              const int64_t* offsets, int32_t groups, int64_t rows, int64_t k, int64_t m, int32_t type,
                              void* workspace, size_t workspace_bytes, void* cuda_stream);

/* Synchronises the stream.  REGTOPK_OK, REGTOPK_ERR_CUDA, or REGTOPK_ERR_INTERNAL if a kernel of the norms or the products on
 * the current device ever gave up waiting for its own copies or tensor core work (every such wait ends after four billion
 * cycles; the outputs of that call are then incomplete).  The internal error stays set until the process ends. */
int regtopk_train_status(void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* REGTOPK_TRAIN_H_ */
