/*
 * regtopk_experts.h: C ABI of the operators around an expert sublayer, for the tokens of N workers batched on one GPU:
 * the router's choice of experts, the tokens' way into the order of their (worker, expert) groups and back, gated
 * activations whose input is kept in 8 bits for the backward pass, and the root-mean-square norm, with their gradients.
 *
 * They stand beside the calls of regtopk_train.h and keep its conventions: device pointers, buffers and workspaces of the
 * caller's, row-major matrices with leading dimensions in elements, work enqueued on cuda_stream, REGTOPK_OK or a negative
 * REGTOPK_ERR_* code, equal bits from equal calls.  regtopk_sort_tokens makes the offsets that regtopk_grouped_matmul and
 * regtopk_grouped_matmul_dw take.  The values of index arrays (experts, places, offsets) are the caller's data and not trusted:
 * one that is out of range counts as "none", and nothing outside the outputs is touched whatever they are.
 *
 * 8-bit rows.  A row of cols elements is kept as cols bytes, e4m3 numbers, and ceil(cols / 32) scale bytes, one for every 32
 * columns: byte b stands for 2^(b - 127), an element for its number times that (the elements and scales of the OCP
 * microscaling formats, MXFP8, v1.0).  b is the smallest with which no finite value of the block passes 448 * 2^(b - 127), at
 * least 0; elements are rounded to nearest, ties to even.  Infinities and NaN become NaN and do not count for the block's
 * scale.  Scale byte 255 is read as NaN and never written.  Leading dimensions count bytes.
 */
#ifndef REGTOPK_EXPERTS_H_
#define REGTOPK_EXPERTS_H_

#include <stddef.h>
#include <stdint.h>

#include "regtopk_train.h"

#ifdef __cplusplus
extern "C" {
#endif

#define REGTOPK_ROUTE_MAX_EXPERTS 512 /* most experts to choose from */
#define REGTOPK_ROUTE_MAX_CHOICES 32  /* most experts of one token */
#define REGTOPK_ROUTE_MAX_GROUPS 32   /* most groups of experts */

/* x [rows][cols] of `type` to 8-bit rows, and back.  rows, cols >= 0, cols <= 2^30.  Errors: INVALID_ARG, NO_DEVICE, CUDA. */
int regtopk_pack8(const void* x, int64_t ldx, uint8_t* values, int64_t ld_values, uint8_t* scales, int64_t ld_scales,
                  int64_t rows, int64_t cols, int32_t type, void* cuda_stream);
int regtopk_unpack8(const uint8_t* values, int64_t ld_values, const uint8_t* scales, int64_t ld_scales, void* x, int64_t ldx,
                    int64_t rows, int64_t cols, int32_t type, void* cuda_stream);

enum { REGTOPK_SCORES_SOFTMAX = 0, REGTOPK_SCORES_SIGMOID = 1 };

/* How experts are chosen: see regtopk_route. */
typedef struct {
  int32_t scores;      /* REGTOPK_SCORES_* */
  int32_t groups;      /* equal groups of neighbouring experts; 1: no groups */
  int32_t groups_kept; /* how many of them a token may choose from, 1 to groups */
  int32_t group_top;   /* 1 or 2: how many of its scores a group is judged by */
  int32_t renormalise; /* != 0: the weights of a token's experts sum up to `scale` */
  float scale;
} regtopk_route_params;

/* The router.  For every token
 *   s = softmax(l) or sigmoid(l) over the n_experts logits l;  c = s + bias  (bias NULL: c = s)
 *   groups: the groups_kept groups with the largest sums of their group_top largest c remain
 *   experts[t]: the k experts with the largest c among those, in descending order
 *   weights[t]: their s, divided by the sum of them if renormalise, times scale
 * Ties go to the lower index, of groups and of experts.  The choice is that of binary64 arithmetic on the given numbers: tokens among
 * whose numbers binary32 cannot tell two apart are done again in it (without bias experts are compared by their logits); exponentials of less than
 * -708 are 0 there.  An expert whose logit or c is
 * -infinity is never chosen; places for which no expert is left hold -1 and weight 0.  A NaN or +infinity among the logits
 * makes the token's softmax scores NaN; NaN is the least c that can be chosen, and counts as -1e300 in the sum of a group.
 * logits [tokens][n_experts] of `type`; bias [n_experts] binary32; experts int32 and weights binary32, [tokens][k] contiguous.
 * 1 <= n_experts <= REGTOPK_ROUTE_MAX_EXPERTS, 1 <= k <= min(REGTOPK_ROUTE_MAX_CHOICES, n_experts), groups divides n_experts.
 * Errors: INVALID_ARG, TOO_LARGE, NO_DEVICE, CUDA. */
int regtopk_route(const void* logits, int64_t ld_logits, const float* bias, int32_t* experts, float* weights, int64_t tokens,
                  int32_t n_experts, int32_t k, int32_t type, const regtopk_route_params* params, void* cuda_stream);

/* The gradient of the weights to the logits, for the experts that were chosen (the choice itself has none; bias gets none).
 * dlogits [tokens][n_experts] of `type` is written whole.  An expert of -1 had no weight.  Errors as above. */
int regtopk_route_backward(const float* dweights, const void* logits, int64_t ld_logits, const int32_t* experts, void* dlogits,
                           int64_t ld_dlogits, int64_t tokens, int32_t n_experts, int32_t k, int32_t type,
                           const regtopk_route_params* params, void* cuda_stream);

/* The places of (token, choice) pairs in the order of their (worker, expert) groups, tokens ascending within each.
 * workers_at: int64 [workers + 1], where each worker's tokens begin and the last one's end; NULL: all tokens are of one worker.
 * offsets: int64 [workers * n_experts + 1], where each group's rows begin, and the number of rows; place int32 [tokens][k]: the row of
 * each pair, -1 where the expert is none of 0 .. n_experts - 1 or the token is of no worker.  experts as regtopk_route writes it.
 * workers * n_experts <= REGTOPK_MATMUL_MAX_GROUPS, tokens * k < 2^31.  workspace: 16-byte aligned, at least
 * regtopk_sort_tokens_workspace_bytes(...) bytes; often 0.  Errors: INVALID_ARG, TOO_LARGE, WORKSPACE_TOO_SMALL, NO_DEVICE, CUDA. */
size_t regtopk_sort_tokens_workspace_bytes(int64_t tokens, int32_t k, int32_t n_experts, int32_t workers);
int regtopk_sort_tokens(const int32_t* experts, const int64_t* workers_at, int32_t workers, int64_t* offsets, int32_t* place,
                        int64_t tokens, int32_t k, int32_t n_experts, void* workspace, size_t workspace_bytes, void* cuda_stream);

/* out[place[t][j]] = x[t]: every token's row to the places of its experts; rows from *filled on become zeros.
 * x [tokens][cols] of `type`, or, where scales is not NULL, the values of 8-bit rows; out [rows][cols] of `type`.  filled: int64 on
 * the device, the last of regtopk_sort_tokens's offsets; NULL: no row is cleared.  Places are distinct.
 * Its gradient is regtopk_join_tokens without weights.  k as above, cols <= 2^30.  Errors: INVALID_ARG, TOO_LARGE, NO_DEVICE, CUDA. */
int regtopk_spread_tokens(const void* x, int64_t ldx, const uint8_t* scales, int64_t ld_scales, const int32_t* place,
                          const int64_t* filled, void* out, int64_t ld_out, int64_t tokens, int32_t k, int64_t rows, int64_t cols,
                          int32_t type, void* cuda_stream);

/* out[t] = residual[t] + sum over j of weights[t][j] * from[place[t][j]]     (weights NULL: 1; residual NULL: 0)
 * from [rows][cols] of `type`; residual and out [tokens][cols] of out_type, which is `type` or F32; out may be residual. */
int regtopk_join_tokens(const void* from, int64_t ld_from, const int32_t* place, const float* weights, const void* residual,
                        int64_t ld_residual, void* out, int64_t ld_out, int64_t tokens, int32_t k, int64_t rows, int64_t cols,
                        int32_t type, int32_t out_type, void* cuda_stream);

/* The gradients of regtopk_join_tokens with weights (that of residual is dout itself):
 *   dfrom[place[t][j]] = weights[t][j] * dout[t],  dweights[t][j] = sum over the columns of dout[t] * from[place[t][j]]
 * rows of dfrom from *filled on become zeros, and dweights is 0 where there is no place.  dout of dout_type, `type` or F32; tokens < 2^31. */
int regtopk_join_tokens_backward(const void* dout, int64_t ld_dout, const void* from, int64_t ld_from, const int32_t* place,
                                 const float* weights, const int64_t* filled, void* dfrom, int64_t ld_dfrom, float* dweights,
                                 int64_t tokens, int32_t k, int64_t rows, int64_t cols, int32_t type, int32_t dout_type,
                                 void* cuda_stream);

/* silu(x) = x / (1 + exp(-x));  gelu(x) = x Phi(x), Phi the normal distribution's;  gelu_tanh: Phi approximated by
 * (1 + tanh(sqrt(2/pi) (x + 0.044715 x^3))) / 2.
 * How good they are: p = f(x) / x and the terms p and x p'(x) of the slope are right to 2^-20 relative for silu and gelu in binary32; for gelu_tanh in
 * binary32, and for 16-bit types before they are rounded to the type (by 2^-9 or 2^-12), to 2^-16, and to 2^-15 where p is below 2^-40.  A p of less
 * than 2^-125 may be 0. */
enum { REGTOPK_ACTIVATION_SILU = 0, REGTOPK_ACTIVATION_GELU = 1, REGTOPK_ACTIVATION_GELU_TANH = 2 };

/* y = f(a), a [rows][cols]; gated != 0: y = f(a[:, :cols]) * a[:, cols:], a [rows][2 cols].  y [rows][cols]; both of `type`.
 * values not NULL: a is kept as 8-bit rows as well; with gated, each half of a row is a row of its own, so that values is [rows][2 cols]
 * and scales [rows][2 ceil(cols / 32)].  rows, cols >= 0, cols <= 2^30.  Errors: INVALID_ARG, NO_DEVICE, CUDA. */
int regtopk_activation(const void* a, int64_t lda, void* y, int64_t ldy, uint8_t* values, int64_t ld_values, uint8_t* scales,
                       int64_t ld_scales, int64_t rows, int64_t cols, int32_t kind, int32_t gated, int32_t type, void* cuda_stream);

/* da, the gradient to a, given dy and a (scales NULL: of `type`; otherwise a is the values of 8-bit rows, and the gradient is the
 * one at what they stand for); y not NULL: the output once more, of the same a. */
int regtopk_activation_backward(const void* dy, int64_t ld_dy, const void* a, int64_t lda, const uint8_t* scales, int64_t ld_scales,
                                void* da, int64_t ld_da, void* y, int64_t ldy, int64_t rows, int64_t cols, int32_t kind, int32_t gated,
                                int32_t type, void* cuda_stream);

/* Root-mean-square norm, alone or behind a residual sum:
 *   h = residual + x  (residual NULL: h = x);  rstd = 1 / sqrt(mean(h^2) + eps) over each row, of h before it is rounded
 *   y = h * rstd * weight, of `type` (NULL: not written) and as 8-bit rows of its binary32 values (values NULL: not written)
 * x, y [rows][cols] of `type`; residual, h [rows][cols] of stream_type, which is `type` or F32; h NULL: not written.
 * weight [cols] and rstd [rows] binary32.  1 <= cols <= REGTOPK_NORM_MAX_COLS, rows >= 0, eps >= 0.  The sum of a row's squares is a
 * binary32 number.  Errors: INVALID_ARG, TOO_LARGE, NO_DEVICE, CUDA. */
int regtopk_rms_norm(const void* x, int64_t ldx, const void* residual, int64_t ld_residual, const float* weight, float eps, void* y,
                     int64_t ldy, uint8_t* values, int64_t ld_values, uint8_t* scales, int64_t ld_scales, void* h, int64_t ldh,
                     float* rstd, int64_t rows, int64_t cols, int32_t type, int32_t stream_type, void* cuda_stream);

/* The gradients of regtopk_rms_norm, given h (x itself where it was not written), rstd and weight:
 *   u = h * rstd,  g = dy * weight,  dresidual = dh + rstd * (g - u * mean(g * u)),  dx = dresidual
 *   dweight[n] (+)= sum of dy * u over the rows of group n
 * with the arguments, types, groups and workspace of regtopk_layer_norm_backward (regtopk_train.h). */
size_t regtopk_rms_norm_backward_workspace_bytes(int64_t rows, int64_t cols, int32_t groups);
int regtopk_rms_norm_backward(const void* dy, int64_t ld_dy, const void* h, int64_t ldh, const float* rstd, const float* weight,
                              const void* dh, int64_t ld_dh, void* dx, int64_t ld_dx, void* dresidual, int64_t ld_dresidual,
                              float* dweight, int64_t ld_dweight, const int64_t* offsets, int32_t groups, int32_t accumulate,
                              int64_t rows, int64_t cols, int32_t type, int32_t stream_type, void* workspace, size_t workspace_bytes,
                              void* cuda_stream);

#ifdef __cplusplus
}
#endif
#endif /* REGTOPK_EXPERTS_H_ */
