"""Operators around an expert sublayer: the calls of include/regtopk_experts.h on torch tensors.

They stand beside those of training.py and keep their manners (current stream, errors, no CPU path, autograd does not see
them).  A sublayer is: rms_norm -> the router's product -> route -> sort_tokens -> spread_tokens -> grouped_matmul ->
activation -> grouped_matmul -> join_tokens, and back by the calls named ..._backward; the gradient of spread_tokens is
join_tokens without weights.

8-bit rows (Rows8) keep activations for the backward pass in half the memory of 16-bit ones: e4m3 numbers, and for every
32 columns of a row a power of two that they are multiplied by, the smallest with which no finite value passes 448.
Infinities and NaN become NaN.
"""
from __future__ import annotations

from typing import NamedTuple, Optional, Tuple, Union

import torch

from . import training
from .training import _load


class Rows8(NamedTuple):
    """values: float8_e4m3fn [..., cols]; scales: float8_e8m0fnu [..., ceil(cols / 32)]."""
    values: torch.Tensor
    scales: torch.Tensor


def pack8(x: torch.Tensor) -> Rows8:
    """x as 8-bit rows; rows are the last dimension."""
    return Rows8(*(training._native or _load()).pack8(x))


def unpack8(rows8: Rows8, dtype: torch.dtype = torch.bfloat16) -> torch.Tensor:
    """What 8-bit rows stand for, rounded to dtype.  float32 holds every value that pack8 gives, bfloat16 those of blocks whose scale byte is at
    least 3 (below, values are multiples of 2^-136 to 2^-134, and bfloat16's smallest number is 2^-133)."""
    return (training._native or _load()).unpack8(rows8, dtype)


def route(logits: torch.Tensor, k: int, *, scores: str = "softmax", bias: Optional[torch.Tensor] = None, groups: int = 1,
          groups_kept: int = 1, group_top: int = 1, renormalise: bool = True, scale: float = 1.0) -> Tuple[torch.Tensor, torch.Tensor]:
    """(experts int32 [..., k], weights float32 [..., k]) of each token, given its logits [..., experts].

    Scores s are the "softmax" or "sigmoid" of the logits.  Chosen are the k largest of c = s + bias, in descending order, among
    the groups_kept groups (of `groups` equal ones, neighbours) with the largest sums of their group_top (1 or 2) largest c;
    ties go to the lower index.  bias, a float32 vector, balances the load and does not enter the weights, which are the s of the
    chosen, over their sum if renormalise, times scale.

    An expert with a logit or c of -inf is never chosen; where none is left the expert is -1 and the weight 0, so a row of -inf
    keeps a token (padding, say) out of the sublayer.  Scores that float32 cannot tell apart are compared in float64."""
    return (training._native or _load()).route(logits, k, scores, bias, groups, groups_kept, group_top, renormalise, scale)


def route_backward(dweights: torch.Tensor, logits: torch.Tensor, experts: torch.Tensor, *, scores: str = "softmax",
                   renormalise: bool = True, scale: float = 1.0) -> torch.Tensor:
    """The gradient to the logits, of their shape and dtype, given the gradient of route's weights and the experts that it chose."""
    return (training._native or _load()).route_backward(dweights, logits, experts, scores, renormalise, scale)


def sort_tokens(experts: torch.Tensor, n_experts: int, workers: Optional[torch.Tensor] = None) -> Tuple[torch.Tensor, torch.Tensor]:
    """(offsets, place): the order by (worker, expert) of all pairs of a token and one of its experts, tokens ascending in a group.

    workers: int64 offsets of each worker's tokens (without it all are one worker's).  offsets, int64 [workers * n_experts + 1], are
    what grouped_matmul and grouped_matmul_dw take; place, int32 of experts' shape, is each pair's row, -1 for an expert that is
    none of the n_experts and for a token that is no worker's."""
    return (training._native or _load()).sort_tokens(experts, n_experts, workers)


def spread_tokens(x: Union[torch.Tensor, Rows8], place: torch.Tensor, offsets: torch.Tensor, dtype: Optional[torch.dtype] = None) -> torch.Tensor:
    """rows [place.numel(), cols] with rows[place[t, j]] = x[t]; those behind the last group are zeros.

    x: a row a token, as a tensor or as 8-bit rows, which are written in dtype (bfloat16 if not given).  The gradient to x is
    join_tokens(drows, place)."""
    return (training._native or _load()).spread_tokens(x, place, offsets, dtype)


def join_tokens(rows: torch.Tensor, place: torch.Tensor, weights: Optional[torch.Tensor] = None,
                residual: Optional[torch.Tensor] = None) -> torch.Tensor:
    """out[t] = residual[t] + the sum over j of weights[t, j] * rows[place[t, j]], summed in float32.

    residual, and the result with it, is of rows' dtype or float32."""
    return (training._native or _load()).join_tokens(rows, place, weights, residual)


def join_tokens_backward(dout: torch.Tensor, rows: torch.Tensor, place: torch.Tensor, weights: torch.Tensor, offsets: torch.Tensor
                         ) -> Tuple[torch.Tensor, torch.Tensor]:
    """(drows, dweights) of join_tokens with weights; the gradient to residual is dout itself, of rows' dtype or float32.

    Rows behind the last group get zeros, and so do weights without a place."""
    return (training._native or _load()).join_tokens_backward(dout, rows, place, weights, offsets)


def activation(a: torch.Tensor, kind: str = "silu", *, gated: bool = False, keep8: bool = False
               ) -> Tuple[torch.Tensor, Union[torch.Tensor, Rows8]]:
    """(y, kept): y = f(a), or f(a[..., :h]) * a[..., h:] if gated; f is "silu", "gelu" or "gelu_tanh".

    gelu is x Phi(x) with the normal distribution's Phi, of large negative x too.  float32 silu and gelu are right to 2^-20 relative, 16-bit types
    and gelu_tanh to 2^-16 before they are rounded to the type.

    kept is what activation_backward takes: a itself, or with keep8 its 8-bit rows.  The blocks of a gated a's second half begin
    anew, so that kept.values[..., h:] and the second half of kept.scales are 8-bit rows too."""
    y, kept = (training._native or _load()).activation(a, kind, gated, keep8)
    return y, Rows8(*kept) if keep8 else a


def activation_backward(dy: torch.Tensor, kept: Union[torch.Tensor, Rows8], kind: str = "silu", *, gated: bool = False,
                        want_y: bool = False) -> Tuple[torch.Tensor, Optional[torch.Tensor]]:
    """(da, y): the gradient to a of dy's dtype, taken at the values that are kept, and with want_y the output at them once more,
    for the weight gradient of the product that follows, so that y need not be kept."""
    return (training._native or _load()).activation_backward(dy, kept, kind, gated, want_y)


def rms_norm(x: torch.Tensor, weight: torch.Tensor, eps: float = 1e-6, *, residual: Optional[torch.Tensor] = None, want_y: bool = True,
             want_y8: bool = False) -> Tuple[Optional[torch.Tensor], Optional[Rows8], torch.Tensor, torch.Tensor]:
    """(y, y8, h, rstd) with h = residual + x, rstd = 1 / sqrt(mean(h^2) + eps) and y = h * rstd * weight over the last dimension.

    y comes in x's dtype (want_y) and as 8-bit rows of its float32 values (want_y8); what is not wanted is None.  residual, and h with
    it, is of x's dtype or float32; without residual h is x itself.  weight is a float32 vector; rstd is float32, one value a row, of h
    before its rounding."""
    y, y8, h, rstd = (training._native or _load()).rms_norm(x, weight, eps, residual, want_y, want_y8)
    return y, Rows8(*y8) if want_y8 else None, h, rstd


def rms_norm_backward(dy: torch.Tensor, h: torch.Tensor, rstd: torch.Tensor, weight: torch.Tensor, *, dh: Optional[torch.Tensor] = None,
                      offsets: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None, accumulate: bool = False
                      ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor]:
    """(dx, dresidual, dweight) of rms_norm, given what it returned and the gradients dy of y and dh of h.

    dweight is float32 [groups, cols], one row for each group of rows that `offsets` delimits (one group without it); given as an
    argument (any row stride, e.g. columns of an accumulator) it is written, or added to if `accumulate`.  With h of dy's dtype, dx and
    dresidual are the same tensor."""
    return (training._native or _load()).rms_norm_backward(dy, h, rstd, weight, dh, offsets, dweight, accumulate)
