"""Training operators that fill the sparsifier's accumulator rows: the calls of include/regtopk_train.h on torch tensors.

The tokens of all N workers lie in one array, sorted by worker (by worker and expert for the products); `offsets`, an
int64 device tensor, says where each group of rows begins and where the last one ends.  Weight gradients are float32
and come per group; they may be written, or added, straight into views of RegTopK.accumulator().

Everything runs on the current torch stream of the tensors' device and is asynchronous like any torch CUDA op; autograd
does not see it, the gradients are calls of their own.  A tensor given to be written must not require a gradient while autograd
records; its version goes up as with torch's in-place operations.  There is no CPU path: if the library is missing or a tensor is
not on a CUDA device, the calls raise.  Wrong types, shapes and devices raise TypeError, wrong values and strides
ValueError, and what the library refuses or fails at RegTopKError.
"""
from __future__ import annotations

import importlib
from typing import Optional, Tuple

import torch

from .binding import RegTopKError

_native = None


def _load():
    """The compiled marshalling module (csrc/training_binding.cpp), which brings the CUDA library with it."""
    global _native
    if _native is None:
        try:
            module = importlib.import_module(__package__ + "._training")
        except ModuleNotFoundError as e:
            raise RuntimeError("the training operators are missing: run paper_2501_05633_b200.build() (needs nvcc); "
                               "there is no CPU implementation to fall back to") from e
        module.raise_with(RegTopKError, torch.OutOfMemoryError)
        _native = module
    return _native


def dropout(x: torch.Tensor, p: float, seed: int, subsequence: int = 0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x with each element kept with probability 1 - t / 65536 and then scaled by its inverse, t = round(65536 p).

    The mask is a function of the element's row and column, seed and subsequence alone (regtopk_train.h states it), and
    is not stored: the same call on the gradient is the backward pass.  Rows are the last dimension.  out may be x, but must
    not overlap it otherwise."""
    return (_native or _load()).dropout(x, p, seed, subsequence, out)


def layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, *,
               residual: Optional[torch.Tensor] = None, p: float = 0.0, seed: int = 0, subsequence: int = 0
               ) -> Tuple[torch.Tensor, torch.Tensor, torch.Tensor, torch.Tensor]:
    """(y, h, mean, rstd) with h = residual + dropout(x) and y = (h - mean) * rstd * weight + bias over the last dimension.

    Without residual and dropout h is x itself.  residual, and h with it, is of x's dtype or float32; weight and bias
    are float32 vectors (views of the flat parameter vector will do); mean and rstd are float32, one value a row, of h
    before its rounding."""
    return (_native or _load()).layer_norm(x, weight, bias, eps, residual, p, seed, subsequence)


def layer_norm_backward(dy: torch.Tensor, h: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: torch.Tensor, *,
                        dh: Optional[torch.Tensor] = None, p: float = 0.0, seed: int = 0, subsequence: int = 0,
                        offsets: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                        dbias: Optional[torch.Tensor] = None, accumulate: bool = False
                        ) -> Tuple[torch.Tensor, torch.Tensor, Optional[torch.Tensor], Optional[torch.Tensor]]:
    """(dx, dresidual, dweight, dbias) of layer_norm, given what it returned and the gradients dy of y and dh of h.

    dweight and dbias are float32 [groups, cols], one row for each group of rows that `offsets` delimits (one group
    without it); given as arguments (any row stride, e.g. columns of an accumulator) they are written, or added to if
    `accumulate`, and one that is not given while the other is stays None; if neither is given both are made here.
    Without dropout, and with h of dy's dtype, dx and dresidual are the same tensor."""
    return (_native or _load()).layer_norm_backward(dy, h, mean, rstd, weight, dh, p, seed, subsequence, offsets, dweight, dbias,
                                                    accumulate)


def grouped_matmul(x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [rows, m] with y[t] = w[g % E] @ x[t] for the rows t of group g; rows of no group become zeros.

    x [rows, k] and w [E, m, k] are both bfloat16 or both float16; either of w's last two dimensions may be the
    contiguous one, so w.transpose(1, 2) of a layer's weights gives the gradient to its tokens.  The number of groups
    is a multiple of E: groups sorted by (worker, expert) use the experts' matrices in turn."""
    return (_native or _load()).grouped_matmul(x, w, offsets, out)


def grouped_matmul_dw(dy: torch.Tensor, x: torch.Tensor, offsets: torch.Tensor, out: Optional[torch.Tensor] = None,
                      accumulate: bool = False) -> torch.Tensor:
    """The gradient of grouped_matmul to the matrices, for every group on its own: out[g] = sum of dy[t] x[t]^T over
    the rows t of group g, float32 [groups, m, k].

    out may be given, as [groups, m, k] or [workers, experts, m, k] with contiguous rows of which no two
    overlap (a view of an accumulator's columns, say), and is added to if `accumulate`."""
    return (_native or _load()).grouped_matmul_dw(dy, x, offsets, out, accumulate)


def training_status(device=None):
    """Synchronises the device's current stream; raises if one of these kernels there ever gave up waiting (a bug)."""
    with torch.cuda.device(device):
        (_native or _load()).status(torch.cuda.current_stream().cuda_stream)
