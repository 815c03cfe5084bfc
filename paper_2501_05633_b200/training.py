"""Training operators that fill the sparsifier's accumulator rows: ctypes marshalling of include/regtopk_train.h.

The tokens of all N workers lie in one array, sorted by worker (by worker and expert for the products); `offsets`, an
int64 device tensor, says where each group of rows begins and where the last one ends.  Weight gradients are binary32
and come per group; they may be written, or added, straight into views of RegTopK.accumulator().

Everything runs on the device's current torch stream and is asynchronous like any torch CUDA op.  There is no CPU
path: if the library is missing or a tensor is not on a CUDA device, the calls raise.
"""
from __future__ import annotations

import ctypes
import os
from typing import Optional, Tuple

import torch

from .binding import OK, RegTopKError

_PKG = os.path.dirname(os.path.abspath(__file__))
_LIB = os.path.join(_PKG, "libregtopk_train.so")

EXPORTS = [
    "regtopk_dropout", "regtopk_layer_norm", "regtopk_layer_norm_backward_workspace_bytes",
    "regtopk_layer_norm_backward", "regtopk_grouped_matmul_workspace_bytes", "regtopk_grouped_matmul",
    "regtopk_grouped_matmul_dw_workspace_bytes", "regtopk_grouped_matmul_dw", "regtopk_train_status",
]

TYPES = {torch.float32: 0, torch.bfloat16: 1, torch.float16: 2}


class DropoutParams(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("subsequence", ctypes.c_uint32)]


_lib = None


def load_library():
    """dlopen the CUDA library and declare its signatures. Raises if it has not been built."""
    global _lib
    if _lib is not None:
        return _lib
    if not os.path.exists(_LIB):
        raise RuntimeError(f"{_LIB} is missing: run paper_2501_05633_b200.build() (needs nvcc); "
                           "there is no CPU implementation to fall back to")
    L = ctypes.CDLL(_LIB)
    vp, i64, i32, f32, size = ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t
    drop = ctypes.POINTER(DropoutParams)
    L.regtopk_dropout.argtypes = [vp, i64, vp, i64, i64, i64, i32, drop, vp]
    L.regtopk_layer_norm.argtypes = [vp, i64, vp, i64, vp, vp, f32, vp, i64, vp, i64, vp, vp, i64, i64, i32, i32, drop, vp]
    L.regtopk_layer_norm_backward_workspace_bytes.argtypes = [i64, i64, i32]
    L.regtopk_layer_norm_backward_workspace_bytes.restype = size
    L.regtopk_layer_norm_backward.argtypes = [vp, i64, vp, i64, vp, vp, vp, vp, i64, vp, i64, vp, i64, vp, i64, vp, i64, vp,
                                              i32, i32, i64, i64, i32, i32, drop, vp, size, vp]
    L.regtopk_grouped_matmul_workspace_bytes.argtypes = [vp, i64, vp, i64, i64, i32, i32, i64, i64, i64]
    L.regtopk_grouped_matmul_workspace_bytes.restype = size
    L.regtopk_grouped_matmul.argtypes = [vp, i64, vp, i64, i64, i32, i32, vp, i64, vp, i32, i64, i64, i64, i32, vp, size, vp]
    L.regtopk_grouped_matmul_dw_workspace_bytes.argtypes = [vp, i64, vp, i64, i32, i64, i64, i64]
    L.regtopk_grouped_matmul_dw_workspace_bytes.restype = size
    L.regtopk_grouped_matmul_dw.argtypes = [vp, i64, vp, i64, vp, i64, i64, i64, i32, i32, vp, i32, i64, i64, i64, i32, vp, size, vp]
    L.regtopk_train_status.argtypes = [vp]
    _lib = L
    return L


def _check(code: int, where: str):
    if code != OK:
        raise RegTopKError(code, where)


def _type(t: torch.Tensor, name: str) -> int:
    if not t.is_cuda:
        raise TypeError(f"{name} must live on the device")
    code = TYPES.get(t.dtype)
    if code is None:
        raise TypeError(f"{name} is float32, bfloat16 or float16")
    return code


def _rows(t: torch.Tensor, name: str) -> Tuple[int, int, int]:
    """(rows, cols, leading dimension) of a tensor whose last dimension is the row."""
    shape = t.shape
    n = len(shape)
    if n == 0:
        raise ValueError(f"{name} needs at least one dimension")
    if n > 2:
        t = t.view(-1, shape[-1]) if t.numel() else t.reshape(0, shape[-1])  # raises where no single stride fits
    rows, cols = (1, shape[0]) if n == 1 else t.shape
    if cols > 1 and t.stride(-1) != 1:
        raise ValueError(f"{name}: the elements of a row must be contiguous")
    ld = t.stride(0) if n > 1 and rows > 1 else cols
    if ld < cols:
        raise ValueError(f"{name}: rows overlap")
    return rows, cols, ld


def _like(t: torch.Tensor, x: torch.Tensor, name: str, dtypes) -> int:
    """Checks that t has x's shape and device and one of the dtypes; its leading dimension."""
    if t.device != x.device or t.shape != x.shape or t.dtype not in dtypes:
        raise TypeError(f"{name} must match the input's shape and device and be of {' or '.join(str(d) for d in dtypes)}")
    return _rows(t, name)[2]


def _vector(t: torch.Tensor, n: int, x: torch.Tensor, name: str):
    if t.device != x.device or t.dtype != torch.float32 or t.numel() != n or not t.is_contiguous():
        raise TypeError(f"{name} must be {n} contiguous float32 values on the input's device")


def _dropout_params(p: float, seed: int, subsequence: int):
    if not 0.0 <= p <= 1.0:
        raise ValueError("p is a probability")
    if not 0 <= seed < 1 << 64 or not 0 <= subsequence < 1 << 32:
        raise ValueError("seed has 64 bits and subsequence 32")
    return DropoutParams(p, seed, subsequence)


def _offsets(offsets: torch.Tensor, x: torch.Tensor) -> int:
    """The number of groups."""
    if offsets.device != x.device or offsets.dtype != torch.int64 or offsets.dim() != 1 or not offsets.is_contiguous() or len(offsets) < 2:
        raise TypeError("offsets must be a contiguous int64 vector of at least two values on the input's device")
    return len(offsets) - 1


class _on:
    """Makes the tensor's device current for a call, if it is not; .stream is that device's current stream."""
    __slots__ = ("index", "old", "stream")

    def __init__(self, t: torch.Tensor):
        self.index, self.old = t.device.index, -1

    def __enter__(self):
        now = torch.cuda.current_device()
        if now != self.index:
            self.old = now
            torch.cuda.set_device(self.index)
        self.stream = torch.cuda.current_stream().cuda_stream
        return self

    def __exit__(self, *exc):
        if self.old >= 0:
            torch.cuda.set_device(self.old)


def dropout(x: torch.Tensor, p: float, seed: int, subsequence: int = 0, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """x with each element kept with probability 1 - t / 65536 and then scaled by its inverse, t = round(65536 p).

    The mask is a function of the element's row and column, seed and subsequence alone (regtopk_train.h states it), and
    is not stored: the same call on the gradient is the backward pass.  Rows are the last dimension.  out may be x."""
    code = _type(x, "x")
    rows, cols, ld = _rows(x, "x")
    if out is None:
        out = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    ld_out = _like(out, x, "out", (x.dtype,))
    params = _dropout_params(p, seed, subsequence)
    with _on(x) as on:
        _check(load_library().regtopk_dropout(x.data_ptr(), ld, out.data_ptr(), ld_out, rows, cols, code, params, on.stream),
               "regtopk_dropout")
    return out


def layer_norm(x: torch.Tensor, weight: torch.Tensor, bias: Optional[torch.Tensor] = None, eps: float = 1e-5, *,
               residual: Optional[torch.Tensor] = None, p: float = 0.0, seed: int = 0, subsequence: int = 0):
    """(y, h, mean, rstd) with h = residual + dropout(x) and y = (h - mean) * rstd * weight + bias over the last dimension.

    Without residual and dropout h is x itself.  residual, and h with it, is of x's dtype or float32; weight and bias
    are float32 vectors (views of the flat parameter vector will do); mean and rstd are float32, one value a row, of h
    before its rounding."""
    code = _type(x, "x")
    rows, cols, ld = _rows(x, "x")
    _vector(weight, cols, x, "weight")
    if bias is not None:
        _vector(bias, cols, x, "bias")
    stream_dtype, ld_res = x.dtype, 0
    if residual is not None:
        ld_res = _like(residual, x, "residual", (x.dtype, torch.float32))
        stream_dtype = residual.dtype
    drop = _dropout_params(p, seed, subsequence) if p else None
    y = torch.empty(x.shape, dtype=x.dtype, device=x.device)
    own_h = residual is not None or drop is not None
    h = torch.empty(x.shape, dtype=stream_dtype, device=x.device) if own_h else x
    stats = torch.empty((2,) + x.shape[:-1], dtype=torch.float32, device=x.device)
    mean, rstd = stats[0], stats[1]
    with _on(x) as on:
        _check(load_library().regtopk_layer_norm(
            x.data_ptr(), ld, residual.data_ptr() if residual is not None else None, ld_res, weight.data_ptr(),
            bias.data_ptr() if bias is not None else None, eps, y.data_ptr(), cols, h.data_ptr() if own_h else None, cols,
            mean.data_ptr(), rstd.data_ptr(), rows, cols, code, TYPES[stream_dtype], drop, on.stream), "regtopk_layer_norm")
    return y, h, mean, rstd


def _gradient_rows(t: Optional[torch.Tensor], groups: int, cols: int, x: torch.Tensor, name: str) -> int:
    if t is None:
        return 0
    if t.device != x.device or t.dtype != torch.float32 or t.shape != (groups, cols):
        raise TypeError(f"{name} must be float32 [{groups}, {cols}] on the input's device")
    return _rows(t, name)[2]


def layer_norm_backward(dy: torch.Tensor, h: torch.Tensor, mean: torch.Tensor, rstd: torch.Tensor, weight: torch.Tensor, *,
                        dh: Optional[torch.Tensor] = None, p: float = 0.0, seed: int = 0, subsequence: int = 0,
                        offsets: Optional[torch.Tensor] = None, dweight: Optional[torch.Tensor] = None,
                        dbias: Optional[torch.Tensor] = None, accumulate: bool = False):
    """(dx, dresidual, dweight, dbias) of layer_norm, given what it returned and the gradients dy of y and dh of h.

    dweight and dbias are float32 [groups, cols], one row for each group of rows that `offsets` delimits (one group
    without it); given as arguments (any row stride, e.g. columns of an accumulator) they are written, or added to if
    `accumulate`, otherwise they are made here.  Without dropout, and with h of dy's dtype, dx and dresidual are the
    same tensor."""
    code = _type(dy, "dy")
    rows, cols, ld = _rows(dy, "dy")
    ldh = _like(h, dy, "h", (dy.dtype, torch.float32))
    _vector(weight, cols, dy, "weight")
    _vector(mean, rows, dy, "mean")
    _vector(rstd, rows, dy, "rstd")
    ld_dh = _like(dh, dy, "dh", (h.dtype,)) if dh is not None else 0
    drop = _dropout_params(p, seed, subsequence) if p else None
    groups = _offsets(offsets, dy) if offsets is not None else 1
    if accumulate and dweight is None and dbias is None:
        raise ValueError("accumulate needs dweight or dbias to add to")
    if dweight is None and dbias is None:
        dweight, dbias = torch.empty((2, groups, cols), dtype=torch.float32, device=dy.device)
    ld_dw = _gradient_rows(dweight, groups, cols, dy, "dweight")
    ld_db = _gradient_rows(dbias, groups, cols, dy, "dbias")
    dx = torch.empty(dy.shape, dtype=dy.dtype, device=dy.device)
    same = drop is None and h.dtype == dy.dtype
    dres = dx if same else torch.empty(dy.shape, dtype=h.dtype, device=dy.device)
    L = load_library()
    nbytes = L.regtopk_layer_norm_backward_workspace_bytes(rows, cols, groups)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dy.device)
    with _on(dy) as on:
        _check(L.regtopk_layer_norm_backward(
            dy.data_ptr(), ld, h.data_ptr(), ldh, mean.data_ptr(), rstd.data_ptr(), weight.data_ptr(),
            dh.data_ptr() if dh is not None else None, ld_dh, dx.data_ptr(), cols, None if same else dres.data_ptr(), cols,
            dweight.data_ptr() if dweight is not None else None, ld_dw, dbias.data_ptr() if dbias is not None else None, ld_db,
            offsets.data_ptr() if offsets is not None else None, groups, int(accumulate), rows, cols, code, TYPES[h.dtype],
            drop, ws.data_ptr(), nbytes, on.stream), "regtopk_layer_norm_backward")
    return dx, dres, dweight, dbias


def _short(t: torch.Tensor, name: str) -> int:
    code = _type(t, name)
    if code == 0:
        raise TypeError(f"{name} is bfloat16 or float16")
    if t.dim() != 2:
        raise ValueError(f"{name} is a matrix")
    return code


def grouped_matmul(x: torch.Tensor, w: torch.Tensor, offsets: torch.Tensor, out: Optional[torch.Tensor] = None) -> torch.Tensor:
    """y [rows, m] with y[t] = w[g % E] @ x[t] for the rows t of group g; rows of no group become zeros.

    x [rows, k] and w [E, m, k] are both bfloat16 or both float16; either of w's last two dimensions may be the
    contiguous one, so w.transpose(1, 2) of a layer's weights gives the gradient to its tokens.  The number of groups
    is a multiple of E: groups sorted by (worker, expert) use the experts' matrices in turn."""
    code = _short(x, "x")
    rows, k, ldx = _rows(x, "x")
    groups = _offsets(offsets, x)
    if w.device != x.device or w.dtype != x.dtype or w.dim() != 3 or w.shape[2] != k:
        raise TypeError(f"w must be [experts, m, {k}] of x's dtype on x's device")
    count, m = w.shape[0], w.shape[1]
    if count < 1 or groups % count:
        raise ValueError("the number of groups must be a multiple of the number of matrices")
    stride, by_row, by_col = w.stride()
    if by_col == 1 or k <= 1:
        transposed, ldw, short = 0, by_row if m > 1 else k, k
    elif by_row == 1 or m <= 1:
        transposed, ldw, short = 1, by_col, m
    else:
        raise ValueError("w: one of its last two dimensions must be contiguous")
    if ldw < short:
        raise ValueError("w: rows overlap")
    if out is None:
        out = torch.empty((rows, m), dtype=x.dtype, device=x.device)
    elif out.device != x.device or out.dtype != x.dtype or out.shape != (rows, m):
        raise TypeError(f"out must be [{rows}, {m}] of x's dtype on x's device")
    ldy = _rows(out, "out")[2]
    L = load_library()
    px, pw = x.data_ptr(), w.data_ptr()
    nbytes = L.regtopk_grouped_matmul_workspace_bytes(px, ldx, pw, ldw, stride, transposed, count, rows, k, m)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=x.device) if nbytes else None
    with _on(x) as on:
        _check(L.regtopk_grouped_matmul(px, ldx, pw, ldw, stride, transposed, count, out.data_ptr(), ldy, offsets.data_ptr(), groups,
                                        rows, k, m, code, ws.data_ptr() if nbytes else None, nbytes, on.stream), "regtopk_grouped_matmul")
    return out


def grouped_matmul_dw(dy: torch.Tensor, x: torch.Tensor, offsets: torch.Tensor, out: Optional[torch.Tensor] = None,
                      accumulate: bool = False) -> torch.Tensor:
    """The gradient of grouped_matmul to the matrices, for every group on its own: out[g] = sum of dy[t] x[t]^T over
    the rows t of group g, float32 [groups, m, k].

    out may be given, as [groups, m, k] or [workers, experts, m, k] with any strides but contiguous rows (a view of an
    accumulator's columns, say), and is added to if `accumulate`."""
    code = _short(dy, "dy")
    rows, m, ld_dy = _rows(dy, "dy")
    groups = _offsets(offsets, dy)
    if x.device != dy.device or x.dtype != dy.dtype or x.dim() != 2 or x.shape[0] != rows:
        raise TypeError(f"x must be [{rows}, k] of dy's dtype on dy's device")
    _, k, ldx = _rows(x, "x")
    if out is None:
        if accumulate:
            raise ValueError("accumulate needs an out to add to")
        out = torch.empty((groups, m, k), dtype=torch.float32, device=dy.device)
    shape = out.shape
    if out.device != dy.device or out.dtype != torch.float32 or len(shape) not in (3, 4) or shape[-2:] != (m, k) \
            or shape[:-2].numel() != groups:
        raise TypeError(f"out must be float32 [{groups}, {m}, {k}] or [workers, experts, {m}, {k}] on dy's device")
    strides = out.stride()
    ld_out = strides[-2] if m > 1 else k
    if (k > 1 and strides[-1] != 1) or ld_out < k:
        raise ValueError("out: the elements of a row must be contiguous and rows must not overlap")
    if len(shape) == 3:
        inner, inner_stride, outer_stride = groups, strides[0], 0
    else:
        inner, inner_stride, outer_stride = shape[1], strides[1], strides[0]
    L = load_library()
    pdy, px = dy.data_ptr(), x.data_ptr()
    nbytes = L.regtopk_grouped_matmul_dw_workspace_bytes(pdy, ld_dy, px, ldx, groups, rows, k, m)
    ws = torch.empty(nbytes, dtype=torch.uint8, device=dy.device) if nbytes else None
    with _on(dy) as on:
        _check(L.regtopk_grouped_matmul_dw(pdy, ld_dy, px, ldx, out.data_ptr(), ld_out, inner_stride, outer_stride, inner, int(accumulate),
                                           offsets.data_ptr(), groups, rows, k, m, code, ws.data_ptr() if nbytes else None, nbytes,
                                           on.stream), "regtopk_grouped_matmul_dw")
    return out


def training_status(device=None):
    """Synchronises the device's current stream; raises if a product's kernel there ever gave up waiting (a bug)."""
    with torch.cuda.device(device):
        _check(load_library().regtopk_train_status(torch.cuda.current_stream().cuda_stream), "regtopk_train_status")
