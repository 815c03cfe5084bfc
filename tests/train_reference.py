"""The training operators from their definitions, in 64 bits on the host (numpy), for the tests of the CUDA kernels."""
import ctypes
import os

import numpy as np
import torch

U = 2.0 ** -24  # half a unit in the last place of binary32, relative
ROUND = {torch.float32: 2.0 ** -24, torch.bfloat16: 2.0 ** -8, torch.float16: 2.0 ** -11}  # one rounding to the type
TINY = {torch.float32: 0.0, torch.bfloat16: 0.0, torch.float16: 2.0 ** -25}  # and to its smallest step


def philox(counter, key, rounds=10):
    """Philox4x32 of four uint64 arrays (or numbers) that hold 32-bit words, and a two-word key."""
    low = np.uint64(0xFFFFFFFF)
    x = [np.asarray(c, np.uint64) for c in counter]
    k0, k1 = int(key[0]), int(key[1])
    for _ in range(rounds):
        a, b = x[0] * np.uint64(0xD2511F53), x[2] * np.uint64(0xCD9E8D57)
        x = [(b >> np.uint64(32)) ^ x[1] ^ np.uint64(k0), b & low, (a >> np.uint64(32)) ^ x[3] ^ np.uint64(k1), a & low]
        k0, k1 = (k0 + 0x9E3779B9) & 0xFFFFFFFF, (k1 + 0xBB67AE85) & 0xFFFFFFFF
    return x


def keep_mask(rows, cols, p, seed, subsequence):
    """Which elements dropout keeps, and the factor by which it scales them."""
    t = int(round(65536 * p))
    groups = (cols + 7) // 8
    r, g = np.meshgrid(np.arange(rows, dtype=np.uint64), np.arange(groups, dtype=np.uint64), indexing="ij")
    words = philox([g, r & np.uint64(0xFFFFFFFF), r >> np.uint64(32), np.full_like(r, subsequence)],
                   (seed & 0xFFFFFFFF, seed >> 32))
    numbers = np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in words for s in (0, 16)], -1)
    return numbers.reshape(rows, groups * 8)[:, :cols] >= t, (65536.0 / (65536 - t) if t < 65536 else 0.0)


def host(t):
    return t.detach().double().cpu().numpy()


def dropped(x, p, seed, subsequence):
    keep, factor = keep_mask(*x.shape, p, seed, subsequence)
    return np.where(keep, x * factor, 0.0)


def layer_norm(x, residual, weight, bias, eps, p, seed, subsequence):
    h = dropped(x, p, seed, subsequence) + (0.0 if residual is None else residual)
    mean = h.mean(1)
    rstd = 1.0 / np.sqrt(((h - mean[:, None]) ** 2).mean(1) + eps)
    y = (h - mean[:, None]) * rstd[:, None] * weight + (0.0 if bias is None else bias)
    return y, h, mean, rstd


def layer_norm_backward(dy, h, mean, rstd, weight, dh, p, seed, subsequence, offsets):
    u = (h - mean[:, None]) * rstd[:, None]
    g = dy * weight
    dres = rstd[:, None] * (g - g.mean(1)[:, None] - u * (g * u).mean(1)[:, None]) + (0.0 if dh is None else dh)
    dw = np.stack([(dy * u)[a:b].sum(0) for a, b in zip(offsets, offsets[1:])])
    db = np.stack([dy[a:b].sum(0) for a, b in zip(offsets, offsets[1:])])
    return dropped(dres, p, seed, subsequence), dres, dw, db


def assert_close(got, want, slack, dtype, what):
    """|got - want| <= one rounding of `want` to the type + slack, element by element; NaN and infinities equal."""
    got = host(got).reshape(want.shape)
    fine = np.isfinite(want)
    assert np.array_equal(got[~fine], want[~fine], equal_nan=True), f"{what}: non-finite values differ"
    off = np.abs(got - np.where(fine, want, 0.0))[fine]
    most = (ROUND[dtype] * np.abs(np.where(fine, want, 0.0)) + TINY[dtype] + slack + 0 * want)[fine]
    bad = ~(off <= most)
    assert not bad.any(), f"{what}: {int(bad.sum())} of {bad.size} too far off, worst {np.nanmax(off / np.maximum(most, 1e-300)):.3g} times the tolerance"


class DropoutParams(ctypes.Structure):
    _fields_ = [("p", ctypes.c_double), ("seed", ctypes.c_uint64), ("subsequence", ctypes.c_uint32)]


def c_library():
    """The C entries of the training operators with their signatures."""
    import paper_2501_05633_b200 as rt
    rt.build()
    L = ctypes.CDLL(os.path.join(os.path.dirname(rt.__file__), "libregtopk_train.so"))
    p, i64, i32, f32, size, drop = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t,
                                    ctypes.POINTER(DropoutParams))
    for name, args, res in [
            ("regtopk_dropout", [p, i64, p, i64, i64, i64, i32, drop, p], i32),
            ("regtopk_layer_norm", [p, i64, p, i64, p, p, f32, p, i64, p, i64, p, p, i64, i64, i32, i32, drop, p], i32),
            ("regtopk_layer_norm_backward_workspace_bytes", [i64, i64, i32], size),
            ("regtopk_layer_norm_backward", [p, i64, p, i64, p, p, p, p, i64, p, i64, p, i64, p, i64, p, i64, p, i32, i32, i64, i64,
                                             i32, i32, drop, p, size, p], i32),
            ("regtopk_grouped_matmul_workspace_bytes", [p, i64, p, i64, i64, i32, i32, i32, i64, i64, i64], size),
            ("regtopk_grouped_matmul", [p, i64, p, i64, i64, i32, i32, p, i64, p, i32, i64, i64, i64, i32, p, size, p], i32),
            ("regtopk_grouped_matmul_dw_workspace_bytes", [p, i64, p, i64, i32, i64, i64, i64], size),
            ("regtopk_grouped_matmul_dw", [p, i64, p, i64, p, i64, i64, i64, i32, i32, p, i32, i64, i64, i64, i32, p, size, p], i32),
            ("regtopk_train_status", [p], i32)]:
        f = getattr(L, name)
        f.argtypes, f.restype = args, res
    return L
