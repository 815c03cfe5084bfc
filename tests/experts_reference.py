"""The operators around an expert sublayer from their definitions, in 64 bits on the host (numpy), for the tests of the CUDA kernels."""
import ctypes
import math
import os

import numpy as np
import torch

# ---- 8-bit rows: by a table of the numbers ----------------------------------------------------------------------------
E4M3 = np.array([(c >> 3 and 2.0 ** ((c >> 3) - 7) * (1 + (c & 7) / 8)) or 2.0 ** -6 * (c & 7) / 8 for c in range(127)])  # codes 0 to 0x7E


def nearest_e4m3(x):
    """The number nearest to each finite x, |x| <= 448; halfway cases to the even code."""
    m = np.abs(x)
    hi = np.clip(np.searchsorted(E4M3, m), 0, 126)
    lo = np.maximum(hi - 1, 0)
    below, above = m - E4M3[lo], E4M3[hi] - m
    code = np.where((below < above) | ((below == above) & (lo % 2 == 0)), lo, hi)
    return np.copysign(E4M3[code], x)


def scale_bytes(x):
    """[rows, cols] to [rows, blocks]: the smallest byte with which no finite value passes 448 times the scale."""
    rows, cols = x.shape
    blocks = (cols + 31) // 32
    m = np.zeros((rows, blocks * 32))
    m[:, :cols] = np.where(np.isfinite(x), np.abs(x), 0.0)
    m = m.reshape(rows, blocks, 32).max(-1)
    byte = np.zeros((rows, blocks), np.int64)
    for b in range(255):
        byte += m > 448 * 2.0 ** (b - 127)
    return byte


def packed(x, halves=1):
    """(values that the 8-bit rows of x stand for, their scale bytes)."""
    if halves == 2:
        h = x.shape[1] // 2
        (a, p), (b, q) = packed(x[:, :h]), packed(x[:, h:])
        return np.concatenate([a, b], 1), np.concatenate([p, q], 1)
    byte = scale_bytes(x)
    scale = 2.0 ** (np.repeat(byte, 32, 1)[:, :x.shape[1]] - 127.0)
    fine = np.isfinite(x)
    return np.where(fine, nearest_e4m3(np.where(fine, x, 0.0) / scale) * scale, np.nan), byte


def unpacked(rows8, halves=1):
    """What a Rows8 of the device holds, in float64."""
    v = rows8.values.detach().cpu().float().double().numpy()
    b = rows8.scales.detach().cpu().view(torch.uint8).numpy().astype(np.int64)
    v, b = v.reshape(-1, v.shape[-1] // halves), b.reshape(-1, b.shape[-1] // halves)
    scale = np.where(b == 255, np.nan, 2.0 ** (b - 127.0))
    return (v * np.repeat(scale, 32, 1)[:, :v.shape[1]]).reshape(rows8.values.shape)


# ---- the router -------------------------------------------------------------------------------------------------------
def scores_of(l, kind):
    """[tokens, experts]; a NaN or +inf among the logits makes the token's softmax NaN."""
    with np.errstate(all="ignore"):
        if kind == "sigmoid":
            return np.where(l >= 0, 1 / (1 + np.exp(-np.abs(l))), np.exp(-np.abs(l)) / (1 + np.exp(-np.abs(l))))
        m = np.where(np.isnan(l), -np.inf, l).max(1, keepdims=True)
        e = np.where(l == -np.inf, 0.0, np.exp(l - m))
        return np.where(l == -np.inf, 0.0, e / e.sum(1, keepdims=True))


def route(l, k, kind, bias, groups, kept, top, renormalise, scale):
    """Token by token: (experts, weights)."""
    s = scores_of(l, kind)
    experts, weights = np.full((len(l), k), -1), np.zeros((len(l), k))
    for t in range(len(l)):
        with np.errstate(all="ignore"):
            c = s[t] + bias if bias is not None else s[t].copy()
        order = c if bias is not None else l[t]  # without bias the logits' order, which is the scores' before rounding
        there = (l[t] != -np.inf) & (c != -np.inf)
        judged = np.where(np.isnan(c if bias is not None or top == 2 else l[t]), -1e300, c if bias is not None or top == 2 else l[t])
        order = np.where(np.isnan(order), -1e300, order)
        strength = []
        for g in range(groups):
            own = judged.reshape(groups, -1)[g][there.reshape(groups, -1)[g]]
            strength.append(np.sort(own)[::-1][:top].sum() if len(own) else -np.inf)
        best = sorted(range(groups), key=lambda g: (-strength[g], g))[:kept]
        size = l.shape[1] // groups
        may = [e for e in range(l.shape[1]) if there[e] and e // size in best]
        may.sort(key=lambda e: (-order[e], e))
        experts[t, :len(may[:k])] = may[:k]
    return experts, route_weights(l, experts, kind, renormalise, scale)


def route_weights(l, experts, kind, renormalise, scale):
    s, there = scores_of(l, kind), experts >= 0
    at = np.where(there, experts, 0)
    w = np.where(there, np.take_along_axis(s, at, 1), 0.0)
    if renormalise:  # relative to the largest logit, so that scores that are all too small for binary64 count too
        own = np.where(there, np.take_along_axis(l, at, 1), -np.inf)
        with np.errstate(all="ignore"):
            top = own.max(1, keepdims=True)
            if kind == "softmax":
                v = np.where(there, np.exp(own - top), 0.0)
            else:
                top = np.minimum(top, 0.0)
                v = np.where(there, np.where(own < 0, np.exp(own - top) / (1 + np.exp(own)), 1 / (1 + np.exp(-own))), 0.0)
            v = np.where(np.isnan(w), np.nan, v)
            total = v.sum(1, keepdims=True)
            w = np.where(there, v / np.where(total == 0, 1.0, total), 0.0)
    return w * scale


def route_backward(dw, l, experts, kind, renormalise, scale):
    """By the chain rule through the scores, every pair on its own (the same expert twice counts twice)."""
    s, out = scores_of(l, kind), np.zeros(l.shape)
    for t in range(len(l)):
        js = [j for j in range(experts.shape[1]) if 0 <= experts[t, j] < l.shape[1]]
        es = [experts[t, j] for j in js]
        g = np.array([dw[t, j] for j in js]) * scale
        if renormalise and js:
            p = route_weights(l[t:t + 1], np.array([es]), kind, True, 1.0)[0]
            d = p * (g - (g * p).sum())
            for e, v in zip(es, d if kind == "softmax" else d * (1 - s[t, es])):
                out[t, e] += v
        elif kind == "sigmoid":
            for e, v in zip(es, g):
                out[t, e] += v * s[t, e] * (1 - s[t, e])
        else:
            ds = np.zeros(l.shape[1])
            for e, v in zip(es, g):
                ds[e] += v
            out[t] = s[t] * (ds - (ds * s[t]).sum())
    return out


# ---- the tokens' way --------------------------------------------------------------------------------------------------
def sort_tokens(experts, n_experts, at):
    offsets, place, n = [0], np.full(experts.shape, -1), 0
    for lo, hi in zip(at, at[1:]):
        for e in range(n_experts):
            for t in range(max(lo, 0), min(hi, len(experts))):
                for j in range(experts.shape[1]):
                    if experts[t, j] == e:
                        place[t, j] = n
                        n += 1
            offsets.append(n)
    return np.array(offsets), place


def spread(x, place, rows):
    out = np.zeros((rows, x.shape[1]))
    t, j = np.nonzero(place >= 0)
    out[place[t, j]] = x[t]
    return out


def join(rows, place, weights, residual):
    w = np.where(place >= 0, 1.0 if weights is None else weights, 0.0)
    out = np.einsum("tj,tjc->tc", w, rows[np.maximum(place, 0)]) if len(rows) else np.zeros((len(place), rows.shape[1]))
    return out + (0.0 if residual is None else residual)


# ---- activations ------------------------------------------------------------------------------------------------------
def activation(a, kind, gated):
    """(y, f(x), f'(x)) with x the first half if gated."""
    h = a.shape[1] // 2 if gated else a.shape[1]
    x = a[:, :h]
    if kind == "gelu":
        p = 0.5 * torch.special.erfc(torch.from_numpy(-x * math.sqrt(0.5))).numpy()  # exact far out, where 1 + erf(x) is 0
        slope = p + x * np.exp(-x * x / 2) / math.sqrt(2 * math.pi)
    else:
        z, dz = (x, 1.0) if kind == "silu" else (2 * math.sqrt(2 / math.pi) * (x + 0.044715 * x ** 3), 2 * math.sqrt(2 / math.pi) * (1 + 3 * 0.044715 * x * x))
        p, q = torch.special.expit(torch.from_numpy(z)).numpy(), torch.special.expit(torch.from_numpy(-z)).numpy()
        slope = p + x * p * q * dz
    f = x * p
    return (f * a[:, h:] if gated else f), f, slope


def activation_backward(dy, a, kind, gated):
    y, f, slope = activation(a, kind, gated)
    h = f.shape[1]
    return (np.concatenate([dy * slope * a[:, h:], dy * f], 1) if gated else dy * slope), y


# ---- the norm ---------------------------------------------------------------------------------------------------------
def rms_norm(x, residual, weight, eps):
    h = x + (0.0 if residual is None else residual)
    rstd = 1.0 / np.sqrt((h ** 2).mean(1) + eps)
    return h * rstd[:, None] * weight, h, rstd


def rms_norm_backward(dy, h, rstd, weight, dh, offsets):
    u = h * rstd[:, None]
    g = dy * weight
    dres = rstd[:, None] * (g - u * (g * u).mean(1)[:, None]) + (0.0 if dh is None else dh)
    return dres, np.stack([(dy * u)[a:b].sum(0) for a, b in zip(offsets, offsets[1:])])


class RouteParams(ctypes.Structure):
    _fields_ = [("scores", ctypes.c_int32), ("groups", ctypes.c_int32), ("groups_kept", ctypes.c_int32), ("group_top", ctypes.c_int32),
                ("renormalise", ctypes.c_int32), ("scale", ctypes.c_float)]


def c_library():
    """The C entries with their signatures."""
    import paper_2501_05633_b200 as rt
    rt.build()
    L = ctypes.CDLL(os.path.join(os.path.dirname(rt.__file__), "libregtopk_train.so"))
    p, i64, i32, f32, size, rp = (ctypes.c_void_p, ctypes.c_int64, ctypes.c_int32, ctypes.c_float, ctypes.c_size_t, ctypes.POINTER(RouteParams))
    for name, args, res in [
            ("regtopk_pack8", [p, i64, p, i64, p, i64, i64, i64, i32, p], i32),
            ("regtopk_unpack8", [p, i64, p, i64, p, i64, i64, i64, i32, p], i32),
            ("regtopk_route", [p, i64, p, p, p, i64, i32, i32, i32, rp, p], i32),
            ("regtopk_route_backward", [p, p, i64, p, p, i64, i64, i32, i32, i32, rp, p], i32),
            ("regtopk_sort_tokens_workspace_bytes", [i64, i32, i32, i32], size),
            ("regtopk_sort_tokens", [p, p, i32, p, p, i64, i32, i32, p, size, p], i32),
            ("regtopk_spread_tokens", [p, i64, p, i64, p, p, p, i64, i64, i32, i64, i64, i32, p], i32),
            ("regtopk_join_tokens", [p, i64, p, p, p, i64, p, i64, i64, i32, i64, i64, i32, i32, p], i32),
            ("regtopk_join_tokens_backward", [p, i64, p, i64, p, p, p, p, i64, p, i64, i32, i64, i64, i32, i32, p], i32),
            ("regtopk_activation", [p, i64, p, i64, p, i64, p, i64, i64, i64, i32, i32, i32, p], i32),
            ("regtopk_activation_backward", [p, i64, p, i64, p, i64, p, i64, p, i64, i64, i64, i32, i32, i32, p], i32),
            ("regtopk_rms_norm", [p, i64, p, i64, p, f32, p, i64, p, i64, p, i64, p, i64, p, i64, i64, i32, i32, p], i32),
            ("regtopk_rms_norm_backward_workspace_bytes", [i64, i64, i32], size),
            ("regtopk_rms_norm_backward", [p, i64, p, i64, p, p, p, i64, p, i64, p, i64, p, i64, p, i32, i32, i64, i64, i32, i32, p, size, p], i32)]:
        f = getattr(L, name)
        f.argtypes, f.restype = args, res
    return L
