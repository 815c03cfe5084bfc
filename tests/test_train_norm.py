"""Dropout and layer norm with their gradients, against the definitions in 64 bits.

Tolerances.  Dropout is one product in binary32 and one rounding: bit for bit.  For the norm let u = 2^-24.  A value of
h is off by at most 2u times the magnitudes that enter it (|x| / (1 - p) + |residual|; they may cancel), a sum over a row,
taken as a tree of at most 8*4 + 5 + 16 steps, by at most 53u times the sum of magnitudes, and every further step adds u
relative to what it handles; 2^-17 = 128u covers the chain, applied to the magnitudes that enter (their largest in the row
times rstd, which is what cancels when the mean is large).  Weight
gradients are sums of at most 256 steps in a row at the sizes here: 2^-16 of the sum of magnitudes."""
import os
import re

import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import train_reference as ref

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
SLACK = 2.0 ** -17


# ---- without a GPU -----------------------------------------------------------------------------------------------------
def test_philox_known_answers():
    """Known answers that its authors publish for Philox4x32-10."""
    for counter, key, want in [
            ((0, 0, 0, 0), (0, 0), (0x6627E8D5, 0xE169C58D, 0xBC57AC4C, 0x9B00DBD8)),
            ((0xFFFFFFFF,) * 4, (0xFFFFFFFF,) * 2, (0x408F276D, 0x41C83B0E, 0xA20BC7C6, 0x6D5451FD)),
            ((0x243F6A88, 0x85A308D3, 0x13198A2E, 0x03707344), (0xA4093822, 0x299F31D0),
             (0xD16CFE09, 0x94FDCCEB, 0x5001E420, 0x24126EA1))]:
        assert tuple(int(w) for w in ref.philox(counter, key)) == want


def test_reference_gradient_against_differences():
    """The formula of the backward pass against central differences of the forward formula, both in 64 bits."""
    rng = np.random.default_rng(3)
    rows, cols = 5, 13
    x, r = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))
    w, b = rng.standard_normal(cols), rng.standard_normal(cols)
    dy, dh = rng.standard_normal((rows, cols)), rng.standard_normal((rows, cols))
    args = (1e-5, 0.3, 11, 5)

    def loss(x, r, w, b):
        y, h, _, _ = ref.layer_norm(x, r, w, b, *args)
        return (y * dy).sum() + (h * dh).sum()

    _, h, mean, rstd = ref.layer_norm(x, r, w, b, *args)
    dx, dr, dw, db = ref.layer_norm_backward(dy, h, mean, rstd, w, dh, *args[1:], [0, rows])
    for grad, k in ((dx, 0), (dr, 1), (dw[0], 2), (db[0], 3)):
        v = rng.standard_normal(grad.shape)
        ends = []
        for s in (1e-5, -1e-5):
            at = [x, r, w, b]
            at[k] = at[k] + s * v
            ends.append(loss(*at))
        assert abs((ends[0] - ends[1]) / 2e-5 - (grad * v).sum()) < 1e-7 * np.abs(grad * v).sum()


@pytest.fixture(scope="module")
def lib():
    return ref.c_library()


def test_exports(lib):
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    header = open(os.path.join(root, "include", "regtopk_train.h")).read()
    declared = set(re.findall(r"^(?:int|size_t) (regtopk_[a-z_]+)\(", header, re.M))
    assert len(declared) == 9
    for name in declared:
        assert hasattr(lib, name)


def test_c_entries_refuse(lib):
    """Bad arguments come back as codes before anything is launched (the pointers here are never followed)."""
    drop = ref.DropoutParams(0.1, 1, 2)
    p = 4096  # an aligned address
    assert lib.regtopk_dropout(p, 8, p, 8, 4, 8, 3, drop, None) == -1  # type
    assert lib.regtopk_dropout(p, 8, p, 8, 4, 8, 0, None, None) == -1
    assert lib.regtopk_dropout(None, 8, p, 8, 4, 8, 0, drop, None) == -1
    assert lib.regtopk_dropout(p, 7, p, 8, 4, 8, 0, drop, None) == -1  # rows overlap
    assert lib.regtopk_dropout(p + 2, 8, p, 8, 4, 8, 0, drop, None) == -1  # a float's address
    assert lib.regtopk_dropout(p, 8, p, 8, -1, 8, 0, drop, None) == -1
    for bad in (-0.1, 1.1, float("nan")):
        assert lib.regtopk_dropout(p, 8, p, 8, 4, 8, 0, ref.DropoutParams(bad, 0, 0), None) == -1
    assert lib.regtopk_dropout(None, 0, None, 0, 0, 8, 0, drop, None) == 0  # nothing to do

    def norm(cols=8, type=0, stream=0, eps=1e-5, weight=p, y=p):
        return lib.regtopk_layer_norm(p, cols, None, 0, weight, None, eps, y, cols, None, 0, p, p, 4, cols, type, stream, None, None)
    assert norm(cols=0) == -1 and norm(cols=16385) == -7 and norm(type=5) == -1 and norm(type=1, stream=2) == -1
    assert norm(eps=-1.0) == -1 and norm(eps=float("nan")) == -1 and norm(weight=None) == -1 and norm(y=None) == -1

    def back(groups=1, offsets=None, ws=p, nbytes=1 << 30, dw=p, ld=8, cols=8):
        return lib.regtopk_layer_norm_backward(p, 8, p, 8, p, p, p, None, 0, p, 8, None, 0, dw, ld, None, 0, offsets, groups, 0,
                                               4, cols, 0, 0, None, ws, nbytes, None)
    assert back(groups=0) == -1 and back(groups=2) == -1 and back(offsets=p + 4) == -1 and back(ws=None) == -1
    assert back(nbytes=8) == -2 and back(groups=2, offsets=p, ld=7) == -1 and back(cols=20000) == -7
    assert lib.regtopk_layer_norm_backward_workspace_bytes(4, 8, 0) == 0
    assert lib.regtopk_layer_norm_backward_workspace_bytes(4, 20000, 1) == 0


def test_no_cpu_path(lib):
    x = torch.zeros(4, 8)
    with pytest.raises(TypeError):
        rt.dropout(x, 0.1, 0)
    with pytest.raises(TypeError):
        rt.layer_norm(x, torch.ones(8))


# ---- on the GPU ----------------------------------------------------------------------------------------------------------
def made(rows, cols, dtype, gen, pad=0, shift=0, scale=1.0):
    """A [rows, cols] tensor with `pad` unused columns between rows, beginning `shift` elements into its storage."""
    flat = torch.zeros(rows * (cols + pad) + shift, dtype=dtype, device="cuda")
    t = flat[shift:].view(rows, cols + pad)[:, :cols]
    t.copy_((scale * torch.randn(rows, cols, generator=gen)).to(dtype))
    return t


SIZES = [(1, 1), (1, 8), (3, 7), (5, 256), (17, 257), (64, 768), (9, 1000), (33, 1023), (7, 1025), (4, 2048), (3, 3001),
         (2, 8192), (2, 16384), (3, 16383), (130, 512)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("rows,cols", SIZES + [(2, 40000), (700, 24), (0, 16), (4, 0)])
def test_dropout(rows, cols, dtype):
    gen = torch.Generator().manual_seed(rows * 31 + cols)
    for p, pad, shift, seed in ((0.1, 0, 0, 0), (0.5, 8, 8, 2**64 - 1), (0.3, 3, 1, 12345678901234567)):
        x = made(rows, cols, dtype, gen, pad, shift)
        if x.numel():
            x[0, 0] = float("inf")
            x[-1, -1] = float("nan")
        keep, factor = ref.keep_mask(rows, cols, p, seed, 77)
        want = torch.where(torch.from_numpy(keep), x.cpu().float() * torch.tensor(factor, dtype=torch.float32), 0.0).to(dtype)
        got = rt.dropout(x, p, seed, 77)
        assert got.dtype == dtype and torch.equal(got.cpu().float().nan_to_num(nan=7e4), want.float().nan_to_num(nan=7e4))
        before = x.clone()
        assert rt.dropout(x, p, seed, 77, out=x) is x
        assert torch.equal(x.float().nan_to_num(nan=7e4), got.float().nan_to_num(nan=7e4)), "in place"
        if x.numel() > 1000:
            assert not torch.equal(rt.dropout(before, p, seed, 78).float(), got.float())
            assert abs(keep.mean() - (1 - p)) < 6 * (p * (1 - p) / keep.size) ** 0.5


@pytest.mark.gpu
def test_dropout_limits_and_shapes():
    x = torch.randn(3, 5, 24, device="cuda")
    assert torch.equal(rt.dropout(x, 0.0, 1), x)
    x[0, 0, 0] = float("nan")
    assert torch.equal(rt.dropout(x, 1.0, 1), torch.zeros_like(x))
    a, b = rt.dropout(x, 0.4, 9, 2), rt.dropout(x.view(15, 24), 0.4, 9, 2)
    assert torch.equal(a.view(15, 24).nan_to_num(), b.nan_to_num())
    assert rt.dropout(torch.ones(7, device="cuda"), 0.0, 0).shape == (7,)


@pytest.mark.gpu
def test_dropout_rows_past_32_bits():
    """Offsets past 2^31 elements: the last rows of a 16-bit array of 2^31 + 2^20 elements."""
    cols = 1 << 20
    rows = (1 << 11) + 1
    x = torch.ones(rows, cols, dtype=BF, device="cuda")
    rt.dropout(x, 0.25, 5, 6, out=x)
    keep, factor = ref.keep_mask(rows, 64, 0.25, 5, 6)
    want = torch.where(torch.from_numpy(keep), torch.tensor(factor), 0.0).to(BF).float()
    assert torch.equal(x[:, :64].cpu().float(), want)


TYPES = [(BF, BF), (BF, F), (HF, HF), (HF, F), (F, F)]


def norm_case(rows, cols, dtype, stream, seed, pad=0, shift=0):
    gen = torch.Generator().manual_seed(seed)
    x = made(rows, cols, dtype, gen, pad, shift)
    residual = made(rows, cols, stream, gen, pad, shift, scale=2.0)
    flat = torch.randn(2 * cols + 1, generator=gen).cuda()
    return x, residual, flat[1: 1 + cols], flat[1 + cols:], gen  # vectors at an odd place of a flat array


def check_norm(x, residual, weight, bias, p, seed, eps=1e-5):
    y, h, mean, rstd = rt.layer_norm(x, weight, bias, eps, residual=residual, p=p, seed=seed, subsequence=3)
    wy, wh, wm, wr = ref.layer_norm(ref.host(x), None if residual is None else ref.host(residual), ref.host(weight),
                                    None if bias is None else ref.host(bias), eps, p, seed, 3)
    enter = np.abs(ref.dropped(ref.host(x), p, seed, 3)) + (0 if residual is None else np.abs(ref.host(residual)))
    enter = np.where(np.isfinite(enter), enter, 0.0)
    top = enter.max(1)
    ref.assert_close(mean, wm, SLACK * top, F, "mean")
    ref.assert_close(rstd, wr, SLACK * wr * (1 + (top * wr) ** 2), F, "rstd")
    unit = np.abs(wh - wm[:, None]) * wr[:, None]
    slack = SLACK * ((top * wr)[:, None] * (1 + unit) * (1 + (top * wr)[:, None]) * np.abs(ref.host(weight)) + (0 if bias is None else np.abs(ref.host(bias))))
    ref.assert_close(y, wy, slack, x.dtype, "y")
    if residual is not None or p:
        ref.assert_close(h, wh, 2 * ref.U * enter, h.dtype, "h")
    else:
        assert h is x
    return y, h, mean, rstd


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_layer_norm(rows, cols, dtype, stream):
    for p, pad, shift in ((0.1, 0, 0), (0.0, 8, 8), (0.5, 5, 1)):
        x, residual, weight, bias, _ = norm_case(rows, cols, dtype, stream, rows + cols, pad, shift)
        check_norm(x, residual, weight, bias, p, 99)
        if stream == dtype:
            check_norm(x, None, weight, None, p, 99)


@pytest.mark.gpu
def test_layer_norm_rows_that_strain_it():
    """Constant rows (variance zero), a large mean beside a small deviation, large and tiny values, many rows."""
    weight, bias = torch.ones(1000, device="cuda"), torch.zeros(1000, device="cuda")
    x = torch.randn(6, 1000, generator=torch.Generator().manual_seed(1)).cuda()
    x[0] = 0.0
    x[1] = 1000.0
    x[2] += 1000.0
    x[3] *= 1e15
    x[4] *= 1e-12
    y, _, mean, rstd = check_norm(x, None, weight, bias, 0.0, 0)
    assert torch.equal(y[0], bias) and mean[1] == 1000.0
    x[5, 3] = float("nan")
    x[4, 7] = float("inf")
    y, _, _, _ = rt.layer_norm(x, weight, bias)
    assert torch.isnan(y[4:]).all() and torch.isfinite(y[:4]).all()
    many = torch.randn(5003, 96, generator=torch.Generator().manual_seed(2)).cuda()
    check_norm(many, None, weight[:96], bias[:96], 0.0, 0)


@pytest.mark.gpu
def test_layer_norm_shapes():
    x = torch.randn(2, 3, 40, device="cuda")
    w = torch.ones(40, device="cuda")
    y, h, mean, rstd = rt.layer_norm(x, w)
    assert y.shape == x.shape and mean.shape == (2, 3) and rstd.shape == (2, 3) and h is x
    y1, _, m1, _ = rt.layer_norm(x[0, 0], w)
    assert torch.equal(y1, y[0, 0]) and torch.equal(m1, mean[0, 0])
    y0, _, m0, _ = rt.layer_norm(x[:0], w)
    assert y0.shape == (0, 3, 40) and m0.shape == (0, 3)
    dx, _, dw, db = rt.layer_norm_backward(x[:0], x[:0], m0, m0, w)
    assert dx.shape == (0, 3, 40) and not dw.any() and not db.any()


def check_back(dy, h, mean, rstd, weight, dh, p, offsets, **kw):
    at = [0, len(dy)] if offsets is None else offsets
    dev = None if offsets is None else torch.tensor(offsets, device="cuda")
    dx, dres, dw, db = rt.layer_norm_backward(dy, h, mean, rstd, weight, dh=dh, p=p, seed=4, subsequence=9, offsets=dev, **kw)
    d = [ref.host(t) for t in (dy, h, mean, rstd, weight)]
    wx, wr, ww, wb = ref.layer_norm_backward(*d, None if dh is None else ref.host(dh), p, 4, 9, at)
    dyn, hn, mn, rn, wn = d
    g, size = np.abs(dyn * wn), (np.abs(hn) + np.abs(mn)[:, None]) * rn[:, None]  # what enters u before it cancels
    slack = SLACK * (rn[:, None] * (g + g.mean(1)[:, None] + size * (g * size).mean(1)[:, None])
                     + (0 if dh is None else np.abs(ref.host(dh))))
    factor = 65536.0 / (65536 - round(65536 * p))
    ref.assert_close(dx, wx, factor * slack, dy.dtype, "dx")
    ref.assert_close(dres, wr, slack, h.dtype, "dresidual")
    sums = [2.0 ** -16 * np.stack([v[a:b].sum(0) for a, b in zip(at, at[1:])]) for v in (np.abs(dyn) * size, np.abs(dyn))]
    return (dx, dres, dw, db), (ww, wb), sums


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_layer_norm_backward(rows, cols, dtype, stream):
    for p, pad, shift, with_dh in ((0.1, 0, 0, True), (0.0, 8, 8, False), (0.5, 5, 1, True)):
        x, residual, weight, bias, gen = norm_case(rows, cols, dtype, stream, rows + cols, pad, shift)
        _, h, mean, rstd = rt.layer_norm(x, weight, bias, residual=residual, p=p, seed=4, subsequence=9)
        dy, dh = made(rows, cols, dtype, gen, pad, shift), made(rows, cols, stream, gen, pad, shift)
        cut = sorted(int(i) for i in torch.randint(0, rows + 1, (3,), generator=gen))
        for offsets in (None, [0, *cut, rows], [0, 0, rows, rows]):
            (dx, dres, dw, db), want, slack = check_back(dy, h, mean, rstd, weight, dh if with_dh else None, p, offsets)
            assert (dx is dres) == (p == 0 and dtype == stream)
            for got, w, s, name in zip((dw, db), want, slack, ("dweight", "dbias")):
                ref.assert_close(got, w, s, F, name)


@pytest.mark.gpu
def test_layer_norm_backward_groups():
    """More groups than blocks, rows of no group before, between and after, sums over many rows, equal bits twice."""
    gen = torch.Generator().manual_seed(8)
    rows, cols = 6001, 136
    h, dy = made(rows, cols, BF, gen), made(rows, cols, BF, gen)
    w = torch.randn(cols, generator=gen).cuda()
    _, _, mean, rstd = rt.layer_norm(h, w)
    many = torch.sort(torch.randint(0, rows + 1, (1500,), generator=gen)).values.tolist()
    for offsets in ([0, rows], [5, 700, 700, 5990], many, [rows, rows], [0, 0]):
        out, want, slack = check_back(dy, h, mean, rstd, w, None, 0.0, offsets)
        for got, v, s, name in zip(out[2:], want, slack, ("dweight", "dbias")):
            ref.assert_close(got, v, s, F, name)
        again, _, _ = check_back(dy, h, mean, rstd, w, None, 0.0, offsets)
        assert all(torch.equal(a, b) for a, b in zip(out, again))


@pytest.mark.gpu
def test_layer_norm_backward_into_rows():
    """Gradients written and added into columns of wider rows, with one rounded addition per element; offsets that are
    out of range or descend touch nothing outside."""
    gen = torch.Generator().manual_seed(2)
    rows, cols, n = 90, 50, 3
    h, dy = made(rows, cols, F, gen), made(rows, cols, F, gen)
    w = torch.randn(cols, generator=gen).cuda()
    _, _, mean, rstd = rt.layer_norm(h, w)
    offsets = torch.tensor([0, 31, 31, 90], device="cuda")
    flat = torch.randn(n, 2 * cols + 7, generator=gen).cuda()
    before = flat.clone()
    dw, db = flat[:, 3: 3 + cols], flat[:, 5 + cols: 5 + 2 * cols]
    _, _, fw, fb = rt.layer_norm_backward(dy, h, mean, rstd, w, offsets=offsets)
    out = rt.layer_norm_backward(dy, h, mean, rstd, w, offsets=offsets, dweight=dw, dbias=db, accumulate=True)
    assert out[2] is dw and out[3] is db
    want = before.clone()
    want[:, 3: 3 + cols] += fw
    want[:, 5 + cols: 5 + 2 * cols] += fb
    assert torch.equal(flat, want)
    rt.layer_norm_backward(dy, h, mean, rstd, w, offsets=offsets, dbias=db)
    want[:, 5 + cols: 5 + 2 * cols] = fb
    assert torch.equal(flat, want), "dbias alone, written"
    for bad in ([-5, 31, 1000, 2**40], [90, 31, 10, 0], [2**62, -2**62, 2**62, 0]):
        edge = flat.clone()
        rt.layer_norm_backward(dy, h, mean, rstd, w, offsets=torch.tensor(bad, device="cuda"), dweight=edge[:, 3: 3 + cols])
        torch.cuda.synchronize()
        keep = torch.ones(2 * cols + 7, dtype=torch.bool, device="cuda")
        keep[3: 3 + cols] = False
        assert torch.equal(edge[:, keep], flat[:, keep])


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [96, 101])
def test_layer_norm_gradient_against_differences(cols):
    """The library's gradients against central differences of the library's forward pass, binary32.  With steps of 2^-7
    of the values' size the truncation is of order 2^-14 and the rounding 2^-24 * 2^7 of the sum of magnitudes."""
    gen = torch.Generator().manual_seed(cols)
    rows = 7
    x, r, dy, dh = (torch.randn(rows, cols, generator=gen).cuda() for _ in range(4))
    w, b = (torch.randn(cols, generator=gen).cuda() for _ in range(2))
    kw = dict(p=0.2, seed=3, subsequence=1)

    def loss(x, r, w, b):
        y, h, _, _ = rt.layer_norm(x, w, b, residual=r, **kw)
        return float((y.double() * dy.double()).sum() + (h.double() * dh.double()).sum())

    _, h, mean, rstd = rt.layer_norm(x, w, b, residual=r, **kw)
    dx, dr, dw, db = rt.layer_norm_backward(dy, h, mean, rstd, w, dh=dh, **kw)
    for k, grad in enumerate((dx, dr, dw[0], db[0])):
        v = torch.randn(grad.shape, generator=gen).cuda()
        ends = []
        for s in (2.0 ** -7, -2.0 ** -7):
            at = [x, r, w, b]
            at[k] = at[k] + s * v
            ends.append(loss(*at))
        got, want = (ends[0] - ends[1]) * 2.0 ** 6, float((grad.double() * v.double()).sum())
        assert abs(got - want) < 2.0 ** -9 * float((grad.double() * v.double()).abs().sum()), k


@pytest.mark.gpu
def test_other_streams():
    """On a stream that is not the default, ordered behind the work that makes the inputs there."""
    side = torch.cuda.Stream()
    x0 = torch.randn(4000, 768, device="cuda")
    w = torch.ones(768, device="cuda")
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        x = x0
        for _ in range(20):
            x = x * 1.01
        y, h, mean, rstd = rt.layer_norm(rt.dropout(x, 0.1, 1), w)
        dx, _, dw, _ = rt.layer_norm_backward(y, h, mean, rstd, w)
    torch.cuda.synchronize()
    y2, h2, m2, r2 = rt.layer_norm(rt.dropout(x, 0.1, 1), w)
    d2, _, dw2, _ = rt.layer_norm_backward(y2, h2, m2, r2, w)
    assert torch.equal(y, y2) and torch.equal(dx, d2) and torch.equal(dw, dw2)


@pytest.mark.gpu
def test_refusals():
    x = torch.randn(4, 16, device="cuda")
    w = torch.ones(16, device="cuda")
    _, _, mean, rstd = rt.layer_norm(x, w)
    for call, error in [
            (lambda: rt.dropout(x.double(), 0.1, 0), TypeError), (lambda: rt.dropout(x.t(), 0.1, 0), ValueError),
            (lambda: rt.dropout(x, 1.5, 0), ValueError), (lambda: rt.dropout(x, 0.5, -1), ValueError),
            (lambda: rt.dropout(x, 0.5, 0, 1 << 32), ValueError), (lambda: rt.dropout(x, 0.5, 0, out=x[:2]), TypeError),
            (lambda: rt.dropout(x, 0.5, 0, out=x.half()), TypeError), (lambda: rt.dropout(x[0, 0], 0.5, 0), ValueError),
            (lambda: rt.dropout(x[:1].expand(4, 16), 0.5, 0), ValueError),
            (lambda: rt.layer_norm(x, w.half()), TypeError), (lambda: rt.layer_norm(x, w[:8]), TypeError),
            (lambda: rt.layer_norm(x, torch.ones(32, device="cuda")[::2]), TypeError),
            (lambda: rt.layer_norm(x, w, w.cpu()), TypeError), (lambda: rt.layer_norm(x, w, residual=x.half()), TypeError),
            (lambda: rt.layer_norm(x.half(), w, residual=x.bfloat16()), TypeError),
            (lambda: rt.layer_norm(x, w, eps=-1.0), rt.RegTopKError),
            (lambda: rt.layer_norm(torch.zeros(2, 16385, device="cuda"), torch.ones(16385, device="cuda")), rt.RegTopKError),
            (lambda: rt.layer_norm(x, w, p=-0.5), ValueError),
            (lambda: rt.layer_norm_backward(x, x[:2], mean, rstd, w), TypeError),
            (lambda: rt.layer_norm_backward(x, x, mean[:2], rstd, w), TypeError),
            (lambda: rt.layer_norm_backward(x, x, mean, rstd, w, dh=x.half()), TypeError),
            (lambda: rt.layer_norm_backward(x, x, mean, rstd, w, offsets=torch.tensor([0, 4], device="cuda", dtype=torch.int32)), TypeError),
            (lambda: rt.layer_norm_backward(x, x, mean, rstd, w, offsets=torch.tensor([0, 4])), TypeError),
            (lambda: rt.layer_norm_backward(x, x, mean, rstd, w, offsets=torch.tensor([0], device="cuda")), TypeError),
            (lambda: rt.layer_norm_backward(x, x, mean, rstd, w, dweight=torch.zeros(2, 16, device="cuda")), TypeError),
            (lambda: rt.layer_norm_backward(x, x, mean, rstd, w, accumulate=True), ValueError)]:
        with pytest.raises(error):
            call()
