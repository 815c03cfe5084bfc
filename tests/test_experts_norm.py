"""The root-mean-square norm and its gradient, against the definitions in 64 bits.

Tolerances.  Let u = 2^-24.  A value of h is off by u times the magnitudes that enter it, a sum over a row (a tree of at most
8*4 + 5 + 16 steps) by at most 53u of the sum of magnitudes, and every further step adds u relative to what it handles: 2^-17 = 128u
covers the chain, applied to the magnitudes that enter.  Weight gradients are sums of at most 256 steps in a row at the sizes here:
2^-16 of the sum of magnitudes.  A value in 8 bits is the number nearest to one that is off by 2^-17 relative, of a block whose scale is
that of a largest magnitude off by as much: half a step, 2^-4 of it or of the smallest normal number's."""
import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import experts_reference as ref
from tests.test_train_norm import made
from tests.train_reference import assert_close, host

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
SLACK = 2.0 ** -17
TYPES = [(BF, BF), (BF, F), (HF, HF), (HF, F), (F, F)]
SIZES = [(1, 1), (1, 8), (3, 7), (5, 256), (17, 257), (64, 768), (9, 1000), (33, 1023), (4, 2048), (3, 3001), (2, 8192), (2, 16384), (3, 16383), (2500, 96)]


def test_reference_gradient_against_differences():
    rng = np.random.default_rng(3)
    x, r, w, dy, dh = rng.standard_normal((5, 13)), rng.standard_normal((5, 13)), rng.standard_normal(13), rng.standard_normal((5, 13)), rng.standard_normal((5, 13))

    def loss(x, r, w):
        y, h, _ = ref.rms_norm(x, r, w, 1e-5)
        return (y * dy).sum() + (h * dh).sum()

    _, h, rstd = ref.rms_norm(x, r, w, 1e-5)
    dres, dw = ref.rms_norm_backward(dy, h, rstd, w, dh, [0, 5])
    for grad, k in ((dres, 0), (dres, 1), (dw[0], 2)):
        v = rng.standard_normal(grad.shape)
        ends = []
        for s in (1e-5, -1e-5):
            at = [x, r, w]
            at[k] = at[k] + s * v
            ends.append(loss(*at))
        assert abs((ends[0] - ends[1]) / 2e-5 - (grad * v).sum()) < 1e-7 * np.abs(grad * v).sum()


def test_c_entries_refuse():
    """Bad arguments come back as codes before anything is launched (the pointers here are never followed)."""
    lib, p = ref.c_library(), 4096

    def norm(x=p, ldx=64, res=None, ldr=64, w=p, eps=1e-6, y=p, ldy=64, v=None, ldv=64, s=None, lds=2, h=None, ldh=64, rstd=p, rows=4, cols=64, type=1, stream=1):
        return lib.regtopk_rms_norm(x, ldx, res, ldr, w, eps, y, ldy, v, ldv, s, lds, h, ldh, rstd, rows, cols, type, stream, None)
    for bad in (dict(type=3), dict(stream=2), dict(x=None), dict(x=p + 1), dict(ldx=63), dict(res=p, ldr=63), dict(w=None), dict(w=p + 2), dict(eps=-1.0),
                dict(eps=float("nan")), dict(y=None), dict(ldy=63), dict(v=p), dict(s=p), dict(v=p, s=p, ldv=63), dict(v=p, s=p, lds=1), dict(h=p, ldh=63),
                dict(rstd=None), dict(rows=-1), dict(cols=0)):
        assert norm(**bad) == -1, bad
    assert norm(cols=16385) == -7 and norm(rows=0) == 0

    def back(groups=1, offsets=None, ws=p, nbytes=1 << 30, dw=p, ld=8, cols=8, dx=p, stream=0):
        return lib.regtopk_rms_norm_backward(p, 8, p, 8, p, p, None, 0, dx, 8, None, 0, dw, ld, offsets, groups, 0, 4, cols, 0, stream, ws, nbytes, None)
    for bad in (dict(groups=0), dict(groups=2), dict(offsets=p + 4), dict(ws=None), dict(ws=p + 8), dict(groups=2, offsets=p, ld=7), dict(dx=None), dict(stream=1)):
        assert back(**bad) == -1, bad
    assert back(nbytes=8) == -2 and back(cols=20000) == -7 and back(groups=65536, offsets=p) == -7
    need = lib.regtopk_rms_norm_backward_workspace_bytes
    assert need(4, 8, 0) == 0 and need(4, 20000, 1) == 0 and need(4, 8, 1) == 5 * 8 * 4


def test_no_cpu_path():
    with pytest.raises(TypeError):
        rt.rms_norm(torch.zeros(4, 8), torch.ones(8))


def check_norm(x, residual, weight, eps):
    rows, cols = x.shape
    y, y8, h, rstd = rt.rms_norm(x, weight, eps, residual=residual, want_y8=True)
    xs, rs, ws = host(x), None if residual is None else host(residual), host(weight)
    wy, wh, wr = ref.rms_norm(xs, rs, ws, eps)
    size = np.abs(xs) + (0.0 if rs is None else np.abs(rs))
    if residual is None:
        assert h is x
    else:
        assert h.dtype == residual.dtype
        assert_close(h, wh, 2.0 ** -24 * size, h.dtype, "h")
    top = (size ** 2).mean(1)  # what cancels between x and residual is lost to rstd
    assert_close(rstd, wr, SLACK * wr * (1 + top * wr ** 2), F, "rstd")
    slack = SLACK * (size * wr[:, None] * np.abs(ws)) * (1 + (top * wr ** 2)[:, None])
    assert y.dtype == x.dtype
    assert_close(y, wy, slack, x.dtype, "y")
    only, both, _, again = rt.rms_norm(x, weight, eps, residual=residual, want_y=False, want_y8=True)
    assert only is None and torch.equal(again, rstd) and torch.equal(both.values.view(torch.uint8), y8.values.view(torch.uint8))
    alone, none, _, _ = rt.rms_norm(x, weight, eps, residual=residual)
    assert none is None and torch.equal(alone, y)
    # 8 bits
    byte = y8.scales.cpu().view(torch.uint8).numpy().astype(int)
    lo, hi = ref.scale_bytes(np.maximum(np.abs(wy) - slack, 0.0)), ref.scale_bytes(np.abs(wy) + slack)
    assert ((lo <= byte) & (byte <= hi)).all()
    step = np.repeat(2.0 ** (byte - 127.0 - 9), 32, 1)[:, :cols]  # of the numbers below the smallest normal one
    assert (np.abs(ref.unpacked(y8) - wy) <= np.maximum(step / 2, 2.0 ** -4 * (np.abs(wy) + slack)) + slack).all()
    return h, rstd


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_forward(rows, cols, dtype, stream):
    gen = torch.Generator().manual_seed(rows * 17 + cols)
    for pad, shift in ((0, 0), (8, 8), (3, 1)):
        x = made(rows, cols, dtype, gen, pad, shift)
        weight = (1 + 0.3 * torch.randn(cols + 1, generator=gen)).cuda()[1:]  # a view into a flat vector
        check_norm(x, made(rows, cols, stream, gen, pad, shift, scale=2.0), weight.contiguous() if pad == 0 else weight, 1e-5)
        check_norm(x, None, weight, 0.0)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("rows,cols", SIZES)
def test_backward(rows, cols, dtype, stream):
    gen = torch.Generator().manual_seed(rows * 19 + cols)
    for pad, shift, with_dh in ((0, 0, True), (8, 8, False), (3, 1, True)):
        h = made(rows, cols, stream, gen, pad, shift, scale=2.0)
        weight = (1 + 0.3 * torch.randn(cols, generator=gen)).cuda()
        rstd = h.float().square().mean(1).add(1e-5).rsqrt()
        dy = made(rows, cols, dtype, gen, pad, shift)
        dh = made(rows, cols, stream, gen, pad, shift) if with_dh else None
        cuts = [0, rows] if pad == 8 else [rows // 5, rows // 5, rows // 2, rows - rows // 7]
        offsets = None if pad == 8 else torch.tensor(cuts, device="cuda")
        dx, dres, dw = rt.rms_norm_backward(dy, h, rstd, weight, dh=dh, offsets=offsets)
        hs, rs, ws, ds = host(h), host(rstd), host(weight), host(dy)
        want, wdw = ref.rms_norm_backward(ds, hs, rs, ws, None if dh is None else host(dh), cuts)
        u, g = np.abs(hs * rs[:, None]), np.abs(ds * ws)
        size = rs[:, None] * (g + u * (g * u).mean(1)[:, None]) + (0.0 if dh is None else np.abs(host(dh)))
        assert dx.dtype == dtype and dres.dtype == stream and (dres is dx) == (dtype == stream)
        assert_close(dx, want, SLACK * size, dtype, "dx")
        assert_close(dres, want, SLACK * size, stream, "dresidual")
        sums = np.stack([np.abs(ds * hs * rs[:, None])[a:b].sum(0) for a, b in zip(cuts, cuts[1:])])
        assert dw.shape == wdw.shape
        assert_close(dw, wdw, 2.0 ** -16 * sums, F, "dweight")
        # into columns of wider rows, written and added to
        wide = torch.full((len(cuts) - 1, cols + 9), 3.0, device="cuda")
        into = wide[:, 4:4 + cols]
        assert rt.rms_norm_backward(dy, h, rstd, weight, dh=dh, offsets=offsets, dweight=into)[2] is into
        assert torch.equal(into, dw)
        rt.rms_norm_backward(dy, h, rstd, weight, dh=dh, offsets=offsets, dweight=into, accumulate=True)
        assert torch.equal(into, dw + dw) and (wide[:, :4] == 3).all() and (wide[:, 4 + cols:] == 3).all()


@pytest.mark.gpu
def test_edges():
    w = torch.ones(40, device="cuda")
    y, y8, h, rstd = rt.rms_norm(torch.zeros(3, 40, device="cuda"), w, want_y8=True)
    assert not y.any() and torch.allclose(rstd, torch.full((3,), 1e3, device="cuda")) and (ref.unpacked(y8) == 0).all()
    x = torch.randn(3, 40, device="cuda")
    x[1, 7] = float("nan")
    y, y8, _, rstd = rt.rms_norm(x, w, want_y8=True)
    assert y[1].isnan().all() and y[0].isfinite().all() and y[2].isfinite().all() and np.isnan(ref.unpacked(y8)[1]).all()
    for rows in (0,):
        y, _, _, rstd = rt.rms_norm(x[:0], w)
        dx, _, dw = rt.rms_norm_backward(y, x[:0], rstd, w)
        assert dx.shape == (0, 40) and dw.shape == (1, 40) and not dw.any()
    for scale in (2.0 ** -60, 2.0 ** 60):  # squares near both ends of binary32
        check_norm(x[::2].contiguous() * scale, None, w, 0.0)
    at = torch.tensor([2**62, -2**62, 5], device="cuda")  # offsets that do not ascend, as for the layer norm: nothing outside is touched
    rt.rms_norm_backward(x, x, rstd.new_ones(3), w, offsets=at)
    rt.training_status()


@pytest.mark.gpu
def test_refusals():
    x, w = torch.zeros(4, 64, device="cuda"), torch.ones(64, device="cuda")
    y, _, h, rstd = rt.rms_norm(x, w)
    for call in (lambda: rt.rms_norm(x.double(), w), lambda: rt.rms_norm(x, w.to(BF)), lambda: rt.rms_norm(x, w[:8]), lambda: rt.rms_norm(x, w, residual=x[:2]),
                 lambda: rt.rms_norm(x, w, residual=x.to(BF)), lambda: rt.rms_norm(x, w.cpu()), lambda: rt.rms_norm_backward(y, x.to(BF), rstd, w),
                 lambda: rt.rms_norm_backward(y, h, rstd[:2], w), lambda: rt.rms_norm_backward(y, h, rstd, w, dh=x.to(BF)),
                 lambda: rt.rms_norm_backward(y, h, rstd, w, dweight=w), lambda: rt.rms_norm_backward(y, h, rstd, w, offsets=torch.zeros(2, device="cuda"))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: rt.rms_norm(x, w, want_y=False), lambda: rt.rms_norm(x.t(), w[:4]), lambda: rt.rms_norm(x[:1].expand(4, 64), w),
                 lambda: rt.rms_norm_backward(y, h, rstd, w, accumulate=True), lambda: rt.rms_norm_backward(y, h, rstd, w, dweight=w.view(1, 64)), lambda: rt.rms_norm_backward(y, h, rstd, w, dweight=h[:1]), lambda: rt.rms_norm_backward(y, h, rstd, w, dweight=torch.zeros(1, 64, device="cuda", requires_grad=True)),
                 lambda: rt.rms_norm_backward(y, h, rstd, w, offsets=torch.tensor([0, 1, 4], device="cuda"), dweight=w.expand(2, 64))):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: rt.rms_norm(x, w, eps=-1.0), lambda: rt.rms_norm(torch.zeros(2, 16385, device="cuda"), torch.ones(16385, device="cuda"))):
        with pytest.raises(rt.RegTopKError):
            call()
