"""Products grouped by expert and their gradients, against the definition in 64 bits.

Tolerance.  The tensor cores add sixteen products and the running sum at a time, aligned to the largest of them and cut
off no earlier than 2^-23 of it, so that a sum of n products is off by at most (n + 32) 2^-23 times the sum of their
magnitudes, in whatever order; then comes one rounding to the output's type."""
import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import train_reference as ref

BF, HF = torch.bfloat16, torch.float16


def want_rows(x, w, offsets):
    y, slack = np.zeros((x.shape[0], w.shape[1])), np.zeros((x.shape[0], w.shape[1]))
    for g, (a, b) in enumerate(zip(offsets, offsets[1:])):
        m = w[g % len(w)].T
        y[a:b] = x[a:b] @ m
        slack[a:b] = np.abs(np.nan_to_num(x[a:b], posinf=0, neginf=0)) @ np.abs(np.nan_to_num(m, posinf=0, neginf=0))
    return y, (x.shape[1] + 32) * 2.0 ** -23 * slack


def want_weights(dy, x, offsets):
    out = np.stack([dy[a:b].T @ x[a:b] for a, b in zip(offsets, offsets[1:])])
    slack = np.stack([(b - a + 32) * 2.0 ** -23 * (np.abs(dy[a:b]).T @ np.abs(x[a:b])) for a, b in zip(offsets, offsets[1:])])
    return out, np.nan_to_num(slack)


def test_reference_gradients_against_differences():
    """The two gradients as products, against central differences of the forward products, in 64 bits."""
    rng = np.random.default_rng(5)
    x, w, dy = rng.standard_normal((9, 4)), rng.standard_normal((2, 3, 4)), rng.standard_normal((9, 3))
    at = [0, 2, 2, 7, 9]
    dx = want_rows(dy, w.transpose(0, 2, 1), at)[0]
    dw = want_weights(dy, x, at)[0].reshape(2, 2, 3, 4).sum(0)
    for grad, k in ((dx, 0), (dw, 1)):
        v = rng.standard_normal(grad.shape)
        ends = []
        for s in (1e-5, -1e-5):
            xw = [x, w]
            xw[k] = xw[k] + s * v
            ends.append((want_rows(*xw, at)[0] * dy).sum())
        assert abs((ends[0] - ends[1]) / 2e-5 - (grad * v).sum()) < 1e-7 * np.abs(grad * v).sum()


def test_c_entries_refuse():
    lib, p = ref.c_library(), 4096

    def rows(x=p, w=p, y=p, off=p, groups=4, weights=2, type=1, rows=8, k=16, m=16, ldx=16, ldw=16, ldy=16, ws=None, nbytes=0, stride=256):
        return lib.regtopk_grouped_matmul(x, ldx, w, ldw, stride, 0, weights, y, ldy, off, groups, rows, k, m, type, ws, nbytes, None)
    assert rows(type=0) == -1 and rows(groups=3) == -1 and rows(groups=0) == -1 and rows(weights=0) == -1
    assert rows(off=None) == -1 and rows(off=p + 4) == -1 and rows(x=None) == -1 and rows(w=None) == -1 and rows(y=None) == -1
    assert rows(ldx=15) == -1 and rows(ldy=15) == -1 and rows(ldw=15) == -1 and rows(x=p + 1) == -1 and rows(stride=-1) == -1
    assert rows(rows=-1) == -1 and rows(rows=1 << 31) == -1 and rows(groups=4096, weights=1) == -7
    assert rows(rows=0) == 0 and rows(m=0) == 0

    def dw(dy=p, x=p, out=p, off=p, groups=4, inner=2, type=2, rows=8, k=16, m=16, ld=16, ldo=16, acc=0):
        return lib.regtopk_grouped_matmul_dw(dy, ld, x, ld, out, ldo, 256, 512, inner, acc, off, groups, rows, k, m, type, None, 0, None)
    assert dw(type=0) == -1 and dw(inner=3) == -1 and dw(inner=0) == -1 and dw(off=None) == -1 and dw(out=None) == -1
    assert dw(out=p + 2) == -1 and dw(ldo=15) == -1 and dw(ld=15) == -1 and dw(dy=None) == -1 and dw(x=None) == -1
    assert dw(groups=4096) == -7 and dw(k=0) == 0 and dw(rows=0, acc=1) == 0
    size = lib.regtopk_grouped_matmul_workspace_bytes
    assert size(p, 16, p, 16, 256, 0, 2, 4, 8, 16, 16) == 0
    assert size(p, 17, p, 16, 256, 0, 2, 4, 8, 16, 16) >= 8 * 16 * 2 and size(p, 16, p, 17, 272, 0, 2, 4, 8, 16, 16) >= 2 * 16 * 16 * 2
    assert size(p, 16, p + 2, 16, 256, 0, 2, 4, 8, 16, 16) > 0 and size(p, 16, p, 16, 260, 0, 2, 4, 8, 16, 16) > 0


# ---- on the GPU ----------------------------------------------------------------------------------------------------------
def made(shape, dtype, gen, pad=0, shift=0):
    """A matrix (or several) with `pad` unused elements behind each row, beginning `shift` elements into its storage."""
    full = (*shape[:-1], shape[-1] + pad)
    flat = torch.full((int(np.prod(full)) + shift,), float("nan"), dtype=dtype, device="cuda")
    t = flat[shift:].view(full)[..., : shape[-1]]
    t.copy_(torch.randn(shape, generator=gen).to(dtype))
    return t


def cut(rows, groups, gen):
    return [0, *sorted(int(i) for i in torch.randint(0, rows + 1, (groups - 1,), generator=gen)), rows]


SIZES = [  # rows, workers, experts, k, m
    (1, 1, 1, 1, 1), (5, 1, 2, 8, 8), (1, 1, 1, 64, 128), (33, 1, 3, 64, 128), (40, 2, 2, 72, 136), (100, 2, 4, 17, 130),
    (257, 1, 2, 128, 130), (300, 1, 5, 65, 257), (64, 4, 16, 40, 24), (1000, 1, 3, 200, 384), (513, 1, 1, 1000, 72),
    (2000, 2, 2, 136, 264), (700, 1, 1, 31, 600), (4500, 1, 2, 264, 1100), (40, 1, 2, 2200, 130), (5, 2, 2, 4100, 60), (90, 1, 1, 2049, 300),
    (3000, 1, 1, 72, 100)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("size", SIZES)
def test_grouped_matmul(size, dtype):
    rows, n, e, k, m = size
    gen = torch.Generator().manual_seed(sum(size))
    at = cut(rows, n * e, gen)
    offsets = torch.tensor(at, device="cuda")
    for pad, shift in ((0, 0), (8, 8), (3, 1)):
        x, w = made((rows, k), dtype, gen, pad, shift), made((e, m, k), dtype, gen, pad, shift)
        want, slack = want_rows(ref.host(x), ref.host(w), at)
        ref.assert_close(rt.grouped_matmul(x, w, offsets), want, slack, dtype, f"pad {pad}")
        wt = made((e, k, m), dtype, gen, pad, shift)
        want, slack = want_rows(ref.host(x), ref.host(wt).transpose(0, 2, 1), at)
        out = made((rows, m), dtype, gen, pad, shift)
        assert rt.grouped_matmul(x, wt.transpose(1, 2), offsets, out=out) is out
        ref.assert_close(out, want, slack, dtype, f"transposed, pad {pad}")
    rt.training_status()


@pytest.mark.gpu
def test_grouped_matmul_groups():
    """Rows of no group become zeros, values in other rows (NaN among them) reach nobody else, one matrix shared by all
    groups, more groups than rows, offsets out of range or descending touch nothing outside."""
    gen = torch.Generator().manual_seed(4)
    rows, k, m = 300, 96, 200
    x, w = made((rows, k), BF, gen), made((3, m, k), BF, gen)
    x[:7] = float("nan")
    x[290:] = float("inf")
    x[100:110] = float("nan")
    for at in ([7, 60, 100, 290], [7, 7, 7, 7], [110, 111, 290, 290], [110, 110, 290, 290]):
        buf = torch.full((rows + 2, m), 3.0, dtype=BF, device="cuda")
        rt.grouped_matmul(x, w, torch.tensor(at, device="cuda"), out=buf[1:-1])
        xs = ref.host(x)
        want, slack = want_rows(xs, ref.host(w), at)
        ref.assert_close(buf[1:-1], want, slack, BF, str(at))
        assert (buf[0] == 3).all() and (buf[-1] == 3).all()
    y = torch.randn(rows, k, generator=gen).to(BF).cuda()
    at = sorted(int(i) for i in torch.randint(0, rows + 1, (2047,), generator=gen))
    at = [0, *at, rows]
    want, slack = want_rows(ref.host(y), ref.host(w[:1]), at)
    offsets = torch.tensor(at, device="cuda")
    ref.assert_close(rt.grouped_matmul(y, w[:1], offsets), want, slack, BF, "one matrix")
    same = rt.grouped_matmul(y, w[:1].expand(4, m, k), offsets)
    ref.assert_close(same, want, slack, BF, "one matrix, expanded")
    for bad in ([-5, 1000, 2**40, 7], [300, 200, 100, 0], [2**62, -2**62, 0, 2**62]):
        buf = torch.full((rows + 2, m), 3.0, dtype=BF, device="cuda")
        rt.grouped_matmul(y, w, torch.tensor(bad, device="cuda"), out=buf[1:-1])
        torch.cuda.synchronize()
        assert (buf[0] == 3).all() and (buf[-1] == 3).all()
    rt.training_status()


@pytest.mark.gpu
def test_grouped_matmul_empty():
    x, w = torch.zeros(0, 16, dtype=BF, device="cuda"), torch.zeros(2, 8, 16, dtype=BF, device="cuda")
    offsets = torch.zeros(3, dtype=torch.int64, device="cuda")
    assert rt.grouped_matmul(x, w, offsets).shape == (0, 8)
    assert not rt.grouped_matmul_dw(x[:, :8], x, offsets).any()
    y = rt.grouped_matmul(torch.ones(3, 0, dtype=BF, device="cuda"), torch.ones(2, 8, 0, dtype=BF, device="cuda"), offsets)
    assert y.shape == (3, 8) and not y.any()
    out = torch.ones(2, 8, 16, device="cuda")
    rt.grouped_matmul_dw(x[:, :8], x, offsets, out=out, accumulate=True)
    assert (out == 1).all()
    assert rt.grouped_matmul_dw(torch.ones(3, 0, dtype=BF, device="cuda"), torch.ones(3, 16, dtype=BF, device="cuda"), offsets).shape == (2, 0, 16)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("size", SIZES)
def test_grouped_matmul_dw(size, dtype):
    rows, n, e, k, m = size
    gen = torch.Generator().manual_seed(sum(size) + 1)
    at = cut(rows, n * e, gen)
    offsets = torch.tensor(at, device="cuda")
    for pad, shift in ((0, 0), (8, 8), (3, 1)):
        dy, x = made((rows, m), dtype, gen, pad, shift), made((rows, k), dtype, gen, pad, shift)
        want, slack = want_weights(ref.host(dy), ref.host(x), at)
        got = rt.grouped_matmul_dw(dy, x, offsets)
        ref.assert_close(got, want, slack, torch.float32, f"pad {pad}")
        # into columns of wider rows, at an odd place, written and then added
        flat = torch.randn(n, 5 + e * m * k + 2, generator=gen).cuda()
        before = flat.clone()
        view = flat[:, 5: 5 + e * m * k].view(n, e, m, k)
        assert rt.grouped_matmul_dw(dy, x, offsets, out=view) is view
        assert torch.equal(view, got.view(n, e, m, k))
        view.copy_(before[:, 5: 5 + e * m * k].view(n, e, m, k))
        rt.grouped_matmul_dw(dy, x, offsets, out=view, accumulate=True)
        before[:, 5: 5 + e * m * k] += got.view(n, -1)
        assert torch.equal(flat, before)
    rt.training_status()


@pytest.mark.gpu
def test_grouped_matmul_dw_groups():
    """A group's values reach its own matrix alone, whatever they are; rows of no group reach none; bad offsets touch
    nothing outside; equal calls give equal bits."""
    gen = torch.Generator().manual_seed(6)
    rows, k, m = 500, 136, 72
    dy, x = made((rows, m), BF, gen), made((rows, k), BF, gen)
    dy[:3] = float("nan")
    x[3:5] = float("inf")
    x[490:] = float("nan")
    dy[201, 5] = float("nan")
    at = [5, 70, 70, 201, 202, 203, 490]
    offsets = torch.tensor(at, device="cuda")
    got = rt.grouped_matmul_dw(dy, x, offsets)
    want, slack = want_weights(ref.host(dy), ref.host(x), at)
    assert np.isnan(want[3]).any() and np.isfinite(np.delete(want, 3, 0)).all()
    ref.assert_close(got, want, slack, torch.float32, "groups")
    assert torch.equal(got.nan_to_num(), rt.grouped_matmul_dw(dy, x, offsets).nan_to_num())
    for bad in ([-5, 1000, 2**40, 7], [300, 200, 100, 0], [2**62, -2**62, 0, 2**62]):
        buf = torch.full((5, m, k), 3.0, device="cuda")
        rt.grouped_matmul_dw(dy, x, torch.tensor(bad, device="cuda"), out=buf[1:-1])
        torch.cuda.synchronize()
        assert (buf[0] == 3).all() and (buf[-1] == 3).all()
    rt.training_status()


@pytest.mark.gpu
@pytest.mark.parametrize("rows,groups", [(6000, 1), (20000, 2), (3000, 7)])
def test_grouped_matmul_dw_long(rows, groups):
    """Long sums of values that do not cancel: the error of a sum that loses its low bits at every step would grow with
    the length; 2^-20 of the result is what sixteen steps of 2^-24 allow."""
    gen = torch.Generator().manual_seed(rows)
    dy = (1 + 0.1 * torch.randn(rows, 130, generator=gen)).to(BF).cuda()
    x = (1 + 0.1 * torch.randn(rows, 70, generator=gen)).to(BF).cuda()
    at = cut(rows, groups, gen)
    got = rt.grouped_matmul_dw(dy, x, torch.tensor(at, device="cuda"))
    want, _ = want_weights(ref.host(dy), ref.host(x), at)
    assert np.linalg.norm(ref.host(got) - want) < 2.0 ** -20 * np.linalg.norm(want)
    rt.training_status()


@pytest.mark.gpu
def test_grouped_matmul_gradient_against_differences():
    """dx and dw against differences of the forward product; the inputs move by steps that bfloat16 holds exactly, the
    products are linear, so that only the output's rounding (2^-8 of y) and binary32 sums are between them."""
    gen = torch.Generator().manual_seed(9)
    rows, e, k, m = 90, 3, 40, 24
    offsets = torch.tensor(cut(rows, e, gen), device="cuda")
    whole = lambda *s: torch.randint(-4, 5, s, generator=gen).to(BF).cuda()  # noqa: E731
    x, w, dy, vx, vw = whole(rows, k), whole(e, m, k), whole(rows, m), whole(rows, k), whole(e, m, k)
    dx, dw = rt.grouped_matmul(dy, w.transpose(1, 2), offsets), rt.grouped_matmul_dw(dy, x, offsets)
    loss = lambda x, w: (rt.grouped_matmul(x, w, offsets).double() * dy.double()).sum()  # noqa: E731
    for got, up, down, grad, v in ((dx, (x + vx, w), (x - vx, w), dx, vx), (dw, (x, w + vw), (x, w - vw), dw, vw)):
        scale = (rt.grouped_matmul(*up, offsets).double().abs() * dy.double().abs()).sum()
        assert abs((loss(*up) - loss(*down)) / 2 - (grad.double() * v.double()).sum()) < 2.0 ** -7 * scale
    rt.training_status()


@pytest.mark.gpu
def test_refusals():
    x, w = torch.zeros(8, 16, dtype=BF, device="cuda"), torch.zeros(2, 24, 16, dtype=BF, device="cuda")
    dy, off = torch.zeros(8, 24, dtype=BF, device="cuda"), torch.tensor([0, 3, 8], device="cuda")
    for call, error in [
            (lambda: rt.grouped_matmul(x.float(), w.float(), off), TypeError), (lambda: rt.grouped_matmul(x, w.half(), off), TypeError),
            (lambda: rt.grouped_matmul(x.cpu(), w, off), TypeError), (lambda: rt.grouped_matmul(x, w[0], off), TypeError),
            (lambda: rt.grouped_matmul(x[:, :8], w, off), TypeError), (lambda: rt.grouped_matmul(x, w, off[:2]), ValueError),
            (lambda: rt.grouped_matmul(x, w, off.int()), TypeError), (lambda: rt.grouped_matmul(x, w, off.cpu()), TypeError),
            (lambda: rt.grouped_matmul(dy.t(), w[:, :, :8], off), ValueError), (lambda: rt.grouped_matmul(x, w, off, out=dy[:4]), TypeError),
            (lambda: rt.grouped_matmul(x, torch.zeros(2, 48, 32, dtype=BF, device="cuda")[:, ::2, ::2], off), ValueError),
            (lambda: rt.grouped_matmul(x, w[:, :1].expand(2, 24, 16), off), ValueError),
            (lambda: rt.grouped_matmul(x[None], w, off), ValueError),
            (lambda: rt.grouped_matmul(x, w[:1], torch.zeros(2050, dtype=torch.int64, device="cuda")), rt.RegTopKError),
            (lambda: rt.grouped_matmul_dw(dy, x[:4], off), TypeError), (lambda: rt.grouped_matmul_dw(dy.float(), x, off), TypeError),
            (lambda: rt.grouped_matmul_dw(dy, x, off, accumulate=True), ValueError),
            (lambda: rt.grouped_matmul_dw(dy, x, off, out=torch.zeros(2, 24, 16, dtype=BF, device="cuda")), TypeError),
            (lambda: rt.grouped_matmul_dw(dy, x, off, out=torch.zeros(3, 24, 16, device="cuda")), TypeError),
            (lambda: rt.grouped_matmul_dw(dy, x, off, out=torch.zeros(2, 16, 24, device="cuda").transpose(1, 2)), ValueError),
            (lambda: rt.grouped_matmul_dw(dy, x, off, out=torch.zeros(2, 1, 16, device="cuda").expand(2, 24, 16)), ValueError)]:
        with pytest.raises(error):
            call()
