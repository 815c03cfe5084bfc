"""The training operators at the edges of what they take: layouts, lengths and values at which the arithmetic of addresses,
counters and sums could go wrong, against the definitions in 64 bits where there is a result."""
import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import train_reference as ref
from tests.test_train_norm import TYPES, check_norm, norm_case
from tests.test_train_norm import made as rows_made

BF, HF, F = torch.bfloat16, torch.float16, torch.float32


def padded(rows, cols, dtype, gen, pad, shift=0, fill=0.0):
    """(a [rows, cols] tensor with `pad` more columns behind each row, beginning `shift` elements into its storage, which is `fill`
    otherwise; the storage's whole rows)."""
    flat = torch.full((rows * (cols + pad) + shift,), fill, dtype=dtype, device="cuda")
    whole = flat[shift:].view(rows, cols + pad)
    whole[:, :cols] = torch.randn(rows, cols, generator=gen).to(dtype)
    return whole[:, :cols], whole


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("rows,cols", [(2, 8), (300, 8), (4099, 8), (300, 16), (129, 24), (65, 520)])
def test_dropout_of_short_rows(rows, cols, dtype):
    """Rows of one group of eight columns and of a few: each row has its own mask and stays in its place, contiguous or a view of
    wider rows, aligned or not, and the columns behind it keep what they hold."""
    gen = torch.Generator().manual_seed(rows + cols)
    keep, factor = ref.keep_mask(rows, cols, 0.4, 2**63 + 5, 31)
    for pad, out_pad, shift in ((0, 0, 0), (16, 0, 0), (0, 8, 0), (8, 24, 0), (8, 8, 1), (0, 0, 3)):
        x, _ = padded(rows, cols, dtype, gen, pad, shift)
        out, whole = padded(rows, cols, dtype, gen, out_pad, shift, fill=3.0)
        want = torch.where(torch.from_numpy(keep), x.cpu().float() * torch.tensor(factor, dtype=F), 0.0).to(dtype)
        assert torch.equal(rt.dropout(x, 0.4, 2**63 + 5, 31).cpu(), want), (pad, shift)
        rt.dropout(x, 0.4, 2**63 + 5, 31, out=out)
        assert torch.equal(out.cpu(), want), (pad, out_pad, shift)
        assert (whole[:, cols:] == 3).all()


def keep_of_groups(groups, p, seed, subsequence):
    """The mask of row 0 in the groups of eight columns that are numbered here."""
    words = ref.philox([np.asarray(groups, np.uint64), 0, 0, subsequence], (seed & 0xFFFFFFFF, seed >> 32))
    numbers = np.stack([(w >> np.uint64(s)) & np.uint64(0xFFFF) for w in words for s in (0, 16)], -1)
    return (numbers >= int(round(65536 * p))).reshape(-1)


def test_mask_of_groups():
    assert np.array_equal(keep_of_groups(range(40), 0.3, 12345678901, 8), ref.keep_mask(1, 320, 0.3, 12345678901, 8)[0][0])


@pytest.mark.gpu
@pytest.mark.parametrize("extra", [4104, 4103])
def test_dropout_of_a_row_past_32_bits(extra):
    """One row of more than 2^32 columns, in place, a multiple of eight columns and not: the start, what lies on both sides of
    column 2^32 and the end."""
    cols = 2**32 + extra
    x = torch.ones(cols, dtype=BF, device="cuda")
    rt.dropout(x, 0.25, 5, 6, out=x)
    for first in (0, 2**31 - 4096, 2**32 - 4096, 2**32):
        here = x[first: first + 8192]
        want = keep_of_groups(range(first // 8, first // 8 + 1024), 0.25, 5, 6)[: here.numel()]
        assert np.array_equal(here.float().cpu().numpy() != 0, want), first


@pytest.mark.gpu
def test_rows_that_repeat_are_refused():
    """An expanded dimension between others has distance 0, which is no distance from row to row: such a tensor (the gradient of
    a sum over tokens, say) holds fewer elements than its rows.  Dimensions of one element may have any distance."""
    x, w = torch.randn(4, 5, 16, device="cuda"), torch.ones(16, device="cuda")
    y, h, mean, rstd = rt.layer_norm(x, w)
    for wide in (torch.randn(4, 1, 16, device="cuda").expand(4, 5, 16), torch.randn(1, 5, 16, device="cuda").expand(4, 5, 16),
                 torch.randn(16, device="cuda").expand(4, 5, 16)):
        for call in (lambda: rt.dropout(wide, 0.1, 0), lambda: rt.dropout(x, 0.1, 0, out=wide), lambda: rt.layer_norm(wide, w),
                     lambda: rt.layer_norm(x, w, residual=wide), lambda: rt.layer_norm_backward(wide, h, mean, rstd, w),
                     lambda: rt.layer_norm_backward(y, wide, mean, rstd, w), lambda: rt.layer_norm_backward(y, h, mean, rstd, w, dh=wide)):
            with pytest.raises(ValueError):
                call()
    four = torch.randn(2, 3, 1, 16, device="cuda").expand(2, 3, 5, 16)
    with pytest.raises(ValueError):
        rt.dropout(four, 0.1, 0)
    one = x[:1].as_strided((1, 5, 16), (0, 16, 1))
    assert torch.equal(rt.layer_norm(one, w)[0], y[:1])
    assert torch.equal(rt.layer_norm(x[:, :1].as_strided((4, 1, 16), (80, 0, 1)), w)[0], y[:, :1])


def test_c_matrices_that_overlap():
    """Before anything is launched (the pointer is never followed): distances that let two rows of the gradient meet."""
    lib = ref.c_library()

    def dw(ld=16, inner=2, inner_stride=384, outer_stride=768, groups=4, m=24):
        p = 4096
        return lib.regtopk_grouped_matmul_dw(p, 24, p, 16, p, ld, inner_stride, outer_stride, inner, 0, p, groups, 0, 16, m, 1, None, 0, None)
    assert dw(inner_stride=0) == -1 and dw(inner_stride=383) == -1 and dw(outer_stride=0) == -1 and dw(outer_stride=767) == -1
    assert dw(ld=17) == -1 and dw(inner=4, inner_stride=383) == -1 and dw(ld=32, inner_stride=15, outer_stride=768) == -1
    assert dw(inner_stride=2**62, outer_stride=2**62) == -1


def test_c_most_groups():
    """More groups than a launch has rows of blocks come back as too large, as the products' do."""
    lib, p = ref.c_library(), 4096

    def back(groups, rows=0):
        return lib.regtopk_layer_norm_backward(p, 8, p, 8, p, p, p, None, 0, p, 8, None, 0, p, 8, None, 0, p, groups, 0, rows, 8, 0, 0, None, p, 1 << 40, None)
    assert back(65536) == -7 and back(65536, 4) == -7 and back(0) == -1


@pytest.mark.gpu
def test_most_groups():
    h = torch.randn(300, 24, generator=torch.Generator().manual_seed(1)).cuda()
    w = torch.ones(24, device="cuda")
    _, _, mean, rstd = rt.layer_norm(h, w)
    at = torch.arange(65536, device="cuda").clamp(max=300)  # a group for each row, and empty ones
    _, _, dw, db = rt.layer_norm_backward(h, h, mean, rstd, w, offsets=at)
    assert torch.equal(db[:300], h) and not db[300:].any() and not dw[300:].any()
    with pytest.raises(rt.RegTopKError):
        rt.layer_norm_backward(h, h, mean, rstd, w, offsets=torch.arange(65537, device="cuda").clamp(max=300))


@pytest.mark.gpu
def test_matrices_that_overlap_are_refused():
    gen = torch.Generator().manual_seed(3)
    dy, x = torch.randn(40, 24, generator=gen).to(BF).cuda(), torch.randn(40, 16, generator=gen).to(BF).cuda()
    off = torch.tensor([0, 3, 8, 30, 40], device="cuda")
    flat = torch.zeros(4 * 24 * 16, device="cuda")
    for out in (flat[:384].view(1, 24, 16).expand(4, 24, 16), flat[:768].view(2, 1, 24, 16).expand(2, 2, 24, 16),
                flat[:768].view(1, 2, 24, 16).expand(2, 2, 24, 16), flat.as_strided((4, 24, 16), (383, 16, 1)),
                flat.as_strided((4, 24, 16), (15, 64, 1)), flat.as_strided((2, 2, 24, 16), (384, 384, 16, 1))):
        for accumulate in (False, True):
            with pytest.raises(ValueError):
                rt.grouped_matmul_dw(dy, x, off, out=out, accumulate=accumulate)
    assert not flat.any()
    want = rt.grouped_matmul_dw(dy, x, off)
    for out in (torch.zeros(24, 4, 16, device="cuda").transpose(0, 1), torch.zeros(24, 2, 2, 16, device="cuda").permute(2, 1, 0, 3),
                torch.zeros(4, 24, 21, device="cuda")[:, :, :16]):
        rt.grouped_matmul_dw(dy, x, off, out=out, accumulate=True)
        assert torch.equal(out.reshape(4, 24, 16), want), "rows that lie between one another do not overlap"


def check_back(dy, h, mean, rstd, weight, dh=None, offsets=None, p=0.0):
    """layer_norm_backward against the formula in 64 bits for the mean and rstd given.

    Tolerance: h - mean is rounded once, and exact where the two are within a factor of two; with the product by rstd the
    normalised value u is off by 2 * 2^-24 of itself, however large the mean.  A sum over a row in a tree of at most 8*4 + 5 + 16
    steps adds 53 * 2^-24 of the sum of magnitudes, and each further step 2^-24 of what it handles: 2^-17 covers the chain, applied
    to the terms rstd |g|, rstd mean|g| and rstd |u| mean|g u|.  The sums over rows take at most 256 steps in a row here: 2^-16."""
    at = [0, len(dy)] if offsets is None else offsets
    dev = None if offsets is None else torch.tensor(offsets, device="cuda")
    dx, dres, dw, db = rt.layer_norm_backward(dy, h, mean, rstd, weight, dh=dh, p=p, seed=4, subsequence=9, offsets=dev)
    d = [ref.host(t) for t in (dy, h, mean, rstd, weight)]
    wx, wr, ww, wb = ref.layer_norm_backward(*d, None if dh is None else ref.host(dh), p, 4, 9, at)
    unit, g = np.abs(d[1] - d[2][:, None]) * d[3][:, None], np.abs(d[0] * d[4])
    slack = 2.0 ** -17 * (d[3][:, None] * (g + g.mean(1)[:, None] + unit * (g * unit).mean(1)[:, None])
                          + (0 if dh is None else np.abs(ref.host(dh))))
    ref.assert_close(dx, wx, slack * 65536 / (65536 - round(65536 * p)), dy.dtype, "dx")
    ref.assert_close(dres, wr, slack, h.dtype, "dresidual")
    for got, want, size, name in ((dw, ww, np.abs(d[0]) * unit, "dweight"), (db, wb, np.abs(d[0]), "dbias")):
        ref.assert_close(got, want, 2.0 ** -16 * np.stack([size[a:b].sum(0) for a, b in zip(at, at[1:])]), F, name)
    return dx, dres, dw, db


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,stream", [(F, F), (BF, F), (BF, BF), (HF, HF)])
@pytest.mark.parametrize("rows,cols", [(60, 1024), (9, 1001), (2500, 768), (2500, 333), (200, 8192)])
def test_norm_gradient_with_a_large_mean(rows, cols, dtype, stream):
    """Rows whose mean is 0 to 10,000 times their deviation, and constant rows, whose normalised values are zeros."""
    gen = torch.Generator().manual_seed(rows + cols)
    means = 10.0 ** torch.randint(-1, 5, (rows, 1), generator=gen).float()
    h = (torch.randn(rows, cols, generator=gen) + means).to(stream).cuda()
    dy, weight = torch.randn(rows, cols, generator=gen).to(dtype).cuda(), torch.randn(cols, generator=gen).cuda()
    _, _, mean, rstd = rt.layer_norm(h, weight)
    check_back(dy, h, mean, rstd, weight, offsets=[0, rows // 3, rows])
    _, _, dw, _ = rt.layer_norm_backward(dy, torch.full_like(h, 100.0), torch.full_like(mean, 100.0), torch.full_like(rstd, 316.0), weight)
    assert not dw.any()


@pytest.mark.gpu
def test_norm_statistics_over_the_range():
    """The division behind the mean and the reciprocal root behind rstd, from the smallest values to the largest.

    Rows [a, -a, 0, 0] with a a power of two have mean 0 and the variance a^2 / 2 without a rounding, down to the smallest
    number that binary32 has (a = 2^-74); the root of Newton's step is within 2^-22.  Rows with a single value v have the sum v
    without a rounding: the mean is off by three roundings at most, each 2^-24 of it or half the smallest number."""
    power = torch.arange(-74, 63)
    a = torch.ldexp(torch.ones(len(power)), power)
    x = torch.stack([a, -a, 0 * a, 0 * a], 1).cuda()
    _, _, mean, rstd = rt.layer_norm(x, torch.ones(4, device="cuda"), eps=0.0)
    want = 2.0 ** (0.5 - power.double().numpy())
    assert not mean.any()
    off = np.abs(ref.host(rstd) / want - 1)
    assert (off < 2.0 ** -22).all(), (power[int(off.argmax())], off.max())
    assert torch.isinf(rt.layer_norm(torch.zeros(2, 4, device="cuda"), torch.ones(4, device="cuda"), eps=0.0)[3]).all()
    v = torch.ldexp(1 + torch.rand(3000, generator=torch.Generator().manual_seed(1)), torch.randint(-149, 128, (3000,), generator=torch.Generator().manual_seed(2)))
    v[:4] = torch.tensor([2.0**-149, 3 * 2.0**-149, 2.0**-126, torch.finfo(F).max])
    for cols in (1, 3, 7, 96, 511, 1000, 3001):
        x = torch.zeros(3000, cols)
        x[torch.arange(3000), torch.arange(3000) % cols] = v
        mean = ref.host(rt.layer_norm(x.cuda(), torch.ones(cols, device="cuda"))[2])
        want = v.double().numpy() / cols
        assert (np.abs(mean - want) <= 3 * (2.0 ** -24 * want + 2.0 ** -150)).all(), cols
    whole = torch.randint(-1000, 1001, (500, 37), generator=torch.Generator().manual_seed(3)).float()
    whole[:, 0] -= whole.sum(1) % 37
    assert torch.equal(rt.layer_norm(whole.cuda(), torch.ones(37, device="cuda"))[2].cpu(), whole.sum(1) / 37), "whole means are exact"


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [8, 20, 300, 520, 1000, 1023])
@pytest.mark.parametrize("rows", [7, 3000])
def test_norm_gradient_of_huge_rows(rows, cols):
    """A mean whose product with rstd passes binary32's range: what lies past the end of a row, where nothing is, must not
    reach the sums over the row.  The rows here are constant, so that dx = rstd (g - mean(g)), and dweight is 0."""
    gen = torch.Generator().manual_seed(cols)
    dy, weight = torch.randn(rows, cols, generator=gen).cuda(), torch.randn(cols, generator=gen).cuda()
    h, mean, rstd = (torch.full(s, v, device="cuda") for s, v in (((rows, cols), 3e37), ((rows,), 3e37), ((rows,), 316.0)))
    _, _, dw, _ = check_back(dy, h, mean, rstd, weight)
    assert not dw.any()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [HF, BF])
@pytest.mark.parametrize("rows,groups,k,m,transposed", [
    (2400, 150, 16384, 128, False), (2400, 150, 65536, 128, False), (3300, 75, 12345, 140, True), (5000, 20, 9000, 300, False),
    (9000, 3, 8192, 1030, True), (9000, 40, 6001, 90, False), (40, 2, 65536, 300, False), (3000, 60, 4097, 264, True)])
def test_long_products(rows, groups, k, m, transposed, dtype):
    """Sums of thousands of values of one sign, in tiles of every width.  The tensor core cuts its running sum off at every step
    of sixteen terms, always to the same side, so that the error grows with the steps of one accumulator.

    Tolerance: half a step of the output's type, and for an accumulator of up to 4,096 terms 256 steps of at most twice 2^-23 of the
    sum, 2^-14 in all; accumulators are joined with one rounding of 2^-24 each."""
    gen = torch.Generator(device="cuda").manual_seed(rows + k)
    made = lambda *s: (1 + 0.1 * torch.randn(*s, generator=gen, device="cuda")).to(dtype)  # noqa: E731
    x, w = made(rows, k), 2.0 ** -8 * made(2, k, m).transpose(1, 2) if transposed else 2.0 ** -8 * made(2, m, k)
    at = [0, *sorted(int(i) for i in torch.randint(0, rows + 1, (2 * groups - 1,), generator=gen, device="cuda")), rows]
    got = rt.grouped_matmul(x, w, torch.tensor(at, device="cuda")).double()
    half, most = 2.0 ** -11 if dtype == HF else 2.0 ** -8, 0.0
    for g, (lo, hi) in enumerate(zip(at, at[1:])):
        if lo < hi:
            want = x[lo:hi].double() @ w[g % 2].double().T
            most = max(most, float(((got[lo:hi] - want).abs() / want).max()))
    assert most < half + 2.0 ** -14 + (k // 4096 + 1) * 2.0 ** -24, most
    rt.training_status()


@pytest.mark.gpu
def test_autograd_notices_what_is_written():
    """A tensor that a call writes: its version goes up (so that a backward pass that saved it refuses to use it), and while
    autograd records it must not require a gradient."""
    x, w = torch.randn(40, 16, device="cuda"), torch.ones(16, device="cuda")
    dy, xs, ws = torch.randn(40, 24, device="cuda").to(BF), x.to(BF), torch.randn(2, 24, 16, device="cuda").to(BF)
    off = torch.tensor([0, 15, 40], device="cuda")
    _, _, mean, rstd = rt.layer_norm(x, w)
    calls = [(lambda out: rt.dropout(x, 0.1, 0, out=out), torch.zeros(40, 16, device="cuda")),
             (lambda out: rt.layer_norm_backward(x, x, mean, rstd, w, offsets=off, dweight=out), torch.zeros(2, 16, device="cuda")),
             (lambda out: rt.layer_norm_backward(x, x, mean, rstd, w, offsets=off, dbias=out, accumulate=True), torch.zeros(2, 16, device="cuda")),
             (lambda out: rt.grouped_matmul(xs, ws, off, out=out), torch.zeros(40, 24, dtype=BF, device="cuda")),
             (lambda out: rt.grouped_matmul_dw(dy, xs, off, out=out), torch.zeros(2, 24, 16, device="cuda"))]
    for call, out in calls:
        before = out._version
        call(out)
        assert out._version == before + 1
        scale = torch.ones_like(out, requires_grad=True)
        loss = (scale * out).sum()  # saves out for the gradient to scale
        call(out)
        with pytest.raises(RuntimeError, match="modified by an inplace operation"):
            loss.backward()
        leaf = out.clone().requires_grad_()
        with pytest.raises(ValueError):
            call(leaf)
        with torch.no_grad():
            call(leaf)
        assert torch.equal(leaf, out) or call is calls[2][0], "accumulates"
    with torch.inference_mode():
        rt.dropout(x, 0.1, 0, out=torch.zeros(40, 16, device="cuda"))
    shared = torch.zeros(2, 32, device="cuda")
    rt.layer_norm_backward(x, x, mean, rstd, w, offsets=off, dweight=shared[:, :16], dbias=shared[:, 16:])
    assert shared._version > 0


@pytest.mark.gpu
def test_outputs_that_overlap_inputs_are_refused():
    flat = torch.ones(4096, device="cuda")
    x = flat[:1024].view(64, 16)
    for out in (flat[16:1040].view(64, 16), flat[1008:2032].view(64, 16)):
        with pytest.raises(ValueError):
            rt.dropout(x, 0.5, 1, out=out)
    assert (flat == 1).all()
    assert torch.equal(rt.dropout(x, 0.5, 1, out=flat[1024:2048].view(64, 16)), rt.dropout(x, 0.5, 1))
    rt.dropout(x, 0.5, 1, out=x)
    off = torch.tensor([0, 10, 32], device="cuda")
    short = torch.ones(4096, dtype=BF, device="cuda")
    a, w = short[:512].view(32, 16), short[1024:1536].view(2, 16, 16)
    for out in (a, short[256:768].view(32, 16), short[1000:1512].view(32, 16)):
        with pytest.raises(ValueError):
            rt.grouped_matmul(a, w, off, out=out)
    assert (short == 1).all()
    assert (rt.grouped_matmul(a, w, off, out=short[512:1024].view(32, 16)) == 16).all()
    # columns of one array beside one another do not overlap
    both = torch.ones(32, 32, dtype=BF, device="cuda")
    assert (rt.grouped_matmul(both[:, :16], w, off, out=both[:, 16:]) == 16).all() and (both[:, :16] == 1).all()


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,stream", TYPES)
@pytest.mark.parametrize("rows,cols", [(4001, 257), (3001, 1023), (2500, 1024), (1301, 2047), (700, 4096), (400, 8192), (200, 16383)])
def test_norm_of_many_rows(rows, cols, dtype, stream):
    """More rows than teams of warps, so that each team takes several, through rings in shared memory: one warp a row and
    several, one to four units of columns a warp, two and three arrays, aligned rows and others, groups that end anywhere.
    The forward pass by test_train_norm's tolerance, the backward pass by check_back's."""
    for p, pad, shift, more in ((0.1, 0, 0, True), (0.0, 5, 1, False), (0.3, 3, 1, True)):
        x, residual, weight, bias, gen = norm_case(rows, cols, dtype, stream, rows + cols, pad, shift)
        if not more:
            residual = None
        if more or stream == dtype:
            check_norm(x, residual, weight, bias, p, 99)
        h = (residual if more else rows_made(rows, cols, stream, gen, pad, shift))
        dy, dh = rows_made(rows, cols, dtype, gen, pad, shift), rows_made(rows, cols, stream, gen, pad, shift)
        _, _, mean, rstd = rt.layer_norm(h, weight, bias)
        cut = sorted(int(i) for i in torch.randint(0, rows + 1, (4,), generator=gen))
        check_back(dy, h, mean, rstd, weight, dh if more else None, [0, *cut, cut[-1], rows], p)
    rt.training_status()


MOST = 2**31 - 2**20  # rows, k and m of a product


def test_c_largest_sizes():
    """What is worked out in 32 bits from rows, k and m stays below 2^31; larger ones are refused before anything is launched."""
    lib, p = ref.c_library(), 4096
    for rows, k, m in ((MOST + 1, 8, 8), (8, MOST + 1, 8), (8, 8, MOST + 1), (2**31 - 256, 8, 8)):
        assert lib.regtopk_grouped_matmul(p, k, p, k, 0, 0, 1, p, m, p, 1, rows, k, m, 1, None, 0, None) == -1
        assert lib.regtopk_grouped_matmul_dw(p, m, p, k, p, k, 0, 0, 1, 0, p, 1, rows, k, m, 1, None, 0, None) == -1
        assert lib.regtopk_grouped_matmul_workspace_bytes(p, k + 1, p, k, 0, 0, 1, 1, rows, k, m) == 0


@pytest.mark.gpu
def test_largest_sizes():
    """The most rows and the longest sum, of values whose sums are exact however they are grouped."""
    x = torch.ones(MOST, 8, dtype=BF, device="cuda")
    off = torch.tensor([0, MOST], device="cuda")
    dw = rt.grouped_matmul_dw(x, x, off)
    assert (dw == float(MOST)).all()
    dw = rt.grouped_matmul_dw(x, x, torch.tensor([0, MOST - 1024, MOST - 1], device="cuda"))
    assert (dw[0] == float(MOST - 1024)).all() and (dw[1] == 1023).all()
    w = torch.eye(8, dtype=BF, device="cuda")[None]
    w[:, 7, 7] = 2.0
    y = rt.grouped_matmul(x, w, off)
    top = torch.tensor([1.0] * 7 + [2.0], device="cuda")
    assert torch.equal(y.amin(0).float(), top) and torch.equal(y.amax(0).float(), top)
    del x, y
    x, w = (torch.full((1, MOST), v, dtype=HF, device="cuda") for v in (2.0**-10, 2.0**-21))
    assert rt.grouped_matmul(x, w[None], torch.tensor([0, 1], device="cuda")).item() == 1 - 2.0**-11
    rt.training_status()


@pytest.mark.gpu
def test_captured_graph():
    """A whole step recorded as a CUDA graph and replayed on other inputs gives the bits of the calls themselves: every launch may
    start while the one before it ends, and unaligned operands, divided sums and joins are among them."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    rows, cols, m = 900, 257, 90
    w, b = torch.randn(cols, generator=gen, device="cuda"), torch.randn(cols, generator=gen, device="cuda")
    experts = (torch.randn(2, m, cols, generator=gen, device="cuda") / 16).to(BF)
    off, one = torch.tensor([0, 100, 500, 620, rows], device="cuda"), torch.tensor([0, rows], device="cuda")
    x, residual = torch.zeros(rows, cols, dtype=BF, device="cuda"), torch.zeros(rows, cols, device="cuda")
    rows_out = torch.zeros(2, 2 * m * cols + 3, device="cuda")

    def step():
        y, h, mean, rstd = rt.layer_norm(rt.dropout(x, 0.1, 3), w, b, residual=residual, p=0.2, seed=5, subsequence=1)
        o = rt.grouped_matmul(y, experts, off)
        dy = rt.grouped_matmul(o, experts.transpose(1, 2), off)
        rt.grouped_matmul_dw(o, y, off, out=rows_out[:, 3:].view(2, 2, m, cols), accumulate=True)
        whole = rt.grouped_matmul_dw(o, y, one)
        return [y, h, mean, rstd, o, dy, whole, *rt.layer_norm_backward(dy, h, mean, rstd, w, dh=h, p=0.2, seed=5, subsequence=1, offsets=off)]

    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step()
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        kept = step()
    for _ in range(3):
        x.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
        residual.copy_(torch.randn(rows, cols, generator=gen, device="cuda"))
        rows_out.zero_()
        graph.replay()
        got = [t.clone() for t in kept] + [rows_out.clone()]
        rows_out.zero_()
        want = step() + [rows_out]
        assert all(torch.equal(a, c) for a, c in zip(got, want))
    rt.training_status()
