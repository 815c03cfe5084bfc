"""The tokens' way into the sorted order and back, against the definitions in 64 bits.

Tolerances.  Spreading is exact.  A token's sum has at most 33 terms, fused products added one after the other: 34 * 2^-24 of the
sum of magnitudes, and a rounding.  The gradient to a weight is a sum over the columns in chains of at most 4 * 64 + 1 + 5 + 8 additions
at the widths here: 2^-16 of the sum of magnitudes.  The gradient to a row is one product."""
import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import experts_reference as ref
from tests.test_train_norm import made
from tests.train_reference import assert_close, host

BF, HF, F = torch.bfloat16, torch.float16, torch.float32


def test_c_entries_refuse():
    """Bad arguments come back as codes before anything is launched (the pointers here are never followed)."""
    lib, p = ref.c_library(), 4096

    def spread(x=p, ldx=64, s=None, lds=2, place=p, filled=p, out=p, ldo=64, tokens=4, k=2, rows=8, cols=64, type=1):
        return lib.regtopk_spread_tokens(x, ldx, s, lds, place, filled, out, ldo, tokens, k, rows, cols, type, None)
    for bad in (dict(type=3), dict(x=None), dict(x=p + 1), dict(ldx=63), dict(s=p, lds=1), dict(place=None), dict(place=p + 2), dict(filled=p + 4), dict(out=None),
                dict(ldo=63), dict(tokens=-1), dict(k=0), dict(rows=-1), dict(cols=-1), dict(cols=2**30 + 1)):
        assert spread(**bad) == -1, bad
    assert spread(k=33) == -7 and spread(rows=0) == 0 and spread(cols=0) == 0

    def join(src=p, ld=64, place=p, w=p, res=None, ldr=64, out=p, ldo=64, tokens=4, k=2, rows=8, type=1, out_type=1):
        return lib.regtopk_join_tokens(src, ld, place, w, res, ldr, out, ldo, tokens, k, rows, 64, type, out_type, None)
    for bad in (dict(src=None), dict(ld=63), dict(place=None), dict(w=p + 2), dict(res=p, ldr=63), dict(out=None), dict(ldo=63), dict(out_type=2), dict(type=0),
                dict(tokens=-1), dict(k=0), dict(rows=-1)):
        assert join(**bad) == -1, bad
    assert join(k=33) == -7 and join(tokens=0) == 0

    def back(dout=p, ldd=64, src=p, ld=64, place=p, w=p, filled=p, out=p, ldo=64, dw=p, tokens=4, k=2, rows=8, type=1, dtype=0):
        return lib.regtopk_join_tokens_backward(dout, ldd, src, ld, place, w, filled, out, ldo, dw, tokens, k, rows, 64, type, dtype, None)
    for bad in (dict(dout=None), dict(ldd=63), dict(src=None), dict(ld=63), dict(place=None), dict(w=None), dict(filled=p + 4), dict(out=None), dict(ldo=63),
                dict(dw=None), dict(dw=p + 2), dict(dtype=2), dict(tokens=-1), dict(k=0)):
        assert back(**bad) == -1, bad
    assert back(k=33) == -7 and back(tokens=0, rows=0) == 0


CASES = [(1, 1, 1, 1), (3, 2, 4, 7), (17, 3, 8, 40), (40, 4, 5, 257), (9, 8, 16, 1032), (64, 2, 8, 777), (5, 20, 24, 96), (3, 32, 32, 33), (6, 5, 6, 4096), (700, 2, 8, 64)]


def plan(tokens, k, n, gen):
    """Distinct experts a token, some of them none; two workers, and tokens of no worker."""
    experts = torch.rand(tokens, n, generator=gen).argsort(1)[:, :k].to(torch.int32)
    experts[torch.rand(tokens, k, generator=gen) < 0.15] = -1
    at = torch.tensor([0, tokens // 2, tokens if tokens < 9 else tokens - 2])
    return rt.sort_tokens(experts.cuda(), n, at.cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("tokens,k,n,cols", CASES)
def test_spread(tokens, k, n, cols, dtype):
    gen = torch.Generator().manual_seed(tokens + cols)
    offsets, place = plan(tokens, k, n, gen)
    for pad, shift in ((0, 0), (8, 8), (3, 1)):
        x = made(tokens, cols, dtype, gen, pad, shift)
        x[0, 0] = float("nan")
        torch.empty(tokens * k * cols, dtype=dtype, device="cuda").fill_(7)  # what the allocator may hand out
        got = rt.spread_tokens(x, place, offsets)
        want = ref.spread(host(x), place.cpu().numpy(), tokens * k)
        assert got.dtype == dtype and np.array_equal(host(got), want, equal_nan=True)
    rows8 = rt.pack8(x.nan_to_num(0.5))
    want = ref.spread(ref.unpacked(rows8), place.cpu().numpy(), tokens * k)
    for to in (BF, F):
        assert np.array_equal(host(rt.spread_tokens(rows8, place, offsets, dtype=to)), want)
    assert rt.spread_tokens(rows8, place, offsets).dtype == BF


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("tokens,k,n,cols", CASES)
def test_join_and_gradient(tokens, k, n, cols, dtype):
    gen = torch.Generator().manual_seed(tokens * 3 + cols)
    offsets, place = plan(tokens, k, n, gen)
    where = place.cpu().numpy()
    w = torch.randn(tokens, k, generator=gen).cuda()
    w[place < 0] = float("nan")  # of no consequence
    wh = np.where(where >= 0, host(w), 0.0)
    for pad, shift in ((0, 0), (8, 8), (3, 1)):
        rows = made(tokens * k, cols, dtype, gen, pad, shift)
        rows[int(offsets[-1]):] = float("inf")  # rows of no group, which nothing may look at
        fine = np.where(np.isfinite(host(rows)), host(rows), 0.0)
        for res in (None, dtype, F):
            residual = None if res is None else made(tokens, cols, res, gen, pad, shift)
            got = rt.join_tokens(rows, place, w, residual)
            assert got.dtype == (res or dtype) and got.shape == (tokens, cols)
            size = ref.join(np.abs(fine), where, np.abs(wh), None if residual is None else np.abs(host(residual)))
            assert_close(got, ref.join(fine, where, wh, None if residual is None else host(residual)), 34 * 2.0 ** -24 * size, got.dtype, res)
        assert_close(rt.join_tokens(rows, place), ref.join(fine, where, None, None), 34 * 2.0 ** -24 * ref.join(np.abs(fine), where, None, None), dtype, "plain")
        for of in {dtype, F}:
            dout = made(tokens, cols, of, gen, pad, shift)
            drows, dw = rt.join_tokens_backward(dout, rows, place, w, offsets)
            d = host(dout)
            want = np.zeros((tokens * k, cols))
            t, j = np.nonzero(where >= 0)
            want[where[t, j]] = wh[t, j][:, None] * d[t]
            assert drows.dtype == dtype
            assert_close(drows, want, 2.0 ** -24 * np.abs(want), dtype, "drows")
            sums, size = np.zeros((tokens, k)), np.zeros((tokens, k))
            sums[t, j] = (d[t] * fine[where[t, j]]).sum(1)
            size[t, j] = np.abs(d[t] * fine[where[t, j]]).sum(1)
            assert_close(dw, sums, 2.0 ** -16 * size, F, "dweights")


@pytest.mark.gpu
def test_gradients_against_differences():
    """The whole way, spread to join, by central differences of its own outputs in float32 (a linear map in x, rows and w each)."""
    gen = torch.Generator().manual_seed(3)
    offsets, place = plan(20, 3, 6, gen)
    x, w, v = (torch.randn(*s, generator=gen).cuda() for s in ((20, 16), (20, 3), (20, 16)))
    rows = rt.spread_tokens(x, place, offsets)
    drows, dw = rt.join_tokens_backward(v, rows, place, w, offsets)
    dx = rt.join_tokens(drows, place)
    for leaf, grad in ((x, dx), (w, dw)):
        step = torch.randn(leaf.shape, generator=gen).cuda()
        ends = []
        for s in (0.5, -0.5):
            xs, ws = (x + s * step, w) if leaf is x else (x, w + s * step)
            ends.append((rt.join_tokens(rt.spread_tokens(xs, place, offsets), place, ws).double() * v).sum())
        want = (grad.double() * step).sum()
        assert abs(ends[0] - ends[1] - want) < 2.0 ** -16 * (grad.double() * step).abs().sum()


@pytest.mark.gpu
def test_places_out_of_range():
    """A place that is no row is none, and nothing is touched for it."""
    x, rows = torch.randn(3, 24, device="cuda"), torch.randn(6, 24, device="cuda")
    place = torch.tensor([[0, 6], [-7, 2**31 - 1], [3, -2**31]], dtype=torch.int32, device="cuda")
    for filled in (4, 99):
        out = rt.spread_tokens(x, place, torch.tensor([0, filled], device="cuda"))
        assert torch.equal(out[0], x[0]) and torch.equal(out[3], x[2]) and (filled == 99 or not out[4:].any())
    assert not rt.spread_tokens(x, torch.full_like(place, -1), torch.tensor([0, -3], device="cuda")).any()
    w = torch.ones(3, 2, device="cuda")
    assert torch.equal(rt.join_tokens(rows, place, w), torch.stack([rows[0], torch.zeros(24, device="cuda"), rows[3]]))
    _, dw = rt.join_tokens_backward(x, rows, place, w, torch.tensor([0, 4], device="cuda"))
    assert (dw[:, 1] == 0).all() and dw[1, 0] == 0


@pytest.mark.gpu
def test_shapes_and_refusals():
    x = torch.randn(2, 3, 16, device="cuda", dtype=BF)
    experts = torch.randint(0, 4, (2, 3, 2), dtype=torch.int32, device="cuda")
    offsets, place = rt.sort_tokens(experts, 4)
    rows = rt.spread_tokens(x, place, offsets)
    w = torch.rand(2, 3, 2, device="cuda")
    assert rows.shape == (12, 16) and rt.join_tokens(rows, place).shape == (2, 3, 16) and rt.join_tokens(rows, place, w, residual=x.float().view(6, 16)).shape == (6, 16)
    drows, dw = rt.join_tokens_backward(x, rows, place, w, offsets)
    assert dw.shape == w.shape and drows.shape == rows.shape
    for call in (lambda: rt.spread_tokens(x, place.long(), offsets), lambda: rt.spread_tokens(x, place[:1].contiguous(), offsets), lambda: rt.spread_tokens(x, place, offsets.int()),
                 lambda: rt.spread_tokens(x, place, offsets, dtype=F), lambda: rt.spread_tokens(x.cpu(), place, offsets), lambda: rt.spread_tokens(x, place.cpu(), offsets),
                 lambda: rt.join_tokens(rows.double(), place), lambda: rt.join_tokens(rows, place, w.to(BF)), lambda: rt.join_tokens(rows, place, w[:1].contiguous()),
                 lambda: rt.join_tokens(rows, place, residual=x.half()), lambda: rt.join_tokens(rows, place, residual=x[:1]),
                 lambda: rt.join_tokens_backward(x.half(), rows, place, w, offsets), lambda: rt.join_tokens_backward(x[:1], rows, place, w, offsets),
                 lambda: rt.join_tokens_backward(x, rows, place, w[..., :1].contiguous(), offsets)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: rt.spread_tokens(x.transpose(1, 2), place, offsets), lambda: rt.join_tokens(rows.view(3, 4, 16), place), lambda: rt.join_tokens(rows.t(), place)):
        with pytest.raises(ValueError):
            call()
    many = torch.zeros(6, 33, dtype=torch.int32, device="cuda")
    with pytest.raises(rt.RegTopKError):
        rt.spread_tokens(x, many, offsets)
    none = torch.zeros(0, 2, dtype=torch.int32, device="cuda")
    offsets, place = rt.sort_tokens(none, 4)
    assert offsets.tolist() == [0] * 5 and rt.spread_tokens(x.view(6, 16)[:0], place, offsets).shape == (0, 16)
    assert rt.join_tokens(rows[:0], place, w.view(6, 2)[:0]).shape == (0, 16)
    assert rt.join_tokens(rows[:0], torch.full((4, 2), -1, dtype=torch.int32, device="cuda")).eq(0).all()


@pytest.mark.gpu
def test_rows_past_32_bits():
    """More than 2^34 elements, which is more than one launch takes."""
    tokens, cols = 2**21 + 5, 8192
    if torch.cuda.mem_get_info()[0] < 80 << 30:
        pytest.skip("needs 80 GB")
    x = torch.zeros(tokens, cols, dtype=BF, device="cuda")
    at = [0, 2**18, 2**19 + 1, 2**20, 2**21 - 1, 2**21, tokens - 1]
    x[at] = torch.randn(len(at), cols, generator=torch.Generator().manual_seed(4)).to(BF).cuda()
    place = torch.arange(tokens - 1, -1, -1, dtype=torch.int32, device="cuda").view(-1, 1)  # the other way round
    place[5] = -1
    rows = rt.spread_tokens(x, place, torch.tensor([0, tokens - 1], device="cuda"))
    for t in at:
        assert torch.equal(rows[tokens - 1 - t], x[t] if t != 0 else torch.zeros_like(x[0])), t  # the last row lies behind the last group
    small = x[at[1:]].clone()
    del x
    torch.cuda.empty_cache()
    back = rt.join_tokens(rows, place)
    assert torch.equal(back[at[1:]], small)
    del rows, back
    torch.cuda.empty_cache()
