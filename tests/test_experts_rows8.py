"""8-bit rows, and the activations that keep their input as such, against the definitions in 64 bits.

Tolerances.  8-bit rows and what they stand for are exact.  Let u = 2^-24.  An exponential here is off by 2^-21.5 relative
(the hardware's, in binary32 CUDA's, which is closer) and by the rounding of its argument, |z| u, z at most 64 where it is above
2^-93; a quotient and three products add 6u: p = f(x) / x is off by 2^-17 relative.  gelu takes p for 16-bit types from a formula
that is off by 7.5e-8 (Abramowitz and Stegun 7.1.26) and 16 u more: 2^-22 in all; in binary32 by a fit that is off
by 1.2e-7 relative and exp(-x^2 / 2), whose argument is rounded: x^2 / 2 u, 2^-18 for x up to 11.  The slope is p + x p'(x), each term off by as much relative to itself.
Results follow by products of one more rounding each, and are rounded once to the type.  Below 2^-120 binary32 may give 0."""
import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import experts_reference as ref
from tests.test_train_norm import made
from tests.train_reference import assert_close, host

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
E4, E8 = torch.float8_e4m3fn, torch.float8_e8m0fnu


# ---- without a GPU -----------------------------------------------------------------------------------------------------
def test_table_of_numbers():
    codes = torch.arange(127, dtype=torch.uint8).view(E4).float().numpy()
    assert np.array_equal(codes, ref.E4M3)
    x = torch.linspace(-448, 448, 40001)
    assert np.array_equal(ref.nearest_e4m3(x.double().numpy()), x.to(E4).double().numpy())


def test_scale_bytes():
    x = np.array([[448.0], [448.0 * (1 + 2 ** -20)], [1.75], [1.7500001], [0.0], [2.0 ** -126], [2.0 ** -149], [3e38], [np.inf]])
    assert ref.scale_bytes(x)[:, 0].tolist() == [127, 128, 119, 120, 0, 0, 0, 247, 0]


def test_reference_slopes_against_differences():
    x = np.linspace(-9, 9, 301)[None]
    for kind in ("silu", "gelu", "gelu_tanh"):
        ends = [ref.activation(x + s, kind, False)[0] for s in (1e-6, -1e-6)]
        assert np.abs((ends[0] - ends[1]) / 2e-6 - ref.activation(x, kind, False)[2]).max() < 1e-8


def test_c_entries_refuse():
    """Bad arguments come back as codes before anything is launched (the pointers here are never followed)."""
    lib, p = ref.c_library(), 4096

    def pack(x=p, ldx=64, v=p, ldv=64, s=p, lds=2, rows=4, cols=64, type=1):
        return lib.regtopk_pack8(x, ldx, v, ldv, s, lds, rows, cols, type, None)
    for bad in (dict(type=3), dict(x=None), dict(x=p + 1), dict(ldx=63), dict(v=None), dict(ldv=63), dict(s=None), dict(lds=1), dict(rows=-1),
                dict(cols=-1), dict(cols=2**30 + 1)):
        assert pack(**bad) == -1, bad
        assert lib.regtopk_unpack8(*[{**dict(x=p, ldx=64, v=p, ldv=64, s=p, lds=2, rows=4, cols=64, type=1), **bad}[i] for i in
                                     ("v", "ldv", "s", "lds", "x", "ldx", "rows", "cols", "type")], None) == -1, bad
    assert pack(rows=0) == 0 and pack(cols=0) == 0

    def act(lda=128, ldy=64, v=None, ldv=128, s=None, lds=4, rows=4, cols=64, kind=0, gated=1, type=0):
        return lib.regtopk_activation(p, lda, p, ldy, v, ldv, s, lds, rows, cols, kind, gated, type, None)
    for bad in (dict(lda=127), dict(ldy=63), dict(v=p), dict(s=p), dict(v=p, s=p, ldv=127), dict(v=p, s=p, lds=3), dict(kind=3), dict(kind=-1), dict(type=4)):
        assert act(**bad) == -1, bad
    assert act(rows=0) == 0 and act(cols=0) == 0

    def back(ldd=64, lda=128, s=None, lds=4, ldda=128, y=None, ldy=64, kind=0, type=0):
        return lib.regtopk_activation_backward(p, ldd, p, lda, s, lds, p, ldda, y, ldy, 4, 64, kind, 1, type, None)
    for bad in (dict(ldd=63), dict(lda=127), dict(s=p, lds=3), dict(ldda=127), dict(y=p, ldy=63), dict(kind=7), dict(type=-1)):
        assert back(**bad) == -1, bad


def test_no_cpu_path():
    x = torch.zeros(4, 8)
    for call in (lambda: rt.pack8(x), lambda: rt.activation(x), lambda: rt.activation_backward(x, x),
                 lambda: rt.unpack8(rt.Rows8(x.to(E4), torch.zeros(4, 1, dtype=torch.uint8).view(E8)))):
        with pytest.raises(TypeError):
            call()


# ---- on the GPU ----------------------------------------------------------------------------------------------------------
SIZES = [(1, 1), (3, 7), (1, 32), (5, 40), (2, 33), (17, 257), (4, 1000), (3, 2304), (130, 96), (2, 8200)]


def hard_rows(rows, cols, dtype, gen, pad=0, shift=0):
    """Numbers of every size, halfway cases and limits of blocks among them."""
    x = made(rows, cols, dtype, gen, pad, shift)
    x *= torch.exp2(torch.randint(-12, 9, (rows, cols), generator=gen).float()).to(dtype).cuda()
    flat = torch.tensor([448.0, 449.0, 1.75, 1.7578125, 0.0, -0.0, 17.0, 19.0, 2.0 ** -14, -3 * 2.0 ** -15, 240.0, 248.0])
    n = min(cols, len(flat))
    x[0, :n] = flat[:n].to(dtype).cuda()
    x[-1, cols // 2:] = 0
    return x


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("rows,cols", SIZES)
def test_pack_and_unpack(rows, cols, dtype):
    gen = torch.Generator().manual_seed(rows * 131 + cols)
    for pad, shift in ((0, 0), (8, 8), (3, 1)):
        x = hard_rows(rows, cols, dtype, gen, pad, shift)
        want, byte = ref.packed(host(x))
        got = rt.pack8(x)
        assert got.values.shape == x.shape and got.values.dtype == E4 and got.scales.dtype == E8 and got.scales.shape == (rows, (cols + 31) // 32)
        assert np.array_equal(got.scales.cpu().view(torch.uint8).numpy(), byte)
        assert np.array_equal(ref.unpacked(got), want)
        for to in (BF, F):  # exact in both
            back = rt.unpack8(got, to)
            assert back.dtype == to and np.array_equal(host(back), want)
        wide = torch.zeros(rows, cols + 5, dtype=torch.uint8, device="cuda").view(E4)
        wide[:, 3:3 + cols].view(torch.uint8).copy_(got.values.view(torch.uint8))
        assert np.array_equal(host(rt.unpack8(rt.Rows8(wide[:, 3:3 + cols], got.scales))), want)
    three = x.new_zeros(rows, 2, cols).copy_(x.unsqueeze(1))
    assert torch.equal(rt.pack8(three).values[:, 1].view(torch.uint8), got.values.view(torch.uint8))


@pytest.mark.gpu
@pytest.mark.parametrize("cols", [64, 61])
def test_pack_what_is_not_finite(cols):
    """Infinities and NaN become NaN and leave the others of their block alone; the smallest and largest numbers."""
    x = torch.randn(6, cols, generator=torch.Generator().manual_seed(1)).cuda()
    x[0, 3], x[0, 40], x[1, 5], x[2] = float("inf"), -float("inf"), float("nan"), float("inf")
    x[3] *= 2.0 ** -126
    x[4] *= 2.0 ** 126
    x[5] *= 2.0 ** -149
    want, byte = ref.packed(host(x))
    got = rt.pack8(x)
    assert np.array_equal(got.scales.cpu().view(torch.uint8).numpy(), byte)
    assert np.array_equal(ref.unpacked(got), want, equal_nan=True)
    assert np.array_equal(host(rt.unpack8(got, F)), want, equal_nan=True)
    bad = rt.Rows8(got.values, torch.full_like(got.scales.view(torch.uint8), 255).view(E8))
    assert rt.unpack8(bad, F).isnan().all()


@pytest.mark.gpu
def test_empty():
    for shape in ((0, 8), (4, 0)):
        x = torch.zeros(shape, device="cuda")
        assert rt.unpack8(rt.pack8(x), F).shape == shape
        y, kept = rt.activation(x, keep8=True)
        assert y.shape == shape and rt.activation_backward(y, kept, want_y=True)[0].shape == shape


def slacks(x, kind, dtype):
    """How far p and the slope may be off."""
    z, f, slope = x, *ref.activation(x, kind, False)[1:]
    with np.errstate(all="ignore"):
        p = np.where(x == 0, 0.5, f / np.where(x == 0, 1.0, x))
    absolute = 2.0 ** -22 if kind == "gelu" and dtype != F else 0.0
    return 2.0 ** -17 * p + absolute, 2.0 ** -17 * (p + np.abs(slope - p)) + absolute


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
@pytest.mark.parametrize("gated", [False, True])
def test_activation(kind, gated, dtype):
    gen = torch.Generator().manual_seed(len(kind) + gated)
    for rows, cols, pad, shift in ((1, 1, 0, 0), (3, 7, 0, 0), (5, 40, 8, 8), (9, 257, 3, 1), (70, 1024, 0, 0), (2, 8200, 16, 0)):
        halves = 2 if gated else 1
        a = made(rows, halves * cols, dtype, gen, pad, shift, scale=2.5)
        edges = torch.tensor([0.0, -0.0, 9.0, -9.0, 40.0, -40.0, -1.2785, 1e-6, -1e-6, 1000.0, -1000.0]).to(dtype).cuda()
        a[0, :min(cols, 11)] = edges[:min(cols, 11)]
        dy = made(rows, cols, dtype, gen, pad, shift)
        up = host(a)[:, cols:] if gated else 1.0

        def check(got_y, got_da, at):
            x, u = at[:, :cols], at[:, cols:] if gated else np.ones((rows, cols))
            y, f, slope = ref.activation(at, kind, gated)
            da, _ = ref.activation_backward(host(dy), at, kind, gated)
            sp, ss = slacks(x, kind, dtype)
            d, tiny = np.abs(host(dy)), 2.0 ** -120
            assert_close(got_y, y, sp * np.abs(x * u) + tiny * (1 + np.abs(u)), dtype, "y")
            if got_da is not None:
                slack = ss * d * np.abs(u)
                if gated:
                    slack = np.concatenate([slack, sp * np.abs(x) * d], 1)
                assert_close(got_da, da, slack + tiny * (1 + np.abs(da)), dtype, "da")

        y, kept = rt.activation(a, kind, gated=gated)
        assert kept is a and y.dtype == dtype
        check(y, None, host(a))
        da, again = rt.activation_backward(dy, kept, kind, gated=gated, want_y=True)
        check(again, da, host(a))
        y8, kept = rt.activation(a, kind, gated=gated, keep8=True)
        assert torch.equal(y8, y)
        want, byte = ref.packed(host(a), halves)
        assert np.array_equal(kept.scales.cpu().view(torch.uint8).numpy(), byte) and np.array_equal(ref.unpacked(kept, halves), want)
        da, again = rt.activation_backward(dy, kept, kind, gated=gated, want_y=True)
        check(again, da, want)
        alone, none = rt.activation_backward(dy, kept, kind, gated=gated)
        assert none is None and torch.equal(alone, da)


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_activation_of_large_numbers(kind):
    """Far out f(x) is x or 0, and its slope 1 or 0, whatever overflows on the way; NaN stays NaN."""
    x = torch.tensor([[1e20, -1e20, 3e38, -3e38, float("nan"), 200.0, -200.0, 0.0]], device="cuda")
    one = torch.ones_like(x)
    for dtype in (F, BF):
        y, _ = rt.activation(x.to(dtype), kind)
        da, _ = rt.activation_backward(one.to(dtype), x.to(dtype), kind)
        assert torch.equal(y[0, [0, 2, 5, 7]], x.to(dtype)[0, [0, 2, 5, 7]]) and (y[0, [1, 3, 6]] == 0).all() and y[0, 4].isnan()
        assert da[0].tolist()[:4] == [1, 0, 1, 0] and da[0, 4].isnan() and da[0].tolist()[5:] == [1, 0, 0.5]


@pytest.mark.gpu
def test_halves_are_rows_of_their_own():
    a = torch.randn(6, 2 * 40, generator=torch.Generator().manual_seed(3)).cuda()
    _, kept = rt.activation(a, gated=True, keep8=True)
    for half in (0, 1):
        own = rt.pack8(a[:, half * 40:half * 40 + 40].contiguous())
        assert torch.equal(kept.values.view(torch.uint8)[:, half * 40:half * 40 + 40], own.values.view(torch.uint8))
        assert torch.equal(kept.scales.view(torch.uint8)[:, half * 2:half * 2 + 2], own.scales.view(torch.uint8))
        assert torch.equal(rt.unpack8(rt.Rows8(kept.values.unflatten(-1, (2, 40)), kept.scales.unflatten(-1, (2, 2))))[:, half], rt.unpack8(own))


@pytest.mark.gpu
def test_refusals():
    x = torch.zeros(4, 64, device="cuda", dtype=BF)
    r = rt.pack8(x)
    for call in (lambda: rt.pack8(x.double()), lambda: rt.unpack8(r, torch.float64), lambda: rt.unpack8(x), lambda: rt.unpack8((r.values, r.scales, x)),
                 lambda: rt.unpack8(rt.Rows8(x, r.scales)), lambda: rt.unpack8(rt.Rows8(r.values, r.values)),
                 lambda: rt.unpack8(rt.Rows8(r.values, r.scales[:, :1])), lambda: rt.unpack8(rt.Rows8(r.values, r.scales[:3])),
                 lambda: rt.activation_backward(x, x.float()), lambda: rt.activation_backward(x, x[:2]), lambda: rt.activation_backward(x, x, gated=True),
                 lambda: rt.activation_backward(x, r, gated=True), lambda: rt.activation_backward(x.cpu(), x), lambda: rt.activation_backward(x, x.cpu())):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: rt.pack8(x.t()), lambda: rt.pack8(x[:1].expand(4, 64)), lambda: rt.pack8(torch.zeros((), device="cuda")), lambda: rt.activation(x, "relu"),
                 lambda: rt.activation(x, None), lambda: rt.activation(x[:, :63], gated=True), lambda: rt.activation_backward(x, x, "tanh")):
        with pytest.raises(ValueError):
            call()


@pytest.mark.gpu
def test_rows_past_32_bits():
    """More than 2^34 elements, which is more than one launch takes: rows before, around and behind the places where 32 bits end."""
    rows, cols = 2**21 + 5, 8192
    if torch.cuda.mem_get_info()[0] < 60 << 30:
        pytest.skip("needs 60 GB")
    x = torch.zeros(rows, cols, dtype=BF, device="cuda")
    at = [0, 1, 2**18 - 1, 2**18, 2**19, 2**20, 2**21 - 2, 2**21 - 1, 2**21, rows - 1]
    x[at] = torch.randn(len(at), cols, generator=torch.Generator().manual_seed(4)).to(BF).cuda()
    small = rt.pack8(x[at])
    got = rt.pack8(x)
    assert torch.equal(got.values.view(torch.uint8)[at], small.values.view(torch.uint8)) and torch.equal(got.scales.view(torch.uint8)[at], small.scales.view(torch.uint8))
    rt.training_status()
    del x
    torch.cuda.empty_cache()
    assert torch.equal(rt.unpack8(got)[at], rt.unpack8(small))
    del got
    torch.cuda.empty_cache()
