"""Calls of the operators around an expert sublayer at the ends of what they allow, against the definitions in 64 bits."""
import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import experts_reference as ref
from tests import test_experts_norm as norm
from tests.test_experts_route import check_route

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
INF = float("inf")


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("groups,kept", [(4, 1), (8, 3), (8, 2), (16, 16)])
def test_groups_with_numbers_that_are_not_finite(groups, kept, scores, dtype):
    """A group whose scores are NaN comes last, but before one that is masked; +inf among the logits makes all softmax scores NaN."""
    experts, size = 64, 64 // groups
    logits = torch.randn(13, experts, generator=torch.Generator().manual_seed(8)).to(dtype)
    logits[:5, :size] = -INF  # the first group is masked
    logits[0, size * 2], logits[1, size * 2] = float("nan"), INF
    logits[2, size:] = float("nan")
    logits[3, size + 1::2] = float("nan")
    logits[4, size:size * 2] = float("nan")
    logits[5, 9], logits[6, 9] = float("nan"), INF
    logits[7, ::2] = float("nan")
    logits[8, ::3] = INF
    logits[9], logits[10] = INF, float("nan")
    logits[11, 5:40] = float("nan")
    for bias in (None, torch.linspace(-1, 1, experts).cuda()):
        for top in (1, 2):
            for renormalise in (True, False):
                e, w = check_route(logits.cuda(), min(4, kept * size), scores=scores, bias=bias, groups=groups, groups_kept=kept, group_top=top,
                                   renormalise=renormalise)
                assert (e >= 0).all(), "a masked group was kept before one with NaN"


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F])
def test_scores_below_the_range(dtype):
    """An exponential of less than -708 is 0, so that its experts are equal, and the lower one comes first; above they are told apart."""
    logits = torch.tensor([[0.0, -800.0, -740.0, -20000.0], [0.0, -704.0, -680.0, -720.0], [-740.0, -800.0, -20000.0, 0.0]]).to(dtype).cuda()
    for scores in ("softmax", "sigmoid"):
        e, _ = rt.route(logits, 4, scores=scores, bias=torch.zeros(4, device="cuda"))
        assert e.tolist() == [[0, 1, 2, 3], [0, 2, 1, 3], [3, 0, 1, 2]]
        e, _ = rt.route(logits, 4, scores=scores)  # by the logits
        assert e.tolist() == [[0, 2, 1, 3], [0, 2, 1, 3], [3, 0, 1, 2]]


def hard_tokens(tokens, experts, dtype, gen):
    """Every seventh token is one that the choice has to take care with: ties, neighbours, masks, numbers that are not finite."""
    logits = (1.5 * torch.randn(tokens, experts, generator=gen)).to(dtype)
    at = torch.arange(0, tokens, 7)
    for kind in range(8):
        t = at[kind::8]
        if kind == 0:
            logits[t] = (torch.randint(-3, 3, (len(t), experts), generator=gen) / 4).to(dtype)
        elif kind == 1:
            logits[t] = (logits[t].float().round() + torch.randint(0, 9, (len(t), experts), generator=gen) * 2.0 ** -22).to(dtype)
        elif kind == 2:
            logits[t, : experts // 2] = -INF
        elif kind == 3:
            logits[t] = -INF
        elif kind == 4:
            logits[t, 1:] = -INF
        elif kind == 5:
            logits[t] = torch.finfo(dtype).min
        else:
            logits[t, torch.randint(0, experts, (len(t),), generator=gen)] = float("nan") if kind == 6 else INF
    return logits, at


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("experts,k,groups,kept,top", [(256, 8, 8, 4, 2), (256, 1, 1, 1, 1), (60, 2, 1, 1, 1), (8, 2, 1, 1, 1), (128, 32, 4, 2, 1), (512, 8, 1, 1, 1),
                                                       (510, 4, 17, 5, 2), (96, 5, 3, 2, 2)])
def test_route_of_many_tokens_a_warp(experts, k, groups, kept, top, dtype):
    """Eleven tokens for every warp that the device holds, which takes up to eight at a time and has three left; the last warp has fewer.  Equal to calls of
    few tokens, where a warp has one, and to the definition."""
    gen = torch.Generator().manual_seed(experts + k)
    each = experts // groups  # a group's experts, of which a lane has `in_lane`
    lanes = 32 >> max(0, (groups - 1).bit_length())
    in_lane = -(-each // lanes)
    warps = torch.cuda.get_device_properties(0).multi_processor_count * 8 * (4 if in_lane <= 8 else 2)
    tokens = 11 * warps - 5
    logits, at = hard_tokens(tokens, experts, dtype, gen)
    bias = (0.1 * torch.randn(experts, generator=gen)).cuda()
    seen = torch.cat([at[torch.randperm(len(at), generator=gen)[:150]], torch.randint(0, tokens, (50,), generator=gen), torch.arange(tokens - 12, tokens)])
    logits = logits.cuda()
    for scores, b, renormalise in (("sigmoid", bias, True), ("softmax", bias, False), ("softmax", None, True), ("softmax", None, False), ("sigmoid", None, False)):
        a = dict(scores=scores, bias=b, groups=groups, groups_kept=kept, group_top=top, renormalise=renormalise, scale=2.5)
        experts_of, weights = rt.route(logits, k, **a)
        for first in range(0, tokens, warps):
            e, w = rt.route(logits[first:first + warps], k, **a)
            assert torch.equal(experts_of[first:first + warps], e)
            assert torch.equal(weights[first:first + warps].nan_to_num(9.0), w.nan_to_num(9.0))
        few, w = check_route(logits[seen.cuda()], k, **a)
        assert torch.equal(experts_of[seen.cuda()], few) and torch.equal(weights[seen.cuda()].nan_to_num(9.0), w.nan_to_num(9.0))


# ---- activations ------------------------------------------------------------------------------------------------------
def gelu_points():
    """Both signs, far out, and around 0."""
    rng = np.random.default_rng(4)
    return np.concatenate([rng.standard_normal(8192), np.linspace(-12.5, 12.5, 16385), np.linspace(-1.01, 1.01, 4097), 10.0 ** np.linspace(-6, 0, 30)])


@pytest.mark.gpu
@pytest.mark.parametrize("kind", ["gelu", "silu"])
def test_binary32_activations(kind):
    """gelu.  Let u = 2^-24.  Further out than 1 Phi(-|x|) = e t S(t): 1 + p |x| is rounded, 1u, its reciprocal off by one in the last place, 2u, and S by 1u
    of its last sum and 1u of those before; the exponential by 2 in the last place, 4u, and 1u of its correction; two products 2u; the fit
    0.1u: 12u.  Nearer to 0 the sum 1/2 + x R is off by 1u of a half and 2u of x R, 3u of a Phi of 0.16 or more.  2^-20 is 16u, of Phi in f(x) and of
    Phi and x phi(x) in the slope.  Where |x| is 0.2 to 0.3 f(x) has one rounding of the sum and one of the product, each 1u at most and less than
    0.6u in the mean square: 1u for both; the slope's two terms and their sum likewise.
    silu.  The exponential is off by 4u, the sum 1 + e, its reciprocal and the product by 1u each, the slope's factors by two more: 2^-20 covers them."""
    x = torch.from_numpy(gelu_points()).float().cuda()
    at = x.double().cpu().numpy()[None]
    _, f, slope = (v[0] for v in ref.activation(at, kind, False))
    y, _ = rt.activation(x, kind)
    dx, again = rt.activation_backward(torch.ones_like(x), x, kind, want_y=True)
    assert torch.equal(again, y)
    x, y, dx = (v.double().cpu().numpy() for v in (x, y, dx))
    p = np.where(x == 0, 0.5, f / np.where(x == 0, 1.0, x))
    assert (np.abs(y - f) <= 2.0 ** -20 * np.abs(f)).all(), np.nanmax(np.abs(y - f) / np.abs(f)) * 2 ** 24
    size = p + np.abs(slope - p)
    assert (np.abs(dx - slope) <= 2.0 ** -20 * size).all(), np.max(np.abs(dx - slope) / size) * 2 ** 24
    near = (np.abs(x) > 0.2) & (np.abs(x) < 0.3) & (kind == "gelu")
    for got, want in ((y, f), (dx, slope)):
        assert not near.any() or np.sqrt(((got[near] / want[near] - 1) ** 2).mean()) <= 2.0 ** -24


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF])
@pytest.mark.parametrize("kind", ["silu", "gelu", "gelu_tanh"])
def test_16_bit_activations_far_out(kind, dtype):
    """f(x) of large negative x has as many bits as any other.  Let u = 2^-24.  The argument z of the exponential is rounded five times at most and has
    constants that are off by 0.6u together (gelu_tanh: the square, the cube's factor, the sum, and two products): 5.6 |z| u; the exponential is off by 2 units
    in the last place, 4u, its reciprocal and what that is of by 3u, products by 4u: 2^-16 = 256u covers |z| up to 43.  gelu has two roundings and a
    fit that is off by 78u: 2.6 |z| u and 89u, |z| up to 64.  2^-15 covers |z| up to 89, where p is 2^-128.  p and the slope's terms, which are up to 200 times
    larger, are above 2^-40 only where |z| is below 34.  And half a step of the type."""
    far = {"silu": 60.0, "gelu": 12.0, "gelu_tanh": 9.0}[kind]
    x = torch.from_numpy(np.concatenate([gelu_points(), np.linspace(-far, far, 8193)])).clamp(-far, far).to(dtype).cuda()
    _, f, slope = (v[0] for v in ref.activation(x.double().cpu().numpy()[None], kind, False))
    y, _ = rt.activation(x, kind)
    dx, again = rt.activation_backward(torch.ones_like(x), x, kind, want_y=True)
    assert torch.equal(again, y)
    x, y, dx = (v.double().cpu().numpy() for v in (x, y, dx))
    p = np.where(x == 0, 0.5, f / np.where(x == 0, 1.0, x))
    info = torch.finfo(dtype)
    for got, want, size in ((y, f, np.abs(f)), (dx, slope, p + np.abs(slope - p))):
        slack = np.where(size > 2.0 ** -40, 2.0 ** -16, 2.0 ** -15) * size
        half = info.eps / 2 * (np.abs(want) + slack) + info.smallest_normal * info.eps / 2  # the second of what is below the normal numbers
        assert (np.abs(got - want) <= slack + half).all(), (x[np.abs(got - want) > slack + half][:5], np.max(np.abs(got - want) / (slack + half)))


# ---- 8-bit rows -------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
@pytest.mark.parametrize("cols", [64, 61])
def test_smallest_rows_in_each_type(cols):
    """Every code with every scale byte that leaves bfloat16's numbers, rounded once to the type; float32 holds them all."""
    codes = torch.arange(256, dtype=torch.int32).repeat(1 + cols * 12 // 256)[:cols * 12].to(torch.uint8).view(12, cols)
    scales = torch.arange(12, dtype=torch.uint8).repeat_interleave((cols + 31) // 32).view(12, -1)
    rows = rt.Rows8(codes.view(torch.float8_e4m3fn).cuda(), scales.view(torch.float8_e8m0fnu).cuda())
    want = ref.unpacked(rows)
    got = rt.unpack8(rows, F)
    assert np.array_equal(got.double().cpu().numpy(), want, equal_nan=True)
    for dtype in (BF, HF):
        exact = torch.from_numpy(want).float().to(dtype)
        assert torch.equal(rt.unpack8(rows, dtype).cpu().nan_to_num(7.0), exact.nan_to_num(7.0))
    place = torch.arange(12, dtype=torch.int32).view(12, 1).cuda()
    spread = rt.spread_tokens(rows, place, torch.tensor([0, 12], device="cuda"))
    assert torch.equal(spread.cpu().nan_to_num(7.0), torch.from_numpy(want).float().to(BF).nan_to_num(7.0))
    fine = scales[:, 0] >= 3
    assert np.array_equal(rt.unpack8(rows).double().cpu().numpy()[fine], want[fine], equal_nan=True)
    assert not np.array_equal(rt.unpack8(rows).double().cpu().numpy()[0], want[0], equal_nan=True)


# ---- outputs ----------------------------------------------------------------------------------------------------------
@pytest.mark.gpu
def test_large_outputs_live_on_their_own():
    """Who keeps one of a call's outputs does not keep the others, once they are larger than a megabyte together."""
    def alone(*tensors):
        for t in tensors:
            assert t.untyped_storage().nbytes() == t.nbytes
    x, stream, w = torch.randn(1200, 512, device="cuda").to(BF), torch.randn(1200, 512, device="cuda"), torch.ones(512, device="cuda")
    y, y8, h, rstd = rt.rms_norm(x, w, residual=stream, want_y8=True)
    alone(y, h, rstd)
    experts, weights = rt.route(torch.randn(70_000, 8, device="cuda"), 2)
    alone(experts, weights)
    alone(*rt.sort_tokens(experts.view(-1, 1).repeat(1, 2), 8))
    alone(*rt.rms_norm_backward(y, h, rstd, w))
    alone(*rt.join_tokens_backward(y, torch.randn(2400, 512, device="cuda").to(BF), torch.arange(2400, dtype=torch.int32, device="cuda").view(1200, 2),
                                   torch.ones(1200, 2, device="cuda"), torch.tensor([0, 2400], device="cuda")))
    alone(*rt.activation_backward(y, x, want_y=True))


# ---- the order of groups ----------------------------------------------------------------------------------------------
def test_workspace_of_the_longest_sort():
    """A row of counts for every chunk of 32,768 pairs and one of the groups' sizes: nothing grows with the square of the pairs."""
    need = ref.c_library().regtopk_sort_tokens_workspace_bytes
    assert need(2**31 - 1, 1, 256, 8) == (65536 + 1) * 2048 * 4 and need(1 << 20, 1, 100, 1) == 128 * 100 * 4


@pytest.mark.gpu
@pytest.mark.parametrize("pairs,n,workers", [(1_500_001, 2048, 1), (10_000_001, 60, 3), (70_000_003, 33, 1), (4_300_000, 1, 1)])
def test_sort_of_many_chunks(pairs, n, workers):
    """Chunks whose counts are added up once for all blocks."""
    gen = torch.Generator(device="cuda").manual_seed(pairs)
    experts = torch.randint(-1, n, (pairs, 1), generator=gen, dtype=torch.int32, device="cuda")
    at = torch.tensor([pairs * i // workers for i in range(workers + 1)], device="cuda")
    offsets, place = rt.sort_tokens(experts, n, at)
    worker = torch.searchsorted(at, torch.arange(pairs, device="cuda"), right=True) - 1
    key = torch.where(experts.flatten() < 0, workers * n, worker * n + experts.flatten())
    assert torch.equal(offsets, torch.cat([key.new_zeros(1), key.bincount(minlength=workers * n + 1)[:-1].cumsum(0)]))
    order = key.argsort(stable=True)[: int(offsets[-1])]
    assert torch.equal(place.flatten()[order].long(), torch.arange(len(order), device="cuda"))
    assert bool((place.flatten()[key == workers * n] == -1).all())


@pytest.mark.gpu
def test_long_sorts_captured_and_at_once():
    """Three launches and a workspace: two captured graphs, replayed on other inputs and on two streams at once, give what calls give."""
    n, made = 256, [torch.randint(-1, 256, (1_300_007, 1), dtype=torch.int32, device="cuda") for _ in range(4)]
    want = [rt.sort_tokens(e, n) for e in made]
    graphs = []
    for _ in range(2):
        into, g = made[0].clone(), torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            out = rt.sort_tokens(into, n)
        graphs.append((into, g, out, torch.cuda.Stream()))
    for first in (0, 2):
        for i, (into, g, out, stream) in enumerate(graphs):
            into.copy_(made[first + i])
            stream.wait_stream(torch.cuda.current_stream())
        for into, g, out, stream in graphs:
            with torch.cuda.stream(stream):
                g.replay()
        torch.cuda.synchronize()
        for i, (into, g, out, stream) in enumerate(graphs):
            assert torch.equal(out[0], want[first + i][0]) and torch.equal(out[1], want[first + i][1])


# ---- the norm ---------------------------------------------------------------------------------------------------------
# More rows than teams on a device of 148 multiprocessors, so that rows come through the rings: one, two and more warps a row, one to four units a
# warp, rows that are kept in registers and rows that are read twice, aligned or not.  Fewer than 60 additions in a row to a weight's gradient.
MANY_ROWS = [(4001, 96), (3700, 250), (2501, 768), (2502, 767), (1902, 1024), (1901, 1023), (700, 2048), (621, 4096), (620, 4095), (301, 8192), (200, 8200), (180, 16383), (181, 16384)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype,stream", norm.TYPES)
@pytest.mark.parametrize("rows,cols", MANY_ROWS)
def test_norm_of_many_rows(rows, cols, dtype, stream):
    norm.test_forward(rows, cols, dtype, stream)
    norm.test_backward(rows, cols, dtype, stream)
    rt.training_status()
