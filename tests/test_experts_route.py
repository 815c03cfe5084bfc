"""Routing and the order of groups, against the definitions in 64 bits.  The experts and their order have to be the same.

Tolerances.  Let u = 2^-24.  A weight is a quotient of exponentials, each off by 2 units in its last place and by the rounding of
its argument, |l - l'| u for logits at most 32 apart here, and of a sum of up to 512 of them (21 additions in a row): 2^-18 of it covers
that.  A gradient is scale p (dw - sum of dw p) with each factor off by as much and a sum of at most 10 additions in a row: 2^-17 of the
magnitudes that enter, and a rounding to the type."""
import numpy as np
import pytest
import torch

import paper_2501_05633_b200 as rt
from tests import experts_reference as ref
from tests.test_train_norm import made
from tests.train_reference import assert_close, host

BF, HF, F = torch.bfloat16, torch.float16, torch.float32
INF = float("inf")


# ---- without a GPU -----------------------------------------------------------------------------------------------------
def test_reference_gradient_against_differences():
    rng = np.random.default_rng(3)
    l, dw = rng.standard_normal((4, 9)), rng.standard_normal((4, 3))
    for kind in ("softmax", "sigmoid"):
        for renormalise in (False, True):
            experts, _ = ref.route(l, 3, kind, rng.standard_normal(9), 1, 1, 1, renormalise, 1.5)
            grad, v = ref.route_backward(dw, l, experts, kind, renormalise, 1.5), rng.standard_normal(l.shape)
            ends = [(ref.route_weights(l + s * v, experts, kind, renormalise, 1.5) * dw).sum() for s in (1e-6, -1e-6)]
            assert abs((ends[0] - ends[1]) / 2e-6 - (grad * v).sum()) < 1e-7


def test_c_entries_refuse():
    """Bad arguments come back as codes before anything is launched (the pointers here are never followed)."""
    lib, p = ref.c_library(), 4096

    def call(tokens=4, n=16, k=2, type=0, ld=16, logits=p, experts=p, weights=p, **params):
        r = ref.RouteParams(*{**dict(scores=0, groups=1, kept=1, top=1, renormalise=1, scale=1.0), **params}.values())
        forward = lib.regtopk_route(logits, ld, None, experts, weights, tokens, n, k, type, r, None)
        assert lib.regtopk_route_backward(weights, logits, ld, experts, p, 1024, tokens, n, k, type, r, None) == forward
        return forward
    for bad in (dict(tokens=-1), dict(n=0), dict(k=0), dict(k=17), dict(type=3), dict(ld=15), dict(logits=None), dict(logits=p + 2), dict(experts=None),
                dict(experts=p + 2), dict(weights=None), dict(scores=2), dict(groups=0), dict(groups=3), dict(groups=4, kept=5), dict(kept=0), dict(top=0),
                dict(top=3), dict(scale=float("nan")), dict(scale=INF)):
        assert call(**bad) == -1, bad
    assert call(n=513, ld=513) == -7 and call(n=64, ld=64, k=33) == -7 and call(n=64, ld=64, groups=64) == -7 and call(tokens=0) == 0

    def sort(tokens=4, k=2, n=8, workers=1, at=None, offsets=p, place=p, ws=p, nbytes=1 << 40):
        return lib.regtopk_sort_tokens(p, at, workers, offsets, place, tokens, k, n, ws, nbytes, None)
    for bad in (dict(tokens=-1), dict(k=0), dict(n=0), dict(workers=0), dict(workers=2), dict(workers=2, at=p + 4), dict(offsets=None), dict(offsets=p + 4),
                dict(place=None), dict(tokens=1 << 20, ws=None), dict(tokens=1 << 20, ws=p + 8)):
        assert sort(**bad) == -1, bad
    assert sort(tokens=1 << 20, nbytes=64) == -2 and sort(n=1025, workers=2, at=p) == -7 and sort(tokens=2**31) == -7
    need = lib.regtopk_sort_tokens_workspace_bytes
    assert need(16, 2, 8, 1) == 0 and need(-1, 2, 8, 1) == 0 and need(1 << 20, 8, 256, 8) >= 4 * 2048 and need(1 << 20, 8, 256, 9) == 0


def test_no_cpu_path():
    with pytest.raises(TypeError):
        rt.route(torch.zeros(4, 8), 2)
    with pytest.raises(TypeError):
        rt.sort_tokens(torch.zeros(4, 2, dtype=torch.int32), 8)


# ---- on the GPU: the router ----------------------------------------------------------------------------------------------
def check_route(logits, k, **kw):
    a = {**dict(scores="softmax", bias=None, groups=1, groups_kept=1, group_top=1, renormalise=True, scale=1.0), **kw}
    experts, weights = rt.route(logits, k, **a)
    l, b = host(logits).reshape(-1, logits.shape[-1]), None if a["bias"] is None else host(a["bias"])
    want, w = ref.route(l, k, a["scores"], b, a["groups"], a["groups_kept"], a["group_top"], a["renormalise"], a["scale"])
    assert experts.dtype == torch.int32 and weights.dtype == F and experts.shape == weights.shape == (*logits.shape[:-1], k)
    got = experts.cpu().numpy().reshape(want.shape)
    assert np.array_equal(got, want), (got[(got != want).any(1)][:3], want[(got != want).any(1)][:3])
    assert_close(weights, w, 2.0 ** -18 * np.abs(np.nan_to_num(w)) + 1e-37, F, "weights")
    return experts, weights


CASES = [  # tokens, experts, k, groups, kept
    (1, 1, 1, 1, 1), (5, 2, 2, 1, 1), (33, 8, 2, 1, 1), (40, 60, 4, 1, 1), (17, 64, 6, 8, 3), (20, 256, 8, 8, 4), (9, 384, 8, 1, 1), (8, 512, 32, 1, 1),
    (7, 500, 9, 4, 2), (11, 96, 5, 3, 2), (6, 32, 32, 1, 1), (5, 64, 3, 32, 7), (300, 128, 8, 4, 4), (3, 510, 7, 3, 1)]


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("tokens,experts,k,groups,kept", CASES)
def test_route(tokens, experts, k, groups, kept, dtype):
    gen = torch.Generator().manual_seed(tokens * 7 + experts)
    k = min(k, kept * experts // groups)
    for pad, shift in ((0, 0), (3, 1)):
        logits = made(tokens, experts, dtype, gen, pad, shift, scale=1.5)
        bias = (0.1 * torch.randn(experts, generator=gen)).cuda()
        for scores in ("softmax", "sigmoid"):
            for b in (None, bias):
                for top in (1, 2):
                    check_route(logits, k, scores=scores, bias=b, groups=groups, groups_kept=kept, group_top=top, renormalise=top == 1, scale=2.5)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("experts,k,groups,kept", [(256, 8, 8, 4), (256, 8, 2, 1), (64, 6, 1, 1), (128, 3, 4, 2), (100, 8, 1, 1), (8, 2, 1, 1), (96, 4, 3, 2), (32, 1, 1, 1)])
def test_route_of_many_tokens(experts, k, groups, kept, dtype):
    """Enough tokens for the kernel that takes four at a time: ordinary ones, and with ties, neighbours, masks and NaN among them."""
    gen = torch.Generator().manual_seed(experts + k)
    tokens = 2501
    logits = (1.5 * torch.randn(tokens, experts, generator=gen)).to(dtype)
    logits[100:160] = (torch.randint(-3, 3, (60, experts), generator=gen) / 4).to(dtype)
    logits[200:260] = (logits[200:260].float().round() + torch.randint(0, 9, (60, experts), generator=gen) * 2.0 ** -22).to(dtype)
    logits[300:320, : experts // 2] = -INF
    logits[320:330] = -INF
    logits[330:340, 1:] = -INF
    logits[340] = torch.finfo(dtype).min
    logits[341, :7] = 9.0  # one lane's
    bias = (0.1 * torch.randn(experts, generator=gen)).cuda()
    logits = logits.cuda()
    for scores, b, top, renormalise in (("sigmoid", bias, 2, True), ("softmax", bias, 1, False), ("softmax", None, 2, True), ("sigmoid", None, 1, False), ("softmax", None, 1, False)):
        check_route(logits, k, scores=scores, bias=b, groups=groups, groups_kept=kept, group_top=top, renormalise=renormalise, scale=2.5)
    logits[400, experts - 1], logits[401, 0] = float("nan"), INF
    e, w = rt.route(logits, k)
    assert w[400:402].isnan().all() and w[402:].isfinite().all() and ((e[400:] >= 0) & (e[400:] < experts)).all()


@pytest.mark.gpu
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("dtype", [BF, F])
def test_ties(scores, dtype):
    """Few different numbers: ties within a lane's experts and between lanes, with and without a bias, and of groups."""
    gen = torch.Generator().manual_seed(2)
    for experts, groups, kept in ((256, 1, 1), (256, 8, 4), (48, 4, 2), (512, 1, 1), (512, 16, 5)):
        logits = (torch.randint(-3, 3, (60, experts), generator=gen) / 4).to(dtype).cuda()
        logits[0] = 0
        logits[1] = -logits[1].abs() * 0  # zeros of both signs
        logits[1, ::3] = 0
        bias = (torch.randint(-2, 2, (experts,), generator=gen) / 8).cuda()
        for b in (None, torch.zeros(experts, device="cuda"), bias):
            for top in (1, 2):
                check_route(logits, 8, scores=scores, bias=b, groups=groups, groups_kept=kept, group_top=top)


@pytest.mark.gpu
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
@pytest.mark.parametrize("experts", [64, 256])
def test_neighbours(scores, experts):
    """Numbers that differ in their last bits alone: binary32 cannot tell the scores apart, the choice has to."""
    gen = torch.Generator().manual_seed(5)
    base = torch.randint(-2, 2, (200, experts), generator=gen).float()
    logits = (base + torch.randint(0, 40, (200, experts), generator=gen) * 2.0 ** -22).cuda()
    bias = (0.5 + torch.randint(0, 8, (experts,), generator=gen) * 2.0 ** -24).cuda()
    for b in (None, bias):
        for groups, top in ((1, 1), (8, 1), (8, 2)):
            check_route(logits, 6, scores=scores, bias=b, groups=groups, groups_kept=max(1, groups // 2), group_top=top)


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("scores", ["softmax", "sigmoid"])
def test_masks(scores, dtype):
    """-inf takes experts out, one or all; the type's lowest value does not; NaN is the last to be chosen."""
    gen = torch.Generator().manual_seed(8)
    for experts, groups in ((8, 1), (64, 8), (256, 1)):
        logits = torch.randn(12, experts, generator=gen).to(dtype).cuda()
        logits[0] = -INF
        logits[1, 1:] = -INF
        logits[2, experts // 2:] = -INF
        logits[3] = torch.finfo(dtype).min
        logits[4, 3:] = torch.finfo(dtype).min
        logits[5, ::2] = torch.finfo(dtype).min
        logits[6, :5] = -INF
        for bias in (None, torch.zeros(experts, device="cuda"), torch.linspace(-1, 1, experts).cuda()):
            for top in (1, 2):
                for renormalise in (True, False):
                    e, w = check_route(logits, 4, scores=scores, bias=bias, groups=groups, groups_kept=max(1, groups // 2), group_top=top, renormalise=renormalise)
        assert (e[0] == -1).all() and (w[0] == 0).all()
    bias = torch.zeros(64, device="cuda")
    bias[::2] = -INF
    bias[1] = INF
    e, _ = check_route(logits[:, :64].contiguous(), 3, scores=scores, bias=bias)
    assert (e[7:] % 2 == 1).all() and (e[7:, 0] == 1).all()


@pytest.mark.gpu
@pytest.mark.parametrize("bias", [False, True])
def test_not_a_number(bias):
    """A NaN makes softmax weights NaN, and a sigmoid's only where it is chosen, which is last; the experts are some of the token's own."""
    logits = torch.randn(4, 64, generator=torch.Generator().manual_seed(8)).cuda()
    logits[0, 9] = float("nan")
    logits[1, 9] = INF
    logits[2] = float("nan")
    b = torch.linspace(-1, 1, 64).cuda() if bias else None
    e, w = rt.route(logits, 4, bias=b)
    assert w[:3].isnan().all() and w[3].isfinite().all() and ((e >= 0) & (e < 64)).all()
    assert all(len(set(row)) == 4 for row in e.tolist())
    e, w = rt.route(logits, 4, scores="sigmoid", bias=b, renormalise=False)
    assert not (e[0] == 9).any() and w[0].isfinite().all() and w[2].isnan().all() and e[2].tolist() == [0, 1, 2, 3]
    assert e[1, 0] == 9 if not bias else (e[1] >= 0).all()
    logits[0, 4:] = -INF
    logits[0, 2] = float("nan")
    e, w = rt.route(logits, 4, scores="sigmoid", bias=b, renormalise=False)
    assert e[0, 3] == 2 and w[0, 3].isnan() and w[0, :3].isfinite().all()


@pytest.mark.gpu
def test_weights_of_small_scores():
    """Renormalised weights where every score is too small for binary32."""
    logits = torch.tensor([[-200.0, -201.0, -202.0, -500.0], [-1e30, -1e30, -3e38, -3e38], [120.0, -120.0, 100.0, 90.0]], device="cuda")
    for scores in ("softmax", "sigmoid"):
        _, w = check_route(logits, 3, scores=scores)
        assert torch.allclose(w.sum(1), torch.ones(3, device="cuda"))
    check_route(logits, 3, bias=torch.tensor([-9.0, 0.0, 0.0, 9.0], device="cuda"))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, HF, F])
@pytest.mark.parametrize("tokens,experts,k,groups,kept", CASES)
def test_route_backward(tokens, experts, k, groups, kept, dtype):
    gen = torch.Generator().manual_seed(tokens + experts)
    for pad, shift in ((0, 0), (3, 1)):
        logits = made(tokens, experts, dtype, gen, pad, shift, scale=1.5)
        chosen = torch.rand(tokens, experts, generator=gen).argsort(1)[:, :k].to(torch.int32)
        if k > 1:
            chosen[0, 0], chosen[-1, 1] = -1, experts  # none
        if tokens > 2 and k > 2:
            chosen[1, :3] = chosen[1, 0]  # the same expert three times
        dw = torch.randn(tokens, k, generator=gen)
        if experts > 2 and tokens > 2:
            logits[2, 0] = -INF
            chosen[2] = torch.arange(experts - k, experts)  # not that one, if there are others
            if k == experts:
                logits[2, 0] = 0.0
        for scores in ("softmax", "sigmoid"):
            for renormalise in (True, False):
                got = rt.route_backward(dw.cuda(), logits, chosen.cuda(), scores=scores, renormalise=renormalise, scale=2.5)
                want = ref.route_backward(dw.double().numpy(), host(logits), chosen.numpy(), scores, renormalise, 2.5)
                most = 2.5 * np.abs(dw.double().numpy()).sum(1, keepdims=True) * np.ones_like(want)
                s = ref.scores_of(host(logits), scores)
                size = np.where(want == 0, 0.0, most) if renormalise else most * s
                assert got.dtype == dtype and got.shape == logits.shape
                assert_close(got, want, 2.0 ** -17 * size, dtype, (scores, renormalise))


@pytest.mark.gpu
@pytest.mark.parametrize("dtype", [BF, F])
@pytest.mark.parametrize("tokens,experts,k,scores,renormalise", [(4801, 8, 2, "softmax", False), (9600, 16, 3, "softmax", False), (4799, 60, 4, "sigmoid", True),
                                                                 (5003, 64, 8, "softmax", True), (20011, 7, 1, "sigmoid", False)])
def test_route_backward_of_many_tokens(tokens, experts, k, scores, renormalise, dtype):
    """Enough tokens for the kernel that takes several at a time, the last ones fewer."""
    gen = torch.Generator().manual_seed(tokens)
    logits = made(tokens, experts, dtype, gen, 3, 1, scale=1.5)
    chosen = torch.rand(tokens, experts, generator=gen).argsort(1)[:, :k].to(torch.int32)
    chosen[torch.rand(tokens, k, generator=gen) < 0.05] = -1
    if k > 2:
        chosen[::7, :3] = chosen[::7, :1]  # the same expert three times
    logits[5] = -INF
    chosen[5] = -1
    dw = torch.randn(tokens, k, generator=gen)
    got = rt.route_backward(dw.cuda(), logits, chosen.cuda(), scores=scores, renormalise=renormalise, scale=2.5)
    want = ref.route_backward(dw.double().numpy(), host(logits), chosen.numpy(), scores, renormalise, 2.5)
    most = 2.5 * np.abs(dw.double().numpy()).sum(1, keepdims=True) * np.ones_like(want)
    hit = np.zeros(want.shape, bool)  # the terms of a chosen expert may add up to 0 (where it is the only one), the others are 0
    for j in range(k):
        t = np.nonzero(chosen[:, j].numpy() >= 0)[0]
        hit[t, chosen[t, j].numpy()] = True
    assert_close(got, want, 2.0 ** -17 * (np.where(hit, most, 0.0) if renormalise else most * ref.scores_of(host(logits), scores)), dtype, scores)


@pytest.mark.gpu
def test_route_refusals():
    l = torch.zeros(4, 16, device="cuda")
    e, w = rt.route(l, 2)
    for call in (lambda: rt.route(l.double(), 2), lambda: rt.route(l, 2, bias=l[0, :8]), lambda: rt.route(l, 2, bias=l[0].to(BF)), lambda: rt.route(l, 2.0),
                 lambda: rt.route_backward(w, l, e.long()), lambda: rt.route_backward(w.to(BF), l, e), lambda: rt.route_backward(w[:2], l, e),
                 lambda: rt.route_backward(w[:2].contiguous(), l, e[:2].contiguous()), lambda: rt.route_backward(w, l[:, :1], e),
                 lambda: rt.sort_tokens(e.long(), 16), lambda: rt.sort_tokens(e.t(), 16), lambda: rt.sort_tokens(e, 16, torch.zeros(2, device="cuda")),
                 lambda: rt.sort_tokens(e, 16, torch.zeros(1, dtype=torch.int64, device="cuda"))):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: rt.route(l, 0), lambda: rt.route(l, 17), lambda: rt.route(l, 2, scores="tanh"), lambda: rt.route(l, 2, scores=None),
                 lambda: rt.route(l, 2, groups=3), lambda: rt.route(l, 2, groups=0), lambda: rt.route(l, 2, groups=4, groups_kept=5),
                 lambda: rt.route(l, 2, groups=4, groups_kept=2, group_top=3), lambda: rt.route(l, 2, scale=INF), lambda: rt.route(l.t(), 2),
                 lambda: rt.route(l[:1].expand(4, 16), 2), lambda: rt.route(l[:, :0], 1), lambda: rt.sort_tokens(e, 0), lambda: rt.sort_tokens(e[:, :0], 16)):
        with pytest.raises(ValueError):
            call()
    for call in (lambda: rt.route(torch.zeros(2, 513, device="cuda"), 2), lambda: rt.route(torch.zeros(2, 64, device="cuda"), 33),
                 lambda: rt.route(torch.zeros(2, 64, device="cuda"), 3, groups=64), lambda: rt.sort_tokens(e, 2049)):
        with pytest.raises(rt.RegTopKError):
            call()
    none = torch.zeros(0, 16, device="cuda")
    e, w = rt.route(none, 2)
    assert e.shape == (0, 2) and rt.route_backward(w, none, e).shape == (0, 16)


# ---- on the GPU: the order of groups -------------------------------------------------------------------------------------
def check_sort(experts, n, at=None):
    offsets, place = rt.sort_tokens(experts, n, at)
    bounds = [0, experts.numel() // experts.shape[-1]] if at is None else at.tolist()
    want, where = ref.sort_tokens(experts.cpu().numpy().reshape(-1, experts.shape[-1]), n, bounds)
    assert offsets.dtype == torch.int64 and place.dtype == torch.int32 and place.shape == experts.shape
    assert np.array_equal(offsets.cpu().numpy(), want) and np.array_equal(place.cpu().numpy().reshape(where.shape), where)
    return offsets, place


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,k,n", [(1, 1, 1), (7, 3, 5), (33, 2, 8), (513, 8, 16), (700, 7, 64), (3000, 2, 512), (2049, 4, 100), (1366, 3, 9)])
def test_sort(tokens, k, n):
    gen = torch.Generator().manual_seed(tokens)
    experts = torch.randint(0, n, (tokens, k), generator=gen, dtype=torch.int32)
    for lost in (False, True):
        if lost:  # none, too large, and tokens of no worker
            experts[torch.rand(tokens, k, generator=gen) < 0.2] = -1
            experts[torch.rand(tokens, k, generator=gen) < 0.05] = n
            experts[0, 0] = -2**31
        check_sort(experts.cuda(), n)
        for cuts in ([0, tokens], [0, 0, tokens // 3, tokens // 3, tokens], [tokens // 4, tokens // 2, tokens - tokens // 8]):
            if (len(cuts) - 1) * n <= 2048:
                check_sort(experts.cuda(), n, torch.tensor(cuts, device="cuda"))
    check_sort(torch.full((tokens, k), n - 1, dtype=torch.int32, device="cuda"), n)
    check_sort(torch.full((tokens, k), -1, dtype=torch.int32, device="cuda"), n)


@pytest.mark.gpu
def test_sort_many_workers():
    gen = torch.Generator().manual_seed(9)
    at = torch.cat([torch.zeros(1, dtype=torch.int64), torch.randint(0, 20, (256,), generator=gen).cumsum(0)])
    experts = torch.randint(0, 8, (int(at[-1]), 2), generator=gen, dtype=torch.int32)
    check_sort(experts.cuda(), 8, at.cuda())
    check_sort(experts.view(-1, 1, 2).cuda(), 8, at.cuda())


@pytest.mark.gpu
@pytest.mark.parametrize("tokens,k,n,workers", [(8192, 8, 256, 8), (8193, 8, 16, 128), (100_000, 8, 256, 8), (300_001, 3, 60, 3), (5_000_000, 1, 2, 1)])
def test_sort_large(tokens, k, n, workers):
    """Against a stable sort by torch."""
    gen = torch.Generator(device="cuda").manual_seed(tokens)
    experts = torch.randint(-1, n, (tokens, k), generator=gen, dtype=torch.int32, device="cuda")
    at = torch.tensor([tokens * i // workers for i in range(workers + 1)], device="cuda")
    offsets, place = rt.sort_tokens(experts, n, at)
    key = torch.where(experts < 0, workers * n, (torch.searchsorted(at, torch.arange(tokens, device="cuda"), right=True) - 1).unsqueeze(1) * n + experts).flatten()
    order = key.argsort(stable=True)
    want = torch.empty_like(order).scatter_(0, order, torch.arange(len(key), device="cuda"))
    assert torch.equal(place.flatten().long(), torch.where(key == workers * n, -1, want))
    assert torch.equal(offsets[1:], key.bincount(minlength=workers * n + 1)[:-1].cumsum(0)) and offsets[0] == 0


@pytest.mark.gpu
def test_sort_bounds_that_do_not_ascend():
    """Whatever the workers' offsets are, the places are distinct and within the groups."""
    experts = torch.randint(0, 4, (500, 3), generator=torch.Generator().manual_seed(1), dtype=torch.int32).cuda()
    for at in ([500, 0, 300], [-5, 900, 100, 500], [2**62, -2**62], [7, 7]):
        offsets, place = rt.sort_tokens(experts, 4, torch.tensor(at, device="cuda"))
        there = place[place >= 0].long()
        assert torch.equal(there.sort().values, torch.arange(int(offsets[-1]), device="cuda")) and (offsets.diff() >= 0).all()
