"""The operators around an expert sublayer together, as examples/routed_training.py uses them: every worker's gradients against
autograd in 64 bits, on streams of their own, and captured as a CUDA graph."""
import importlib.util
import os

import pytest
import torch
import torch.nn.functional as F

import paper_2501_05633_b200 as rt

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def example():
    spec = importlib.util.spec_from_file_location("routed_training", os.path.join(ROOT, "examples", "routed_training.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def parts(example, gen, workers=3, tokens=90, width=40, hidden=56, experts=6, chosen=2):
    block = example.RoutedBlock(width, hidden, experts, chosen)
    theta = block.new_parameters(gen)
    v = block.views(theta)
    for name in ("router", "up", "down"):
        v[name].copy_(v[name].bfloat16())
    x, at = example.batch(gen, workers, tokens, width)
    return block, theta, x.bfloat16().float(), at


def test_gradients_of_the_sublayer(example):
    """Rows of the accumulator against autograd in float64 on the same bfloat16 weights, for the experts that were chosen.  Between
    them lie roundings of activations and gradients to bfloat16 (2^-8 each, ten in a row: 2^-4 of each tensor's norm) and of what is
    kept in 8 bits (at most 2^-4)."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    workers, width, hidden = 3, 40, 56
    block, theta, x, at = parts(example, gen)
    sp = rt.RegTopK(block.size, workers, 100)
    sp.accumulator().normal_(generator=gen)
    before = sp.accumulator().clone()
    y, kept = block.forward(theta, x, at)
    dy = torch.randn(y.shape, generator=gen, device="cuda") / 90
    dx = block.backward(dy, kept, at, sp.accumulator())
    got, chosen, cuts = (sp.accumulator() - before).double(), kept[8].long(), at.tolist()
    for n in range(workers):
        flat = theta.double().requires_grad_()
        w, own = block.views(flat), slice(cuts[n], cuts[n + 1])
        xs = x[own].double().requires_grad_()
        normed = xs * torch.rsqrt(xs.square().mean(1, keepdim=True) + 1e-6) * w["norm"]
        share = torch.softmax(torch.gather(normed @ w["router"].T, 1, chosen[own]), 1)
        a = torch.einsum("tc,thc->th", normed.repeat_interleave(2, 0), w["up"][chosen[own].flatten()])
        o = torch.einsum("th,tch->tc", F.silu(a[:, :hidden]) * a[:, hidden:], w["down"][chosen[own].flatten()])
        out = xs + (o.view(-1, 2, width) * share.unsqueeze(2)).sum(1)
        out.backward(dy[own].double())
        assert (y[own].double() - out).norm() < 2.0 ** -4 * out.norm()
        assert (dx[own].double() - xs.grad).norm() < 2.0 ** -3 * xs.grad.norm()
        want, have = block.views(flat.grad), block.views(got[n])
        for name in want:
            assert (have[name] - want[name]).norm() < 2.0 ** -3 * want[name].norm(), (n, name)


def step_of(example, block, theta, x, at, dy, rows):
    y, kept = block.forward(theta, x, at)
    return y, block.backward(dy, kept, at, rows), rows


def test_other_streams(example):
    """Two sublayers at once on two streams give the bits that each gives alone."""
    gen = torch.Generator(device="cuda").manual_seed(6)
    block, theta, x, at = parts(example, gen, tokens=700)
    xs = [x, torch.randn(x.shape, generator=gen, device="cuda")]
    dy = torch.randn(x.shape, generator=gen, device="cuda")
    alone = [[t.clone() for t in step_of(example, block, theta, v, at, dy, torch.zeros(3, block.size, device="cuda"))] for v in xs]
    torch.cuda.synchronize()
    streams, got = [torch.cuda.Stream() for _ in xs], []
    for _ in range(5):
        for s, v in zip(streams, xs):
            with torch.cuda.stream(s):
                got.append(step_of(example, block, theta, v, at, dy, torch.zeros(3, block.size, device="cuda")))
    torch.cuda.synchronize()
    for i, g in enumerate(got):
        assert all(torch.equal(a, b) for a, b in zip(g, alone[i % 2])), i
    rt.training_status()


@pytest.mark.parametrize("tokens", [500, 1500, 4000])
def test_captured_step(example, tokens):
    """A whole step as a CUDA graph, replayed on other inputs, other routes and other workers' shares among them; by its number of
    tokens the sort is one block, a cluster, or two launches with a workspace."""
    gen = torch.Generator(device="cuda").manual_seed(7)
    block, theta, x, at = parts(example, gen, tokens=tokens)
    dy, rows = torch.randn(x.shape, generator=gen, device="cuda"), torch.zeros(3, block.size, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(side):
        step_of(example, block, theta, x, at, dy, rows)
    torch.cuda.current_stream().wait_stream(side)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        y, dx, _ = step_of(example, block, theta, x, at, dy, rows)
    for seed in range(3):
        gen.manual_seed(seed)
        x.normal_(generator=gen)
        dy.normal_(generator=gen)
        at[1], at[2] = 100 * seed, 3 * tokens - 7 * seed
        rows.zero_()
        graph.replay()
        want = step_of(example, block, theta, x, at, dy, torch.zeros_like(rows))
        assert torch.equal(y, want[0]) and torch.equal(dx, want[1]) and torch.equal(rows, want[2])
    rt.training_status()


def test_padding_stays_out(example):
    """Tokens whose logits are -inf reach no expert: they pass as they are, and no weight gradient sees them."""
    gen = torch.Generator(device="cuda").manual_seed(8)
    block, theta, x, at = parts(example, gen)
    logits = torch.randn(270, 6, generator=gen, device="cuda")
    logits[::3] = -float("inf")
    experts, weights = rt.route(logits, 2)
    groups, place = rt.sort_tokens(experts, 6, at)
    assert int(groups[-1]) == 360 and (place[::3] == -1).all()
    rows = rt.spread_tokens(x, place, groups)
    assert not rows[360:].any()
    assert torch.equal(rt.join_tokens(rows, place, weights, residual=x)[::3], x[::3])
    drows, dw = rt.join_tokens_backward(x, rows, place, weights, groups)
    assert not dw[::3].any() and not drows[360:].any() and not rt.route_backward(dw, logits, experts)[::3].any()


def test_training_runs(example):
    losses = example.train(steps=12, workers=3, tokens=64, width=64, hidden=48, experts=4, share=0.05)
    assert len(losses) == 12 and all(l == l for l in losses)
