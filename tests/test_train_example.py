"""The training operators together, as examples/expert_training.py uses them: every worker's gradient of the whole sublayer
against autograd in 64 bits, and the training loop with the sparsifier."""
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
    spec = importlib.util.spec_from_file_location("expert_training", os.path.join(ROOT, "examples", "expert_training.py"))
    module = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(module)
    return module


def test_gradients_of_the_sublayer(example):
    """Rows of the accumulator against autograd in float64 on the same bfloat16 weights.  Between them lie the roundings of
    the activations and their gradients to bfloat16 (2^-8 each, ten in a row): 2^-4 of each tensor's norm."""
    gen = torch.Generator(device="cuda").manual_seed(5)
    workers, tokens, width, hidden, experts = 3, 90, 40, 56, 4
    block = example.ExpertBlock(width, hidden, experts)
    theta = block.new_parameters(gen)
    v = block.views(theta)
    for name in ("up", "down"):
        v[name].copy_(v[name].bfloat16())
    x, groups, by_worker = example.batch(gen, workers, tokens, width, experts)
    x = x.bfloat16().float()
    sp = rt.RegTopK(block.size, workers, 100)
    sp.accumulator().normal_(generator=gen)
    before = sp.accumulator().clone()
    y, kept = block.forward(theta, x, groups, p=0.25, seed=7, step=3)
    dy = (torch.randn(y.shape, generator=gen, device="cuda") / tokens).bfloat16()
    dx = block.backward(dy, kept, groups, by_worker, sp.accumulator())
    got = (sp.accumulator() - before).double()

    factor = rt.dropout(torch.ones(workers * tokens, width, device="cuda"), 0.25, 7, 3).double()
    at, cuts = groups.tolist(), by_worker.tolist()
    for n in range(workers):
        flat = theta.double().requires_grad_()
        w = block.views(flat)
        own = slice(cuts[n], cuts[n + 1])
        xs = x[own].double().requires_grad_()
        n1 = F.layer_norm(xs, (width,), w["norm1"][0], w["norm1"][1])
        o = torch.zeros_like(xs)
        for e in range(experts):
            lo, hi = (at[n * experts + e + i] - cuts[n] for i in (0, 1))
            o = torch.cat([o[:lo], F.gelu(n1[lo:hi] @ w["up"][e].T) @ w["down"][e].T, o[hi:]])
        out = F.layer_norm(xs + o * factor[own], (width,), w["norm2"][0], w["norm2"][1])
        out.backward(dy[own].double())
        assert (y[own].double() - out).norm() < 2.0 ** -4 * out.norm()
        assert (dx[own].double() - xs.grad).norm() < 2.0 ** -4 * xs.grad.norm()
        want, have = block.views(flat.grad), block.views(got[n])
        for name in want:
            assert (have[name] - want[name]).norm() < 2.0 ** -4 * want[name].norm(), (n, name)


def test_training_falls(example):
    """The loss falls by half, with all coordinates sent and with one in fifty (error feedback makes up for it)."""
    for share in (1.0, 0.02):
        losses = example.train(steps=60, workers=4, tokens=128, width=64, hidden=96, experts=3, share=share)
        assert all(l == l for l in losses) and sum(losses[-5:]) < 0.5 * sum(losses[:5]), losses[::10]
