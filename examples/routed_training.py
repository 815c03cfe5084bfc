"""N workers train a transformer's routed expert sublayer on one GPU, with RegTop-k between their gradients.

    python examples/routed_training.py [--steps 200] [--workers 8] [--share 0.01] [--mu 4]

One step is: root-mean-square norm -> router -> tokens sorted by (worker, expert) -> up products -> gated SiLU -> down products ->
weighted sum on top of the residual stream -> squared error against a teacher of the same shape, and back.  For the backward pass the
norm's output and the activation's input are kept in 8 bits.  Every weight gradient is formed per worker and added straight into that
worker's row of the sparsifier's accumulator.
"""
import argparse
import os
import sys

import torch

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2501_05633_b200 as rt  # noqa: E402


class RoutedBlock:
    """The sublayer's parameters as views of one flat float32 vector, and of any rows that are laid out like it."""

    def __init__(self, width: int, hidden: int, experts: int, chosen: int):
        self.shapes = {"norm": (width,), "router": (experts, width), "up": (experts, 2 * hidden, width), "down": (experts, width, hidden)}
        self.experts, self.chosen = experts, chosen
        self.at, self.size = {}, 0
        for name, shape in self.shapes.items():
            self.at[name] = self.size
            self.size += torch.Size(shape).numel()

    def views(self, flat: torch.Tensor) -> dict:
        """The tensors within [size] or [rows, size]."""
        return {name: flat[..., self.at[name]: self.at[name] + torch.Size(shape).numel()].unflatten(-1, shape)
                for name, shape in self.shapes.items()}

    def new_parameters(self, gen: torch.Generator) -> torch.Tensor:
        theta = torch.zeros(self.size, device="cuda")
        v = self.views(theta)
        v["norm"].fill_(1.0)
        for name in ("router", "up", "down"):
            v[name].copy_(torch.randn(v[name].shape, generator=gen, device="cuda") * v[name].shape[-1] ** -0.5)
        return theta

    def forward(self, theta: torch.Tensor, x: torch.Tensor, workers: torch.Tensor):
        """(output, what the backward pass needs).  x: the float32 residual stream; workers: offsets by worker."""
        v = self.views(theta)
        router, up, down = v["router"].bfloat16().unsqueeze(0), v["up"].bfloat16(), v["down"].bfloat16()
        stream = x.bfloat16()
        n, n8, _, rstd = rt.rms_norm(stream, v["norm"], want_y8=True)
        logits = rt.grouped_matmul(n, router, workers)
        experts, weights = rt.route(logits, self.chosen)
        groups, place = rt.sort_tokens(experts, self.experts, workers)
        a = rt.grouped_matmul(rt.spread_tokens(n, place, groups), up, groups)
        g, a8 = rt.activation(a, gated=True, keep8=True)
        o = rt.grouped_matmul(g, down, groups)
        return rt.join_tokens(o, place, weights, residual=x), (v, router, up, down, stream, n8, rstd, logits, experts, weights, groups, place, a8, o)

    def backward(self, dy: torch.Tensor, kept, workers: torch.Tensor, rows: torch.Tensor) -> torch.Tensor:
        """Adds every worker's parameter gradients into its row; the gradient to x."""
        v, router, up, down, stream, n8, rstd, logits, experts, weights, groups, place, a8, o = kept
        d = self.views(rows)
        do, dweights = rt.join_tokens_backward(dy, o, place, weights, groups)
        da, g = rt.activation_backward(rt.grouped_matmul(do, down.transpose(1, 2), groups), a8, gated=True, want_y=True)
        rt.grouped_matmul_dw(do, g, groups, out=d["down"], accumulate=True)
        rt.grouped_matmul_dw(da, rt.spread_tokens(n8, place, groups), groups, out=d["up"], accumulate=True)
        dlogits = rt.route_backward(dweights, logits, experts)
        rt.grouped_matmul_dw(dlogits, rt.unpack8(n8), workers, out=d["router"], accumulate=True)
        dn = rt.join_tokens(rt.grouped_matmul(da, up.transpose(1, 2), groups), place, residual=rt.grouped_matmul(dlogits, router.transpose(1, 2), workers))
        dx, _, _ = rt.rms_norm_backward(dn, stream, rstd, v["norm"], offsets=workers, dweight=d["norm"], accumulate=True)
        return dy + dx


def batch(gen, workers, tokens, width):
    """The float32 stream of all workers and the offsets by worker."""
    return torch.randn(workers * tokens, width, generator=gen, device="cuda"), torch.arange(workers + 1, device="cuda") * tokens


def train(steps=200, workers=8, tokens=256, width=256, hidden=256, experts=8, chosen=2, share=0.01, mu=4.0, eta=20.0, seed=0, report=None):
    """The mean loss of every step."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    block = RoutedBlock(width, hidden, experts, chosen)
    teacher, theta = block.new_parameters(gen), block.new_parameters(gen)
    block.views(theta)["router"].copy_(block.views(teacher)["router"])
    sp = rt.RegTopK(block.size, workers, max(1, int(share * block.size)), mu=mu)
    losses = []
    for step in range(steps):
        x, by_worker = batch(gen, workers, tokens, width)
        target, _ = block.forward(teacher, x, by_worker)
        y, kept = block.forward(theta, x, by_worker)
        error = y - target
        losses.append(error.square().mean())
        block.backward(error * (2.0 / (tokens * width)), kept, by_worker, sp.accumulator())
        sp.worker_step_inplace()
        sp.aggregate_update(theta, eta)
        if report and (step + 1) % report == 0:
            print(f"step {step + 1}: loss {float(losses[-1]):.4f}")
    sp.status()
    rt.training_status()
    return torch.stack(losses).tolist()


if __name__ == "__main__":
    ap = argparse.ArgumentParser(description=__doc__.split("\n")[0])
    ap.add_argument("--steps", type=int, default=200)
    ap.add_argument("--workers", type=int, default=8)
    ap.add_argument("--share", type=float, default=0.01, help="share of the coordinates that each worker sends")
    ap.add_argument("--mu", type=float, default=4.0)
    args = ap.parse_args()
    losses = train(args.steps, args.workers, share=args.share, mu=args.mu, report=max(1, args.steps // 10))
    print(f"loss {losses[0]:.4f} -> {losses[-1]:.4f}")
