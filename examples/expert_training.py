"""N workers train a transformer's expert feed-forward sublayer on one GPU, with RegTop-k between their gradients.

    python examples/expert_training.py [--steps 200] [--workers 8] [--share 0.01] [--mu 4]

One step is: layer norm -> up products -> GELU -> down products -> dropout, residual sum and layer norm -> squared error
against a teacher of the same shape, and back.  The tokens of all workers lie in one array, sorted by worker and expert;
every weight gradient is formed per worker and added straight into that worker's row of the sparsifier's accumulator.
worker_step_inplace then sends each worker's k largest scores and aggregate_update applies what the server sums up to
the flat parameter vector, of which the model's tensors are views.
"""
import argparse
import os
import sys

import torch
import torch.nn.functional as F

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))
import paper_2501_05633_b200 as rt  # noqa: E402


class ExpertBlock:
    """The sublayer's parameters as views of one flat float32 vector, and of any rows that are laid out like it."""

    def __init__(self, width: int, hidden: int, experts: int):
        self.shapes = {"norm1": (2, width), "up": (experts, hidden, width), "down": (experts, width, hidden), "norm2": (2, width)}
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
        for name in ("norm1", "norm2"):
            v[name][0] = 1.0
        for name in ("up", "down"):
            v[name].copy_(torch.randn(v[name].shape, generator=gen, device="cuda") * v[name].shape[-1] ** -0.5)
        return theta

    def forward(self, theta: torch.Tensor, x: torch.Tensor, groups: torch.Tensor, p: float = 0.0, seed: int = 0, step: int = 0):
        """(output, what the backward pass needs).  x: the float32 residual stream; groups: offsets by (worker, expert)."""
        v = self.views(theta)
        up, down = v["up"].bfloat16(), v["down"].bfloat16()
        stream = x.bfloat16()
        n1, _, mean1, rstd1 = rt.layer_norm(stream, v["norm1"][0], v["norm1"][1])
        a = rt.grouped_matmul(n1, up, groups)
        g = F.gelu(a)
        o = rt.grouped_matmul(g, down, groups)
        y, h, mean2, rstd2 = rt.layer_norm(o, v["norm2"][0], v["norm2"][1], residual=x, p=p, seed=seed, subsequence=step)
        return y, (v, up, down, stream, n1, mean1, rstd1, a, g, h, mean2, rstd2, p, seed, step)

    def backward(self, dy: torch.Tensor, kept, groups: torch.Tensor, workers: torch.Tensor, rows: torch.Tensor) -> torch.Tensor:
        """Adds every worker's parameter gradients into its row; the gradient to x.  workers: offsets by worker."""
        v, up, down, stream, n1, mean1, rstd1, a, g, h, mean2, rstd2, p, seed, step = kept
        d = self.views(rows)
        do, dx, _, _ = rt.layer_norm_backward(dy, h, mean2, rstd2, v["norm2"][0], p=p, seed=seed, subsequence=step, offsets=workers,
                                              dweight=d["norm2"][:, 0], dbias=d["norm2"][:, 1], accumulate=True)
        rt.grouped_matmul_dw(do, g, groups, out=d["down"], accumulate=True)
        da = torch.ops.aten.gelu_backward(rt.grouped_matmul(do, down.transpose(1, 2), groups), a)
        rt.grouped_matmul_dw(da, n1, groups, out=d["up"], accumulate=True)
        dn1 = rt.grouped_matmul(da, up.transpose(1, 2), groups)
        dstream, _, _, _ = rt.layer_norm_backward(dn1, stream, mean1, rstd1, v["norm1"][0], offsets=workers,
                                                  dweight=d["norm1"][:, 0], dbias=d["norm1"][:, 1], accumulate=True)
        return dx + dstream


def batch(gen, workers, tokens, width, experts):
    """Tokens sorted by (worker, expert): the float32 stream, the offsets by group and by worker."""
    expert = torch.randint(0, experts, (workers, tokens), generator=gen, device="cuda").sort(dim=1).values
    group = expert + experts * torch.arange(workers, device="cuda").unsqueeze(1)
    counts = torch.bincount(group.reshape(-1), minlength=workers * experts)
    groups = F.pad(counts.cumsum(0), (1, 0))
    return torch.randn(workers * tokens, width, generator=gen, device="cuda"), groups, groups[::experts].contiguous()


def train(steps=200, workers=8, tokens=256, width=256, hidden=512, experts=4, share=0.01, mu=4.0, eta=20.0, p=0.1, seed=0, report=None):
    """The mean loss of every step."""
    gen = torch.Generator(device="cuda").manual_seed(seed)
    block = ExpertBlock(width, hidden, experts)
    teacher, theta = block.new_parameters(gen), block.new_parameters(gen)
    sp = rt.RegTopK(block.size, workers, max(1, int(share * block.size)), mu=mu)
    losses = []
    for step in range(steps):
        x, groups, by_worker = batch(gen, workers, tokens, width, experts)
        target, _ = block.forward(teacher, x, groups)
        y, kept = block.forward(theta, x, groups, p=p, seed=seed, step=step)
        error = y.float() - target.float()
        losses.append(error.square().mean())
        block.backward((error * (2.0 / (tokens * width))).bfloat16(), kept, groups, by_worker, sp.accumulator())
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
