"""A compressed projection and the adapters that make up for it.

A gate projection of the 1500-wide LSTM language model (1500 -> 6000) is pruned and rounded to bfloat16 by one C-step and
stays as it is. What it lost is trained back with low-rank adapters beside it, one per task, all tasks in one batch: forward,
gradients, the norm that clips them, an AdamW step with 8-bit states (rounded by chance, from a seed) that also writes the
bfloat16 copies which the next forward pass reads. At the end a decoding step serves the tasks' requests, a token each, with and without an adapter.

    python examples/compressed_adapters.py [steps]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import numpy as np
import torch

from paper_1911_02497_b200 import cstep


def compress(ctx, w, sparsity=0.9):
    """theta of a C-step on ``w`` (no multipliers yet), rounded to bfloat16: prune, then quantise."""
    theta, theta_h = torch.empty_like(w), torch.empty(w.shape, dtype=torch.int16, device=w.device)
    tab = cstep.tensor_table([w], None, [theta], theta_h=[theta_h])
    ctx.cstep_prune(tab, 1, sparsity, 1e-3, fuse=("bf16",), stream=torch.cuda.current_stream())
    return theta_h.view(torch.bfloat16)


class Adapters:
    """fp32 masters of A and B for ``tasks`` tasks, their bfloat16 copies, gradients, and 8-bit AdamW states."""

    def __init__(self, tasks, k, n, rank, scale, generator):
        make = lambda *shape: torch.randn(*shape, device="cuda", generator=generator)
        self.a = [make(rank, k) / k ** 0.5 for _ in range(tasks)]
        self.b = [torch.zeros(n, rank, device="cuda") for _ in range(tasks)]
        self.master = self.a + self.b
        self.copy = [x.bfloat16() for x in self.master]
        self.grad = [torch.zeros_like(x) for x in self.master]
        blocks = [-(-x.numel() // cstep.STATE_BLOCK) for x in self.master]
        state = lambda: [torch.zeros(x.numel(), dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn) for x in self.master]
        scales = lambda: [torch.zeros(n, device="cuda") for n in blocks]
        self.m, self.v, self.m_scale, self.v_scale = state(), state(), scales(), scales()
        self.table = cstep.adapter_table(self.copy[:tasks], self.copy[tasks:], [scale] * tasks, self.grad[:tasks], self.grad[tasks:])
        self.optimizer = cstep.adamw_table(self.master, self.grad, self.m, self.v, self.m_scale, self.v_scale, w_h=self.copy)
        self.clip = torch.zeros(4, device="cuda")


def train(steps=150, tasks=3, rank=16, k=1500, n=6000, rows=256, seed=0, lr=4e-3):
    """Mean squared error of every task before and after, and a served batch's error with the adapters."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ctx, stream = cstep.Context(torch.cuda.current_device()), torch.cuda.current_stream()
    w = (torch.rand(n, k, device="cuda", generator=g) * 2 - 1) * 0.1
    theta = compress(ctx, w)
    # a task's inputs lie near a space of `rank` dimensions of its own, as far as an adapter can follow
    space = [torch.randn(rank, k, device="cuda", generator=g) for _ in range(tasks)]
    draw = lambda t, m: (torch.randn(m, rank, device="cuda", generator=g) @ space[t] / rank ** 0.5).bfloat16()
    ad = Adapters(tasks, k, n, rank, 2.0, g)
    length, which = np.full(tasks, rows, dtype=np.int64), np.arange(tasks, dtype=np.int32)
    h = torch.empty(tasks * rows, rank, device="cuda")
    errors = []
    for step in range(1, steps + 1):
        x = torch.cat([draw(t, rows) for t in range(tasks)])
        y = x @ theta.t()
        ctx.adapter_forward(ad.table, length, which, x, y, h, stream=stream)
        miss = y.float() - x.float() @ w.t()
        if step in (1, steps):
            errors.append([float(e) for e in miss.square().view(tasks, -1).mean(dim=1)])
        dy = (miss * (2.0 / rows)).bfloat16()
        ctx.adapter_backward(ad.table, length, which, x, dy, h, stream=stream)
        ctx.grad_norm(ad.optimizer, 0.0, 10.0, ad.clip, stream=stream)
        ctx.lstep_adamw(ad.optimizer, lr=lr, weight_decay=0.0, step=step, clip=ad.clip, state_seed=seed + 1, stream=stream)
    # a decoding step: a token per request, in any order, one of them without an adapter
    which = np.array([t % tasks for t in range(4 * tasks)] + [-1], dtype=np.int32)
    length = np.ones(len(which), dtype=np.int64)
    x = torch.cat([draw(max(int(t), 0), 1) for t in which])
    y = x @ theta.t()
    ctx.adapter_forward(ad.table, length, which, x, y, stream=stream)
    served = (y.float() - x.float() @ w.t()).square().mean(dim=1)
    out = {"before": errors[0], "after": errors[-1], "served": float(served[:-1].mean()), "without": float(served[-1])}
    ctx.close()
    return out


if __name__ == "__main__":
    r = train(int(sys.argv[1]) if len(sys.argv) > 1 else 150)
    print("mean squared error of the compressed projection, by task:", ["%.4f" % e for e in r["before"]])
    print("with the adapters:                                       ", ["%.4f" % e for e in r["after"]])
    print("decoding step, requests with an adapter: %.4f, the one without: %.4f" % (r["served"], r["without"]))
