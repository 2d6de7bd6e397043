"""A residual block around a projection in 8 bits, with adapters and the norm's gain trained through it.

    h = x + r;   z = norm(h) * gain, in bfloat16 and in 8 bits;   y = z theta^T + adapter(z)

theta, a gate projection of the 1500-wide LSTM language model (1500 -> 6000), is pruned by a C-step, encoded in blocks of 8 bits and
stays as it is; the multipliers of a further C-step go by the values that its codes hold. The backward pass encodes dy by rows, takes
it through the codes (dz = dy theta), adds the adapter's part, and through the norm; an 8-bit code passes its gradient on as if it were
not rounded. Gain and adapters take AdamW steps. At the end one token is served by the captured forward pass.

    python examples/compressed_block.py [steps]
"""
import os
import sys

sys.path.insert(0, os.path.dirname(os.path.dirname(os.path.abspath(__file__))))

import torch

from paper_1911_02497_b200 import cstep


def coded(rows, cols, blocks=False):
    """Room for an 8-bit matrix: rows of codes a multiple of 128 bytes apart, of scales a multiple of 4."""
    groups = -(-cols // cstep.CODE_GROUP)
    codes = torch.zeros(rows, groups * cstep.CODE_GROUP, dtype=torch.uint8, device="cuda")[:, :cols].view(torch.float8_e4m3fn)
    scales = torch.zeros(-(-rows // cstep.CODE_GROUP) if blocks else rows, -(-groups // 4) * 4, dtype=torch.uint8, device="cuda")[:, :groups]
    return (cstep.coded_blocks if blocks else cstep.coded_rows)(codes, scales)


def compress(ctx, w, sparsity=0.5):
    """theta of a C-step on ``w`` in 8 bits, the values that it holds, and the multipliers that follow from them."""
    theta, lam = torch.empty_like(w), torch.zeros_like(w)
    stream = torch.cuda.current_stream()
    tab = cstep.tensor_table([w], [lam], [theta])
    ctx.cstep_prune(tab, 1, sparsity, 1e-3, stream=stream)
    weight = coded(w.shape[0], w.shape[1], blocks=True)
    ctx.encode_blocks(theta, weight, theta=theta, stream=stream)
    ctx.cstep_lagrange_update(tab, 1, 1e-3, fuse=("lambda",), stream=stream)
    return weight, theta, lam


class Block:
    """The block's buffers for ``rows`` rows, its parameters and their gradients."""

    def __init__(self, ctx, weight, rows, rank, generator):
        n, k = weight.rows, weight.cols
        bf16 = lambda *shape: torch.zeros(*shape, dtype=torch.bfloat16, device="cuda")
        self.ctx, self.weight, self.rows = ctx, weight, rows
        self.gain = torch.ones(k, device="cuda")
        self.a = torch.randn(rank, k, device="cuda", generator=generator) / k ** 0.5
        self.b = torch.zeros(n, rank, device="cuda")
        self.copy = [self.a.bfloat16(), self.b.bfloat16()]
        self.grad = [torch.zeros_like(t) for t in (self.gain, self.a, self.b)]
        self.h, self.z, self.y, self.dz, self.dx = bf16(rows, k), bf16(rows, k), bf16(rows, n), bf16(rows, k), bf16(rows, k)
        self.z8, self.dy8 = coded(rows, k), coded(rows, n)
        self.rstd, self.hidden = torch.zeros(rows, device="cuda"), torch.zeros(rows, rank, device="cuda")
        self.adapters = cstep.adapter_table([self.copy[0]], [self.copy[1]], [2.0], [self.grad[1]], [self.grad[2]])

    def forward(self, x, r, stream=None):
        self.ctx.norm_forward(x, self.gain, residual=r, h=self.h, y=self.z, code=self.z8, rstd=self.rstd, stream=stream)
        self.ctx.projection_forward(self.weight, self.z8, self.y, stream=stream)
        self.ctx.adapter_forward(self.adapters, [self.rows], [0], self.z, self.y, self.hidden, stream=stream)
        return self.y

    def backward(self, dy, dh, stream=None):
        """``dy``: gradient of y; ``dh``: of h, from the residual stream. The gradient of x and r is returned, those of the parameters are
        left in ``grad``."""
        self.ctx.encode_rows(dy, self.dy8, stream=stream)
        self.ctx.projection_backward(self.weight, self.dy8, self.dz, stream=stream)
        self.ctx.adapter_backward(self.adapters, [self.rows], [0], self.z, dy, self.hidden, self.dz, stream=stream)
        self.ctx.norm_backward(self.dz, self.h, self.gain, self.rstd, dh=dh, dx=self.dx, dgain=self.grad[0], stream=stream)
        return self.dx


def train(steps=60, rank=16, k=1500, n=6000, rows=512, seed=0, lr=4e-3):
    """Mean squared error of the block against the uncompressed one, before and after, and of one token from a captured pass."""
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    ctx, stream = cstep.Context(torch.cuda.current_device()), torch.cuda.current_stream()
    w = (torch.rand(n, k, device="cuda", generator=g) * 2 - 1) * 0.1
    weight, theta, _ = compress(ctx, w)
    block = Block(ctx, weight, rows, rank, g)
    master = [block.gain, block.a, block.b]
    state = [[torch.zeros_like(t) for t in master] for _ in range(2)]
    optimizer, clip = cstep.adamw_table(master, block.grad, *state, w_h=[None] + block.copy), torch.zeros(4, device="cuda")
    space = torch.randn(rank, k, device="cuda", generator=g)           # inputs lie near a space that the adapters can follow
    draw = lambda m: (torch.randn(m, rank, device="cuda", generator=g) @ space / rank ** 0.5).bfloat16()
    target = lambda h: (h * (h.square().mean(dim=1, keepdim=True) + 1e-5).rsqrt()) @ w.t()
    dh = torch.zeros(rows, k, dtype=torch.bfloat16, device="cuda")
    errors = []
    for step in range(1, steps + 1):
        x, r = draw(rows), draw(rows)
        y = block.forward(x, r, stream)
        miss = y.float() - target(block.h.float())
        if step in (1, steps):
            errors.append(float(miss.square().mean()))
        block.backward((miss * (2.0 / rows)).bfloat16(), dh, stream)
        ctx.grad_norm(optimizer, 0.0, 10.0, clip, stream=stream)
        ctx.lstep_adamw(optimizer, lr=lr, weight_decay=0.0, step=step, clip=clip, stream=stream)
    # one token: the pass is captured once and replayed for every further one
    one = Block(ctx, weight, 1, rank, g)
    one.gain.copy_(block.gain)
    for mine, other in zip(one.copy, block.copy):
        mine.copy_(other)
    x, r = draw(1), draw(1)
    one.forward(x, r, stream)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        one.forward(x, r, torch.cuda.current_stream())
    x.copy_(draw(1))
    graph.replay()
    served = float((one.y.float() - target(one.h.float())).square().mean())
    torch.cuda.synchronize()
    del graph
    ctx.close()
    return {"before": errors[0], "after": errors[-1], "served": served}


if __name__ == "__main__":
    print("mean squared error against the uncompressed block: before %(before).4f, after %(after).4f, one served token %(served).4f"
          % train(int(sys.argv[1]) if len(sys.argv) > 1 else 60))
