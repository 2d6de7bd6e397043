"""The 8-bit operators in a run, as a block uses them: gradients against the formulas in 64 bits, captured passes, streams, the C-step
that the codes belong to."""
import os
import sys

import numpy as np
import pytest

from coded_util import GROUP, encode, f64, read, spread, values

pytestmark = pytest.mark.gpu
sys.path.insert(0, os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "examples"))


@pytest.fixture()
def ctx():
    from paper_1911_02497_b200 import cstep
    c = cstep.Context(0)
    yield c
    c.close()


def _block(ctx, rows, k=300, n=520, rank=8, seed=0):
    import torch
    import compressed_block as example
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    w = (torch.rand(n, k, device="cuda", generator=g) * 2 - 1) * 0.1
    weight, theta, lam = example.compress(ctx, w)
    block = example.Block(ctx, weight, rows, rank, g)
    block.gain += 0.2 * torch.randn(k, device="cuda", generator=g)
    block.copy[1].copy_(torch.randn(n, rank, device="cuda", generator=g) * 0.05)
    draw = lambda width, size=1.0: (torch.randn(rows, width, device="cuda", generator=g) * size).bfloat16()
    return block, (w, theta, lam), (draw(k), draw(k), draw(n, 0.01), draw(k, 0.01))


def test_the_example_runs():
    import compressed_block as example
    out = example.train(steps=3, rows=64)
    assert all(np.isfinite(v) for v in out.values())


def test_codes_and_multipliers_of_a_c_step(ctx):
    """theta holds what the codes stand for, lambda <- -mu (w - theta) goes by it (mu = 1e-3, single fp32 operations)."""
    _, (w, theta, lam), _ = _block(ctx, 3)
    W = f64(w)
    kept = np.abs(W) >= np.sort(np.abs(W).ravel())[W.size // 2]
    q, s = encode(np.where(kept, W, 0.0), GROUP)
    assert np.array_equal(f64(theta), q * 2.0 ** (spread(s, GROUP, q.shape) - 127.0))
    d = w.cpu().numpy() - theta.cpu().numpy()
    assert np.array_equal(lam.cpu().numpy(), -(np.float32(1e-3) * d))


@pytest.mark.parametrize("rows", [1, 70, 600])
def test_gradients_of_the_block(ctx, rows):
    """Each result from the 16-bit and 8-bit values that it is formed from: half a step of bfloat16 (2^-8, two of them where the adapter
    adds to what the projection wrote) of its value, and fp32 sums of up to 520 terms (cut: 33 * 2^-24 of the magnitudes for 32, see the
    projection's tests), 16-bit parts of the adapter's coefficients (2^-16)."""
    block, _, (x, r, dy, dh) = _block(ctx, rows)
    y = f64(block.forward(x, r))
    dx = f64(block.backward(dy, dh))
    W, gain, A, B = values(block.weight), f64(block.gain), f64(block.copy[0]), f64(block.copy[1])
    h, z, z8, dy8 = f64(block.h), f64(block.z), values(block.z8), values(block.dy8)
    eps, step = (33 * 520 / 32 + 40) * 2.0 ** -24 + 2.0 ** -15, 2.0 ** -8
    # the norm's two results hold the same values
    R = 1.0 / np.sqrt((h ** 2).mean(axis=1, keepdims=True) + 1e-5)
    assert np.all(np.abs(z - h * R * gain) <= 1.01 * step * np.abs(z) + 1e-30)
    most = np.abs(h * R * gain).max(axis=1, keepdims=True)
    assert np.all(np.abs(z8 - h * R * gain) <= 2.0 ** -4 * np.abs(h * R * gain) + most * 2.0 ** -17)
    want, size = z8 @ W.T + 2.0 * (z @ A.T) @ B.T, np.abs(z8) @ np.abs(W).T + 2.0 * (np.abs(z) @ np.abs(A).T) @ np.abs(B).T
    assert np.all(np.abs(y - want) <= 1.01 * step * (np.abs(want) + np.abs(z8 @ W.T)) + eps * size)
    dz = f64(block.dz)
    want = dy8 @ W + 2.0 * (f64(dy) @ B) @ A
    size = np.abs(dy8) @ np.abs(W) + 2.0 * (np.abs(f64(dy)) @ np.abs(B)) @ np.abs(A)
    assert np.all(np.abs(dz - want) <= 1.01 * step * (np.abs(want) + np.abs(dy8 @ W)) + eps * size)
    t, unit = dz * gain, h * R
    want = f64(dh) + R * (t - unit * (t * unit).mean(axis=1, keepdims=True))
    size = np.abs(f64(dh)) + R * (np.abs(t) + np.abs(unit) * np.abs(t * unit).mean(axis=1, keepdims=True))
    assert np.all(np.abs(dx - want) <= 1.01 * step * np.abs(want) + 60 * 2.0 ** -24 * size)
    assert np.all(np.abs(f64(block.grad[0]) - (dz * unit).sum(axis=0)) <= (rows + 60) * 2.0 ** -24 * np.abs(dz * unit).sum(axis=0) + 1e-30)
    da = 2.0 * (f64(dy) @ B).T @ z
    assert np.all(np.abs(f64(block.grad[1]) - da) <= (rows + 1200) * 2.0 ** -24 * (2.0 * (np.abs(f64(dy)) @ np.abs(B)).T @ np.abs(z)) + 1e-30)


@pytest.mark.parametrize("rows", [1, 70, 600])
def test_captured_passes_of_two_graphs(ctx, rows):
    """Forward and backward captured, in two graphs that share the context's workspace, replayed in turn with new inputs."""
    import torch
    blocks = [_block(ctx, rows, seed=s) for s in (1, 2)]
    outputs = lambda b: [b.y, b.h, b.z, b.dx, b.dz, *b.grad, b.z8.codes.view(torch.uint8), b.z8.scales, b.dy8.scales]
    want = []
    for b, _, (x, r, dy, dh) in blocks:
        b.forward(x, r)
        b.backward(dy, dh)
        want.append([t.clone() for t in outputs(b)])
    torch.cuda.synchronize()
    graphs = []
    for b, _, (x, r, dy, dh) in blocks:
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            s = torch.cuda.current_stream()
            b.forward(x, r, s)
            b.backward(dy, dh, s)
        graphs.append(g)
    large = _block(ctx, 4000, seed=3)                       # outgrows the workspace that the graphs know
    large[0].forward(*large[2][:2])
    large[0].backward(*large[2][2:])
    for _ in range(2):
        for (b, _, (x, r, dy, dh)), g, expected in zip(blocks, graphs, want):
            for t in outputs(b):
                t.zero_()
            g.replay()
            torch.cuda.synchronize()
            assert all(torch.equal(p, q) for p, q in zip(outputs(b), expected))
            kept = x.clone()
            x.neg_(), r.neg_()                              # new inputs: the other sign throughout
            g.replay()
            torch.cuda.synchronize()
            assert torch.equal(b.h, -expected[1]) and torch.equal(b.z, -expected[2])
            x.copy_(kept), r.neg_()
    del graphs, g


def test_two_streams_at_once(ctx):
    """Calls without a workspace on two streams of one context, neither waiting for the other."""
    import torch
    blocks = [_block(ctx, rows, seed=s) for rows, s in ((600, 1), (3, 2))]
    want = []
    for b, _, (x, r, dy, _) in blocks:
        b.forward(x, r)
        want.append(b.y.clone())
    streams = [torch.cuda.Stream() for _ in blocks]
    torch.cuda.synchronize()
    for _ in range(20):
        for (b, _, (x, r, _, _)), s in zip(blocks, streams):
            b.forward(x, r, s)
    torch.cuda.synchronize()
    assert all(torch.equal(b.y, w) for (b, _, _), w in zip(blocks, want))


def test_backward_on_another_stream_waits_for_the_workspace(ctx):
    """The sums for the gain go through the context's workspace: calls on other streams are ordered behind one another."""
    import torch
    b, _, (x, r, dy, dh) = _block(ctx, 600, k=1500)
    b.forward(x, r)
    b.backward(dy, dh)
    torch.cuda.synchronize()
    want = b.grad[0].clone()
    outs = [torch.zeros_like(want) for _ in range(8)]
    streams = [torch.cuda.Stream() for _ in outs]
    for o, s in zip(outs, streams):
        ctx.norm_backward(b.dz, b.h, b.gain, b.rstd, dgain=o, stream=s)
    torch.cuda.synchronize()
    assert all(torch.equal(o, want) for o in outs)
