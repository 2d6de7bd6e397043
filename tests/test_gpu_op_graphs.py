"""Captured calls of the operators, replayed after calls that outgrew the workspace which the capture knew."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu


def _inputs(torch, rows, k, n, ranks, seed):
    """Adapters whose B must be laid out anew (odd ranks), a batch, and everything the calls write."""
    gen = torch.Generator(device="cuda")
    gen.manual_seed(seed)
    draw = lambda *s: torch.randn(*s, device="cuda", generator=gen)
    t = torch.bfloat16
    s = dict(a=[(draw(r, k) / k ** 0.5).to(t) for r in ranks], b=[(draw(n, r) * 0.1).to(t) for r in ranks], x=draw(rows, k).to(t),
             y=draw(rows, n).to(t), dy=draw(rows, n).to(t), dx=draw(rows, k).to(t), h=torch.zeros(rows, max(ranks), device="cuda"),
             ga=[torch.zeros(r, k, device="cuda") for r in ranks], gb=[torch.zeros(n, r, device="cuda") for r in ranks],
             clip=torch.zeros(4, device="cuda"), norms=torch.zeros(2 * len(ranks), device="cuda"))
    share = rows // len(ranks)
    s["rows"] = np.array([share] * (len(ranks) - 1) + [rows - share * (len(ranks) - 1)], dtype=np.int64)
    s["which"] = np.arange(len(ranks), dtype=np.int32)
    return s


def _calls(ctx, s, stream=None):
    from paper_1911_02497_b200 import cstep
    tab = cstep.adapter_table(s["a"], s["b"], [0.5] * len(s["a"]), s["ga"], s["gb"])
    ctx.adapter_forward(tab, s["rows"], s["which"], s["x"], s["y"], s["h"], stream=stream)
    ctx.adapter_backward(tab, s["rows"], s["which"], s["x"], s["dy"], s["h"], s["dx"], stream=stream)
    grads = s["ga"] + s["gb"]
    ctx.grad_norm(cstep.adamw_table(grads, grads), 0.0, 1.0, s["clip"], s["norms"], stream=stream)


def test_a_replay_after_the_workspace_has_grown():
    import torch
    from paper_1911_02497_b200 import cstep
    ctx = cstep.Context(0)
    small = lambda: _inputs(torch, 90, 200, 136, [5, 7], 1)
    want, got = small(), small()
    _calls(ctx, want)                                   # plain, and the call that a capture needs ahead of it
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        _calls(ctx, got, torch.cuda.current_stream())
    large = _inputs(torch, 20000, 256, 192, [33, 64], 2)
    _calls(ctx, large)
    taken = [torch.full((1 << 20,), float("nan"), device="cuda") for _ in range(8)]      # what has been freed is soon somebody else's
    torch.cuda.synchronize()
    g.replay()
    torch.cuda.synchronize()
    for key in ("y", "h", "dx", "clip", "norms"):
        assert torch.equal(got[key], want[key]), key
    for p, q in zip(got["ga"] + got["gb"], want["ga"] + want["gb"]):
        assert torch.equal(p, q)
    assert all(bool(torch.isnan(t).all()) for t in taken)
    del g
    ctx.close()
