"""AdamW over a tensor list (32- and 8-bit states) and the gradient norm, against the formulas in 64 bits.

Tolerances come from the arithmetic: every value is a short chain of single fp32 operations, so its error is a few units
of 2^-24 of the magnitudes that enter it. An 8-bit state lies within half a step of its format around the 64-bit value."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
BLOCK = 256


def _torch():
    import torch
    return torch


@pytest.fixture()
def ctx():
    from paper_1911_02497_b200 import cstep
    c = cstep.Context(0)
    yield c
    c.close()


class Lists:
    """Device lists with guard elements around every array; `off` elements ahead of each."""

    def __init__(self, sizes, seed, grad="float32", states=32, penalty=False, copy=None, off=0, zero_state=False):
        torch = _torch()
        rs = np.random.RandomState(seed)
        self.sizes, self.states, self.copy_type = sizes, states, copy
        self.held = []
        self.host = {k: [] for k in ("w", "grad", "theta", "lam", "m", "v")}
        self.dev = {k: [] for k in ("w", "grad", "theta", "lam", "m", "v", "m_scale", "v_scale", "w_h")}
        for i, n in enumerate(sizes):
            w = (rs.standard_normal(n) * 0.05).astype(np.float32)
            g = (rs.standard_normal(n) * 0.02 * (1 + i % 3)).astype(np.float32)
            g[rs.rand(n) < 0.1] = 0
            m = (rs.standard_normal(n) * 0.01).astype(np.float32)
            v = ((rs.standard_normal(n) * 0.02) ** 2).astype(np.float32)
            if zero_state:
                m[:], v[:] = 0, 0
            has_th = penalty and i % 3 != 2
            th = np.where(np.abs(w) > 0.04, w, 0).astype(np.float32) if has_th else None
            lam = (rs.standard_normal(n) * 1e-3).astype(np.float32) if has_th and i % 2 == 0 else None
            gd = torch.from_numpy(g).to(getattr(torch, grad))
            self.host["grad"].append(gd.double().numpy())
            for key, a in (("w", w), ("theta", th), ("lam", lam)):
                self.host[key].append(None if a is None else a.astype(np.float64))
                self.dev[key].append(None if a is None else self.put(torch.from_numpy(a), off))
            self.dev["grad"].append(self.put(gd, off))
            if states == 32:
                for key, a in (("m", m), ("v", v)):
                    self.host[key].append(a.astype(np.float64))
                    self.dev[key].append(self.put(torch.from_numpy(a), off))
                self.dev["m_scale"].append(None), self.dev["v_scale"].append(None)
            else:
                for key, a in (("m", m), ("v", np.sqrt(v))):
                    nb = -(-n // BLOCK)
                    pad = np.zeros(nb * BLOCK)
                    pad[:n] = a
                    most = np.abs(pad.reshape(nb, BLOCK)).max(axis=1)
                    scale = np.exp2(np.maximum(np.frexp(most)[1] - 8, -126.0)).astype(np.float32)
                    code = torch.from_numpy((pad.reshape(nb, BLOCK) / scale[:, None]).astype(np.float32)).to(torch.float8_e4m3fn)
                    value = code.double().numpy() * scale[:, None]
                    value = value.reshape(-1)[:n]
                    self.host[key].append(value if key == "m" else value ** 2)
                    self.dev[key].append(self.put(code.reshape(-1)[:n].view(torch.uint8), off).view(torch.float8_e4m3fn))
                    self.dev[key + "_scale"].append(self.put(torch.from_numpy(scale), 0))
            self.dev["w_h"].append(None if copy is None else self.put(torch.zeros(n, dtype=getattr(torch, copy)), off))

    def put(self, t, off):
        torch = _torch()
        room = torch.full((off + t.numel() + 64,), 93, dtype=torch.uint8).repeat_interleave(t.element_size()).view(t.dtype).cuda()
        room[off:off + t.numel()] = t.cuda()
        self.held.append((room, off, t.numel()))
        return room[off:off + t.numel()]

    def guards_intact(self):
        torch = _torch()
        for room, off, n in self.held:
            b = room.view(torch.uint8)
            e = room.element_size()
            if not (bool((b[:off * e] == 93).all()) and bool((b[(off + n) * e:] == 93).all())):
                return False
        return True

    def table(self):
        from paper_1911_02497_b200 import cstep
        d = self.dev
        return cstep.adamw_table(d["w"], d["grad"], d["m"], d["v"], d["m_scale"], d["v_scale"], d["theta"], d["lam"], d["w_h"])


def gradient(L, t, mu, gs):
    """The 64-bit gradient and the magnitude its fp32 error is measured by."""
    g = gs * L.host["grad"][t]
    size = np.abs(g)
    if L.host["theta"][t] is not None:
        w, th = L.host["w"][t], L.host["theta"][t]
        lam = L.host["lam"][t] if L.host["lam"][t] is not None else 0.0
        g = g + mu * (w - th) - lam
        size = size + np.abs(mu) * (np.abs(w) + np.abs(th)) + np.abs(lam)
    return g, size


def half_step(x, scale):
    """Half the distance of neighbouring E4M3 values around x, under `scale`; subnormal below 2^-6."""
    e = np.maximum(np.floor(np.log2(np.maximum(np.abs(x) / scale, 1e-30))), -6)
    return np.exp2(e - 4) * scale


def step_and_check(ctx, L, mu, clip=None, gs=1.0, stream=None, **kw):
    torch = _torch()
    p = dict(lr=1e-2, beta1=0.9, beta2=0.99, eps=1e-8, weight_decay=0.1, step=3)
    p.update(kw)
    dev_clip = None if clip is None else torch.tensor([9.0, clip, 1.0, 0.0], device="cuda")
    ctx.lstep_adamw(L.table(), mu, clip=dev_clip, grad_scale=gs, stream=stream, **p)
    torch.cuda.synchronize()
    assert L.guards_intact()
    b1, b2, lr, eps, wd = (float(np.float32(p[k])) for k in ("beta1", "beta2", "lr", "eps", "weight_decay"))
    coef, gs = float(np.float32(1.0 if clip is None else clip)), float(np.float32(gs))
    mu = float(np.float32(mu))
    for t, n in enumerate(L.sizes):
        if n == 0:
            continue
        g, size = gradient(L, t, mu, gs)
        g, size = coef * g, coef * size
        m0, v0, w0 = L.host["m"][t], L.host["v"][t], L.host["w"][t]
        c1, c2 = float(np.float32(1) - np.float32(b1)), float(np.float32(1) - np.float32(b2))
        m, v = b1 * m0 + c1 * g, b2 * v0 + c2 * g * g
        em = 8 * EPS * (np.abs(b1 * m0) + c1 * size)                     # five operations on the gradient, two here, one sum
        ev = 4 * EPS * b2 * v0 + c2 * (14 * EPS * size * np.abs(g) + (7 * EPS * size) ** 2)
        root = np.sqrt(v)
        eroot = np.where(v > 0, ev / np.maximum(root, 1e-300), np.sqrt(ev)) + 2 * EPS * root
        corr, step = 1 / np.sqrt(1 - b2 ** p["step"]), lr / (1 - b1 ** p["step"])
        den = root * corr + eps
        w = w0 * (1 - lr * wd) - step * m / den
        with np.errstate(divide="ignore", invalid="ignore"):
            ew = 3 * EPS * np.abs(w0) + step * (em / den + np.abs(m) / den * (eroot * corr / den + 8 * EPS)) + EPS * np.abs(w)
        got = L.dev["w"][t].double().cpu().numpy()
        assert np.all(np.abs(got - w) <= ew + 1e-37), (t, n, np.max(np.abs(got - w) / (ew + 1e-300)))
        if L.copy_type:
            got_h = L.dev["w_h"][t].cpu()
            assert torch.equal(got_h, L.dev["w"][t].cpu().to(got_h.dtype))
        if L.states == 32:
            assert np.all(np.abs(L.dev["m"][t].double().cpu().numpy() - m) <= em + 1e-44)
            assert np.all(np.abs(L.dev["v"][t].double().cpu().numpy() - v) <= ev + 1e-44)
            continue
        for key, x, ex in (("m", m, em), ("v", root, eroot)):
            nb = -(-n // BLOCK)
            scale = L.dev[key + "_scale"][t].double().cpu().numpy()
            pad, epad = np.zeros(nb * BLOCK), np.zeros(nb * BLOCK)
            pad[:n], epad[:n] = np.abs(x), ex
            most, slack = pad.reshape(nb, BLOCK).max(axis=1), epad.reshape(nb, BLOCK).max(axis=1)
            lo, hi = (np.exp2(np.maximum(np.frexp(np.maximum(q, 0))[1] - 8, -126.0)) for q in (most - slack, most + slack))
            zero = most <= slack
            assert np.all((scale >= lo) & (scale <= hi) | zero), key
            s = np.repeat(scale, BLOCK)[:n]
            got = L.dev[key][t].double().cpu().numpy() * s
            allowed = half_step(np.abs(x) + ex, s) + ex
            if key == "v":                          # a positive root keeps the smallest code
                allowed = np.where((x > 0) & (got == s * 2.0 ** -9), np.maximum(allowed, s * 2.0 ** -9), allowed)
                assert np.all(got[x > ex] > 0)
            assert np.all(np.abs(got - x) <= allowed), (key, t)


SIZES = [1, 255, 256, 257, 0, 2048, 5000, 3, 12289, 70001]


@pytest.mark.parametrize("states", [32, 8])
@pytest.mark.parametrize("grad", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("penalty", [False, True])
@pytest.mark.parametrize("off", [0, 4, 1])
def test_step_matches_the_formula(ctx, states, grad, penalty, off):
    copy = {"float32": None, "float16": "float16", "bfloat16": "bfloat16"}[grad]
    L = Lists(SIZES, 5 + off, grad, states, penalty, copy, off)
    step_and_check(ctx, L, 1e-2, clip=0.37 if off else None, gs=0.5)


@pytest.mark.parametrize("states", [32, 8])
def test_first_step_from_zero_states_and_long_lists(ctx, states):
    """More tensors than one launch holds (360), from the zero states that an optimizer starts with."""
    rs = np.random.RandomState(3)
    sizes = [int(x) for x in rs.randint(0, 600, 771)]
    L = Lists(sizes, 4, "float32", states, True, "bfloat16", 0, zero_state=True)
    step_and_check(ctx, L, 1e-3, step=1)


@pytest.mark.parametrize("states", [32, 8])
def test_a_large_tensor_and_another_stream(ctx, states):
    """Several work items per CTA and chunks per item; the call on a stream that is not the default one."""
    torch = _torch()
    L = Lists([7_000_003, 900], 8, "bfloat16", states, False, "bfloat16")
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    step_and_check(ctx, L, 0.0, stream=s)


@pytest.mark.parametrize("states", [32, 8])
def test_a_step_that_overflowed_is_skipped(ctx, states):
    torch = _torch()
    L = Lists([1000, 300], 1, "float32", states, False, "float16")
    L.dev["grad"][1][17] = float("inf")
    before = {k: [None if x is None else x.clone() for x in L.dev[k]] for k in L.dev}
    clip = torch.zeros(4, device="cuda")
    ctx.grad_norm(L.table(), 0.0, 1.0, clip)
    ctx.lstep_adamw(L.table(), clip=clip)
    torch.cuda.synchronize()
    assert clip[2].item() == 0.0 and not np.isfinite(clip[0].item()) and clip[1].item() == 1.0
    for k in L.dev:
        for x, y in zip(L.dev[k], before[k]):
            assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k


@pytest.mark.parametrize("states", [32, 8])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_bad_gradient_stays_in_its_element(ctx, states, bad):
    """Without a clip record nothing is skipped: the element is lost, its block's scale and neighbours are not."""
    torch = _torch()
    a, b = (Lists([700], 6, "float32", states) for _ in range(2))
    a.dev["grad"][0][300] = bad
    for L in (a, b):
        ctx.lstep_adamw(L.table(), lr=1e-2, step=2)
    torch.cuda.synchronize()
    keep = torch.ones(700, dtype=torch.bool, device="cuda")
    keep[300] = False
    assert torch.equal(a.dev["w"][0][keep], b.dev["w"][0][keep]) and torch.isnan(a.dev["w"][0][300])
    for k in ("m", "v"):
        x, y = a.dev[k][0].float(), b.dev[k][0].float()
        assert not torch.isfinite(x[300])
        if states == 32:
            assert torch.equal(x[keep], y[keep])
        else:
            xs, ys = (L.dev[k + "_scale"][0].repeat_interleave(BLOCK)[:700] for L in (a, b))
            assert torch.isfinite(xs).all() and torch.allclose((x * xs)[keep], (y * ys)[keep], rtol=0.13, atol=0.0)


def test_tiny_and_huge_blocks_keep_their_range(ctx):
    """Blocks whose largest value is subnormal, and near the top of fp32."""
    torch = _torch()
    n = 512
    L = Lists([n], 2, "float32", 8, zero_state=True)
    g = torch.zeros(n, device="cuda")
    g[:256] = torch.linspace(1, 200, 256, device="cuda") * 1e-41
    g[256:] = torch.linspace(-1, 1, 256, device="cuda") * 1e17
    L.dev["grad"][0].copy_(g)
    ctx.lstep_adamw(L.table(), lr=0.0, weight_decay=0.0, beta1=0.5, beta2=0.5, step=1)
    torch.cuda.synchronize()
    m = L.dev["m"][0].double() * L.dev["m_scale"][0].double().repeat_interleave(BLOCK)
    want = g.double() * 0.5
    s = L.dev["m_scale"][0].double().repeat_interleave(BLOCK).cpu().numpy()
    # (the first block's scale is the least one: its codes are steps of 2^-9 * 2^-126; values may underflow)
    assert np.all(np.abs((m - want).cpu().numpy()) <= half_step(want.cpu().numpy(), s) + 2.0 ** -149)
    assert torch.isfinite(L.dev["w"][0]).all()


@pytest.mark.parametrize("grad", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("penalty", [False, True])
@pytest.mark.parametrize("off", [0, 1])
@pytest.mark.parametrize("sizes", [SIZES, [0, 0, 5], [1], [3_000_001], [17] * 800])
def test_norm_matches_the_formula(ctx, grad, penalty, off, sizes):
    torch = _torch()
    L = Lists(sizes, 9, grad, 32, penalty, None, off)
    clip, norms = torch.full((4,), 7.0, device="cuda"), torch.full((len(sizes),), 7.0, device="cuda")
    tab = L.table()
    ctx.grad_norm(tab, 1e-2, 0.25, clip, norms, grad_scale=0.5)
    again, nagain = torch.zeros_like(clip), torch.zeros_like(norms)
    ctx.grad_norm(tab, 1e-2, 0.25, again, nagain, grad_scale=0.5)
    torch.cuda.synchronize()
    assert torch.equal(clip, again) and torch.equal(norms, nagain)
    total = 0.0
    for t, n in enumerate(sizes):
        g, size = gradient(L, t, float(np.float32(1e-2)), 0.5) if n else (np.zeros(1), np.zeros(1))
        want = float(np.sqrt(np.sum(g * g)))
        total += want * want
        assert abs(norms[t].item() - want) <= 6 * EPS * np.sqrt(np.sum(size * size)) + 2 * EPS * want, t
    want = np.sqrt(total)
    size = np.sqrt(sum(np.sum(gradient(L, t, 1e-2, 0.5)[1] ** 2) for t, n in enumerate(sizes) if n))
    assert abs(clip[0].item() - want) <= 6 * EPS * size + 2 * EPS * want
    assert abs(clip[1].item() - min(1.0, 0.25 / (want + 1e-6))) <= 16 * EPS * max(1.0, size / max(want, 1e-30))
    assert clip[2].item() == 1.0 and clip[3].item() == 0.0


def test_norm_of_large_and_tiny_values(ctx):
    """Squares leave the range of fp32 on both sides; the norm does not."""
    torch = _torch()
    for scale, n in ((1e25, 1000), (1e-30, 1000)):
        L = Lists([n], 1)
        L.dev["grad"][0].fill_(scale)
        clip = torch.zeros(4, device="cuda")
        ctx.grad_norm(L.table(), 0.0, 0.0, clip)
        torch.cuda.synchronize()
        want = float(np.float32(scale)) * np.sqrt(n)
        assert abs(clip[0].item() - want) <= 2 * EPS * want and clip[1].item() == 1.0 and clip[2].item() == 1.0
    L = Lists([4], 1)
    L.dev["grad"][0].fill_(3e38)
    ctx.grad_norm(L.table(), 0.0, 1.0, clip)
    torch.cuda.synchronize()
    assert np.isinf(clip[0].item()) and clip[2].item() == 0.0


def test_norm_on_alternating_streams(ctx):
    """The calls share a workspace: each waits for the one before, whatever stream that was on."""
    torch = _torch()
    lists = [Lists([400_000 + 1000 * i], 20 + i) for i in range(4)]
    clips = [torch.zeros(4, device="cuda") for _ in lists]
    tabs = [L.table() for L in lists]
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for _ in range(10):
        for i, (tab, c) in enumerate(zip(tabs, clips)):
            ctx.grad_norm(tab, 0.0, 1.0, c, stream=streams[i % 2])
    torch.cuda.synchronize()
    for L, c in zip(lists, clips):
        want = np.linalg.norm(L.host["grad"][0])
        assert abs(c[0].item() - want) <= 4 * EPS * want


def test_both_calls_in_a_graph(ctx):
    torch = _torch()
    L, M = Lists([5000, 70], 3, "bfloat16", 8, True, "bfloat16"), Lists([5000, 70], 3, "bfloat16", 8, True, "bfloat16")
    clip = torch.zeros(4, device="cuda")

    def both(X, stream):
        ctx.grad_norm(X.table(), 1e-2, 0.1, clip, stream=stream)
        ctx.lstep_adamw(X.table(), 1e-2, clip=clip, step=5, stream=stream)
    for _ in range(3):
        both(L, None)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(M, torch.cuda.current_stream())
    for _ in range(3):
        g.replay()
    torch.cuda.synchronize()
    for k in ("w", "m", "v", "m_scale", "v_scale", "w_h"):
        for x, y in zip(L.dev[k], M.dev[k]):
            assert torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k


def test_refusals(ctx):
    """Nothing is launched and no buffer touched where an argument is wrong."""
    torch = _torch()
    from paper_1911_02497_b200 import cstep
    L = Lists([300, 40], 7, "float32", 8, True, "float16")
    before = {k: [None if x is None else x.clone() for x in L.dev[k]] for k in L.dev}
    launches = ctx.launch_count()

    def refused(code, change=None, mu=1e-2, **kw):
        tab = L.table()
        if change:
            change(tab)
        with pytest.raises(cstep.CondensaError) as e:
            ctx.lstep_adamw(tab, mu, **kw)
        assert e.value.code == code, e.value

    bad, no = cstep.ERR_INVALID_ARG, cstep.ERR_UNSUPPORTED
    for field in ("w", "grad", "m", "v", "m_scale", "v_scale"):
        refused(bad, lambda tab: setattr(tab.entries[1], field, None))
    refused(bad, lambda tab: setattr(tab.entries[0], "w", tab.entries[0].w + 2))
    refused(bad, lambda tab: setattr(tab.entries[0], "w_h", tab.entries[0].w_h + 1))
    refused(bad, lambda tab: setattr(tab.entries[0], "numel", -1))
    refused(bad, lambda tab: setattr(tab.entries[0], "m", tab.entries[0].v))
    refused(bad, lambda tab: setattr(tab.entries[0], "grad", tab.entries[0].w))
    refused(bad, lambda tab: setattr(tab.entries[0], "m_scale", tab.entries[0].v_scale))
    refused(bad, lambda tab: setattr(tab, "T", 0))
    refused(cstep.ERR_TOO_LARGE, lambda tab: setattr(tab.entries[0], "numel", (1 << 40) + 1))
    refused(no, lambda tab: setattr(tab, "grad_dtype", 3))
    refused(no, lambda tab: setattr(tab, "state_dtype", 4))
    refused(no, lambda tab: setattr(tab, "w_h_dtype", 0))
    for kw in (dict(beta1=1.0), dict(beta2=-0.1), dict(step=0), dict(eps=-1.0), dict(lr=float("nan")), dict(weight_decay=float("inf")),
               dict(grad_scale=float("nan")), dict(eps=float("nan")), dict(mu=-1.0), dict(mu=float("nan"))):
        refused(bad, **kw)
    clip = torch.zeros(5, device="cuda")
    with pytest.raises(cstep.CondensaError):
        ctx.grad_norm(L.table(), 1e-2, 1.0, None)
    with pytest.raises(cstep.CondensaError):
        ctx.grad_norm(L.table(), 1e-2, float("nan"), clip)
    with pytest.raises(cstep.CondensaError):
        ctx.grad_norm(L.table(), -1.0, 1.0, clip)
    with pytest.raises(TypeError):
        cstep.adamw_table([torch.zeros(4, device="cuda", dtype=torch.float64)], [torch.zeros(4, device="cuda")])
    with pytest.raises(ValueError):
        cstep.adamw_table([torch.zeros(5, device="cuda")], [torch.zeros(4, device="cuda")])
    with pytest.raises(ValueError):
        cstep.adamw_table([torch.zeros(4, 4, device="cuda").t()], [torch.zeros(4, 4, device="cuda")])
    torch.cuda.synchronize()
    assert ctx.launch_count() == launches and L.guards_intact()
    for k in L.dev:
        for x, y in zip(L.dev[k], before[k]):
            assert x is None or torch.equal(x.view(torch.uint8), y.view(torch.uint8)), k
