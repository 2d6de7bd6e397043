"""8-bit moments rounded by chance: the rule of the header bit for bit, and many steps beside 32-bit moments.

Over many steps: a code's step is at most 1/8 of its value. By chance the mean of r = sqrt(v) is kept and its variance grows by up to
|change| * step in a call, so v = mean(r)^2 + variance settles at most 1/16 above its own average (root: 3 %), and once more as
much is left from values that have come down to where they are by a factor of about e. m is not biased at all."""
import numpy as np
import pytest

BLOCK = 256
F, U = np.float32, np.uint64


def _mix(z):
    z = z ^ (z >> U(30))
    z = z * U(0xBF58476D1CE4E5B9)
    z = z ^ (z >> U(27))
    z = z * U(0x94D049BB133111EB)
    return z ^ (z >> U(31))


def random_bits(seed, step, tensor, n):
    """16 bits for m and 16 for r of each element."""
    i = np.arange(n, dtype=U)
    with np.errstate(over="ignore"):
        key = _mix(np.array([seed], U))
        for x in (step, tensor):
            key = _mix(key ^ U(x))
        z = _mix(key ^ (i >> U(1)))
    at = (i & U(1)) * U(16)
    return ((z >> at) & U(0xFFFF)).astype(np.uint32), ((z >> (at + U(32))) & U(0xFFFF)).astype(np.uint32)


def by_chance(y, b):
    """E4M3 values of the scaled values ``y``."""
    a = np.abs(y)
    q = np.where(a < F(2.0 ** -6), F(2.0 ** -6), F(0)).astype(F)
    t = ((a + q).view(np.uint32) + (b << np.uint32(4)) + np.uint32(8)) & np.uint32(0xFFF00000)
    return np.copysign(t.view(F) - q, y)


def encode(x, b, floor):
    """(values of the codes, scales) of one tensor."""
    n = len(x)
    pad = np.zeros(-(-n // BLOCK) * BLOCK, F)
    pad[:n] = x
    e = np.maximum((np.abs(pad).reshape(-1, BLOCK).max(axis=1).view(np.uint32) >> 23).astype(np.int64) - 7, 1).astype(np.uint32)
    scale, inverse = (e << np.uint32(23)).view(F), ((np.uint32(254) - e) << np.uint32(23)).view(F)
    y = (x * np.repeat(inverse, BLOCK)[:n]).astype(F)
    if floor:
        y = np.where(x > 0, np.maximum(y, F(2.0 ** -9)), y)
    return by_chance(y, b), scale


# ------------------------------------------------------------------ the rule itself

def test_the_rule_rounds_to_neighbours_and_keeps_the_mean():
    import torch
    codes = np.unique(torch.arange(127, dtype=torch.uint8).view(torch.float8_e4m3fn).float().numpy())
    codes = codes[codes <= 256]
    rs = np.random.RandomState(0)
    n = 1 << 16
    b, _ = random_bits(5, 3, 1, n)
    for y in list(np.exp(rs.uniform(np.log(2.0 ** -11), np.log(255.9), 60))) + [2.0 ** -6, 2.0 ** -9, 1.0, 255.9999]:
        y = F(y)
        got = by_chance(np.full(n, y), b)
        lo, hi = codes[codes <= y].max(), codes[codes >= y].min()
        assert set(np.unique(got)) <= {lo, hi}, y
        # the mean of n draws: four standard deviations, and the 2^-17 that 16 bits leave
        assert abs(got.astype(np.float64).mean() - float(y)) <= (hi - lo) * (4 * 0.5 / np.sqrt(n) + 2.0 ** -16)
        assert np.array_equal(by_chance(np.full(n, -y), b), -got)
    assert np.array_equal(by_chance(codes, b[:len(codes)]), codes)          # what a code holds stays


def test_random_bits_of_elements_steps_and_tensors_are_unrelated():
    n = 1 << 16
    sets = [random_bits(*k, n)[i].astype(np.float64) / 65536 for k in ((1, 1, 0), (1, 2, 0), (2, 1, 0), (1, 1, 1)) for i in (0, 1)]
    for i, x in enumerate(sets):
        assert abs(x.mean() - 0.5) < 5 / np.sqrt(12 * n)
        assert abs(np.corrcoef(x[:-1], x[1:])[0, 1]) < 5 / np.sqrt(n) and abs(np.corrcoef(x[:-2], x[2:])[0, 1]) < 5 / np.sqrt(n)
        for y in sets[:i]:
            assert abs(np.corrcoef(x, y)[0, 1]) < 5 / np.sqrt(n)


def test_the_binding_checks_the_seed_and_tells_of_the_other_rounding():
    import warnings

    from paper_1911_02497_b200 import cstep

    class Library:
        def __getattr__(self, name):
            return lambda *args: 0
    ctx = cstep.Context.__new__(cstep.Context)
    ctx._lib, ctx._h = Library(), None
    tab = cstep.AdamwTable(1)
    tab.state_dtype = cstep.DTYPE_FP8_E4M3
    for bad in (-1, 1 << 32):
        with pytest.raises(ValueError):
            ctx.lstep_adamw(tab, state_seed=bad)
    with warnings.catch_warnings(record=True) as told:
        warnings.simplefilter("always")
        ctx.lstep_adamw(tab, step=1)
        ctx.lstep_adamw(tab, step=2, state_seed=1)
        assert not told
        ctx.lstep_adamw(tab, step=2)
        ctx.lstep_adamw(tab, step=3)
        assert len(told) == 1 and "state_seed" in str(told[0].message)
    tab.state_dtype = cstep.DTYPE_FP32
    fresh = cstep.Context.__new__(cstep.Context)
    fresh._lib, fresh._h = Library(), None
    with warnings.catch_warnings():
        warnings.simplefilter("error")
        fresh.lstep_adamw(tab, step=2)


# ------------------------------------------------------------------ on the GPU

@pytest.fixture()
def ctx():
    from paper_1911_02497_b200 import cstep
    c = cstep.Context(0)
    yield c
    c.close()


class State:
    """Weights, 8-bit moments and gradients of a list on the device."""

    def __init__(self, sizes, grad="float32", penalty=False, off=0):
        import torch
        self.sizes, self.off = sizes, off
        put = lambda n, t: torch.zeros(off + n, dtype=t, device="cuda")[off:]
        self.w, self.grad = [put(n, torch.float32) for n in sizes], [put(n, getattr(torch, grad)) for n in sizes]
        self.m, self.v = ([put(n, torch.uint8).view(torch.float8_e4m3fn) for n in sizes] for _ in range(2))
        self.ms, self.vs = ([torch.zeros(-(-n // BLOCK), device="cuda") for n in sizes] for _ in range(2))
        self.theta = [put(n, torch.float32) for n in sizes] if penalty else None

    def table(self):
        from paper_1911_02497_b200 import cstep
        return cstep.adamw_table(self.w, self.grad, self.m, self.v, self.ms, self.vs, theta=self.theta)

    def buffers(self):
        return self.w + self.m + self.v + self.ms + self.vs


@pytest.mark.gpu
@pytest.mark.parametrize("grad", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("penalty", [False, True])
@pytest.mark.parametrize("off", [0, 1])
def test_codes_and_scales_are_the_header_s_bit_for_bit(ctx, grad, penalty, off):
    """Five steps from zero states; every operation up to the codes is a single fp32 one, so numpy has the same bits."""
    import torch
    sizes = [1, 255, 256, 257, 0, 5000, 12289, 70001] + [3] * 360
    S, rs = State(sizes, grad, penalty, off), np.random.RandomState(4)
    b1, b2, mu, gs = F(0.9), F(0.95), F(1e-2), F(0.5)
    state = [(np.zeros(n, F), np.zeros(n, F)) for n in sizes]
    for step in range(1, 6):
        for t, n in enumerate(sizes):
            g = (rs.standard_normal(n) * 0.02 * 10.0 ** rs.uniform(-3, 1, n)).astype(F)
            g[rs.rand(n) < 0.1] = 0
            S.grad[t].copy_(torch.from_numpy(g))
            w = S.w[t].cpu().numpy()
            g = gs * S.grad[t].float().cpu().numpy()
            if penalty:
                g = g + (mu * (w - F(0)) - F(0))
            m, r = state[t]
            m = b1 * m + (F(1) - b1) * g
            r = np.sqrt(b2 * (r * r) + (F(1) - b2) * (g * g))
            bm, br = random_bits(77, step, t, n)
            state[t] = (encode(m, bm, False), encode(r, br, True))
        ctx.lstep_adamw(S.table(), float(mu), lr=1e-3, beta1=0.9, beta2=0.95, step=step, grad_scale=0.5, state_seed=77)
        torch.cuda.synchronize()
        for t, n in enumerate(sizes):
            held = []
            for (value, scale), code, got in zip(state[t], (S.m[t], S.v[t]), (S.ms[t], S.vs[t])):
                if n:
                    assert np.array_equal(got.cpu().numpy(), scale), (step, t)
                    assert np.array_equal(code.float().cpu().numpy(), value), (step, t)
                held.append(value * np.repeat(scale, BLOCK)[:n])
            state[t] = tuple(held)


@pytest.mark.gpu
def test_equal_seeds_give_equal_bits_others_do_not(ctx):
    import torch
    runs = []
    for seed in (3, 3, 4):
        S = State([5000, 300])
        torch.manual_seed(0)
        for step in range(1, 4):
            for g in S.grad:
                g.copy_(torch.randn_like(g))
            ctx.lstep_adamw(S.table(), step=step, state_seed=seed)
        runs.append([x.view(torch.uint8).clone() for x in S.buffers()])
    torch.cuda.synchronize()
    assert all(torch.equal(x, y) for x, y in zip(runs[0], runs[1]))
    assert not torch.equal(runs[0][2], runs[2][2]) and not torch.equal(runs[0][4], runs[2][4])


@pytest.mark.gpu
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_a_bad_gradient_stays_in_its_element(ctx, bad):
    import torch
    a, b = State([700]), State([700])
    torch.manual_seed(0)
    g = torch.randn(700, device="cuda")
    for S in (a, b):
        S.grad[0].copy_(g)
    a.grad[0][300] = bad
    # (the block's largest value is another element's in both)
    for S in (a, b):
        S.grad[0][301] = 9.0
        ctx.lstep_adamw(S.table(), step=1, state_seed=11)
    torch.cuda.synchronize()
    keep = torch.arange(700, device="cuda") != 300
    assert torch.isnan(a.m[0].float()[300]) and torch.isnan(a.v[0].float()[300]) and torch.isnan(a.w[0][300])
    for x, y in zip(a.buffers()[:3], b.buffers()[:3]):
        assert torch.equal(x.float()[keep], y.float()[keep])
    assert torch.equal(a.ms[0], b.ms[0]) and torch.equal(a.vs[0], b.vs[0])


@pytest.mark.gpu
@pytest.mark.parametrize("beta2", [0.95, 0.999])
def test_a_thousand_steps_follow_the_32_bit_moments(ctx, beta2):
    """A thousand steps of noise about a small slope, then a thousand more at a tenth of the size."""
    import torch
    from paper_1911_02497_b200 import cstep
    n = 40_000
    S = State([n])
    w, m, v = (torch.zeros(n, device="cuda") for _ in range(3))
    grad = torch.zeros(n, device="cuda")
    torch.manual_seed(2)
    slope = torch.where(torch.rand(n, device="cuda") < 0.5, 0.3, -0.3)
    plain, tab = cstep.adamw_table([w], [grad], [m], [v]), S.table()
    moved = []
    for phase, size in enumerate((1.0, 0.1)):
        from8, from32 = S.w[0].clone(), w.clone()
        for step in range(1 + 1000 * phase, 1001 + 1000 * phase):
            grad.normal_().add_(slope).mul_(size)
            S.grad[0].copy_(grad)
            for table, seed in ((plain, 0), (tab, 9)):
                ctx.lstep_adamw(table, lr=1e-3, beta1=0.9, beta2=beta2, weight_decay=0.0, step=step, state_seed=seed)
        r8 = S.v[0].double() * S.vs[0].double().repeat_interleave(BLOCK)[:n]
        m8 = S.m[0].double() * S.ms[0].double().repeat_interleave(BLOCK)[:n]
        ratio = float((r8.square().mean() / v.double().mean()).sqrt())
        assert 0.97 <= ratio <= 1.07, (phase, ratio)
        # m: the mean along the slope. Its noise, 0.23 of the gradient's (and the rounding's, less than that), is averaged over n
        along8, along32 = float((m8 * slope.sign()).mean()), float((m.double() * slope.sign()).mean())
        assert abs(along8 - along32) <= 5 * 0.35 * size / np.sqrt(n), (phase, along8, along32)
        moved.append((float(((S.w[0] - from8) * slope.sign()).double().mean()), float(((w - from32) * slope.sign()).double().mean())))
    torch.cuda.synchronize()
    # a step is m / r: r's root mean square up to 7 % above and its relative variance up to 1/16 twice over
    for got, want in moved:
        assert 0.93 <= got / want <= 1.13, moved
