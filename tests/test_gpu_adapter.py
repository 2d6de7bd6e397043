"""Low-rank adapters of many requests, forward and backward, against the formulas in 64 bits.

Tolerances come from the arithmetic: products of 16-bit operands are exact, sums run in fp32 (whose matrix instruction
truncates: an error of up to 2^-23 of the running sum per step of 8 or 16 terms), h and u keep at least 16 bits in the second product,
and a 16-bit result is rounded once."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
# relative error of an operand's parts: 22 bits (TF32 pairs, binary16 pairs), 16 bits (bfloat16 pairs)
PART = {"float32": 2.0 ** -21, "float16": 2.0 ** -21, "bfloat16": 2.0 ** -16}


def _torch():
    import torch
    return torch


@pytest.fixture()
def ctx():
    from paper_1911_02497_b200 import cstep
    c = cstep.Context(0)
    yield c
    c.close()


class Batch:
    """A batch in guarded buffers; `pad` extra elements between rows, `off` ahead of the first."""

    def __init__(self, dtype, k, n, requests, ranks, seed=0, pad=0, off=0, scales=None, xs=1.0, dys=0.01):
        torch = _torch()
        self.dtype, self.k, self.n, self.ranks = dtype, k, n, ranks
        self.t = getattr(torch, dtype)
        self.rows = np.array([r for r, _ in requests], dtype=np.int64)
        self.which = np.array([a for _, a in requests], dtype=np.int32)
        self.m = m = int(self.rows.sum())
        self.rs = np.random.RandomState(seed)
        self.held = []
        self.scale = scales or [0.5 + 0.75 * i for i in range(len(ranks))]
        self.a = [self.put(self.draw(r, k) / np.sqrt(k), self.t, off=off) for r in ranks]
        self.b = [self.put(self.draw(n, r) * 0.1, self.t, off=off) for r in ranks]
        self.x = self.put(self.draw(m, k) * xs, self.t, pad, off)
        self.y = self.put(self.draw(m, n), self.t, pad, off)
        self.dy = self.put(self.draw(m, n) * dys, self.t, pad, off)
        self.dx = self.put(self.draw(m, k) * dys, self.t, pad, off)
        self.h = self.put(np.full((m, max(ranks)), 7.0), torch.float32, 1 if off else 0, off)
        self.ga = [self.put(self.draw(r, k), torch.float32, off=off) for r in ranks]
        self.gb = [self.put(self.draw(n, r), torch.float32, off=off) for r in ranks]
        self.row_of = np.repeat(self.which, self.rows)

    def draw(self, *shape):
        return self.rs.standard_normal(shape)

    def put(self, a, t, pad=0, off=0):
        torch = _torch()
        m, w = a.shape
        size = torch.zeros(0, dtype=t).element_size()
        room = torch.full(((off + m * (w + pad) + 64) * size,), 93, dtype=torch.uint8, device="cuda").view(t)
        v = torch.as_strided(room, (m, w), (w + pad, 1), off)
        v.copy_(torch.from_numpy(a).to(t))
        mask = torch.ones(room.numel(), dtype=torch.bool, device="cuda")
        torch.as_strided(mask, (m, w), (w + pad, 1), off)[:] = False
        self.held.append((room, mask, size))
        return v

    def guards_intact(self):
        for room, mask, size in self.held:
            if not bool((room.view(_torch().uint8).view(-1, size)[mask] == 93).all()):
                return False
        return True

    def table(self, grads=True):
        from paper_1911_02497_b200 import cstep
        return cstep.adapter_table(self.a, self.b, self.scale, self.ga if grads else None, self.gb if grads else None)


def f64(t):
    return t.detach().double().cpu().numpy()


def within(got, want, err, t):
    """`got` is a value within `err` of `want`, rounded once to type `t` (rounding keeps order)."""
    torch = _torch()
    lo, hi = (torch.from_numpy(v).to(t).double().numpy() for v in (want - err, want + err))
    assert np.all((got >= lo) & (got <= hi)), np.max(np.maximum(lo - got, got - hi) / (np.abs(want) + err))


def steps(n):
    """Sums of n terms by steps of 8 in up to 64 partial sums, each truncated: units of 2^-24."""
    return 2 * (n / 8 + 80)


def check_forward(ctx, B, keep_h=True, stream=None):
    torch = _torch()
    x, y0, h0 = f64(B.x), f64(B.y), f64(B.h)
    ctx.adapter_forward(B.table(False), B.rows, B.which, B.x, B.y, B.h if keep_h else None, stream=stream)
    torch.cuda.synchronize()
    assert B.guards_intact()
    y, h = f64(B.y), f64(B.h)
    idle = B.row_of < 0
    assert np.array_equal(y[idle], y0[idle]) and np.array_equal(h[idle], h0[idle])
    for i, r in enumerate(B.ranks):
        at = B.row_of == i
        if not at.any():
            continue
        a, b, s = f64(B.a[i]), f64(B.b[i]), float(np.float32(B.scale[i]))
        hw, size = x[at] @ a.T, np.abs(x[at]) @ np.abs(a).T
        eh = (steps(B.k) * EPS + (0 if B.dtype != "float32" else 4 * PART["float32"])) * size
        if keep_h:
            assert np.all(np.abs(h[at][:, :r] - hw) <= eh), (i, np.max(np.abs(h[at][:, :r] - hw) / eh))
            assert np.array_equal(h[at][:, r:], h0[at][:, r:])
        want = y0[at] + s * hw @ b.T
        mag = np.abs(s) * (np.abs(hw) + eh) @ np.abs(b).T
        err = np.abs(s) * eh @ np.abs(b).T + (2 * PART[B.dtype] + steps(r) * EPS) * mag
        within(y[at], want, err + 2 * EPS * (np.abs(want) + err), B.t)


def check_backward(ctx, B, accumulate=False, with_dx=True, seed=1):
    torch = _torch()
    for i, r in enumerate(B.ranks):                 # h as a forward pass would have left it (fp32, rounded here)
        at = B.row_of == i
        full = f64(B.x)[at] @ f64(B.a[i]).T
        B.h[torch.from_numpy(np.flatnonzero(at)).cuda(), :r] = torch.from_numpy(full).float().cuda()
    dy, dx0, h, x = f64(B.dy), f64(B.dx), f64(B.h), f64(B.x)
    ga0, gb0 = [f64(g) for g in B.ga], [f64(g) for g in B.gb]
    ctx.adapter_backward(B.table(), B.rows, B.which, B.x, B.dy, B.h, B.dx if with_dx else None, accumulate=accumulate)
    torch.cuda.synchronize()
    assert B.guards_intact()
    dx = f64(B.dx)
    idle = B.row_of < 0
    assert np.array_equal(dx[idle], dx0[idle])
    exact = 0 if B.dtype != "float32" else 4 * PART["float32"]
    for i, r in enumerate(B.ranks):
        at = B.row_of == i
        a, b, s = f64(B.a[i]), f64(B.b[i]), float(np.float32(B.scale[i]))
        u, size = s * dy[at] @ b, np.abs(s) * np.abs(dy[at]) @ np.abs(b)
        eu = (steps(B.n) * EPS + exact + EPS) * size
        if with_dx:
            want = dx0[at] + u @ a
            mag = (np.abs(u) + eu) @ np.abs(a)
            err = eu @ np.abs(a) + (2 * PART[B.dtype] + steps(r) * EPS) * mag
            within(dx[at], want, err + 2 * EPS * (np.abs(want) + err), B.t)
        else:
            assert np.array_equal(dx, dx0)
        m = int(at.sum())
        part = 2.0 ** -21                       # three bfloat16 parts, two of binary16 or TF32
        for name, got, want, mag, before in (
                ("a", f64(B.ga[i]), u.T @ x[at], (np.abs(u) + eu).T @ np.abs(x[at]) if m else 0 * ga0[i], ga0[i]),
                ("b", f64(B.gb[i]), s * dy[at].T @ h[at][:, :r], np.abs(s) * np.abs(dy[at]).T @ np.abs(h[at][:, :r]), gb0[i])):
            err = (4 * part + steps(m) * EPS) * mag + (eu.T @ np.abs(x[at]) if name == "a" else 0)
            if accumulate:
                want, err = want + before, err + 2 * EPS * (np.abs(want) + np.abs(before))
            if B.dtype == "float16" and m:      # coefficients under one power of two: an absolute floor
                c = np.abs(u) + eu if name == "a" else np.abs(s * h[at][:, :r])
                act = np.abs(x[at]) if name == "a" else np.abs(dy[at])
                floor = c.max() * 2.0 ** -23 * act.sum(axis=0)
                err = err + (floor[None, :] if name == "a" else floor[:, None])
            assert np.all(np.abs(got - want) <= err + 1e-37), (name, i, np.max(np.abs(got - want) / (err + 1e-300)))


TYPES = ["bfloat16", "float16", "float32"]
MIXED = [(1, 0), (5, 1), (0, 2), (3, -1), (17, 0), (64, 2), (1, 1), (130, 2), (2, -1), (33, 0)]
DECODE = [(1, i % 5 - 1) for i in range(43)]


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k,n,pad,off", [(128, 64, 0, 0), (1500, 600, 0, 0), (333, 97, 0, 0), (64, 1000, 8, 0), (200, 130, 3, 1), (1, 1, 0, 0), (7, 3000, 4, 2)])
@pytest.mark.parametrize("requests,ranks", [(MIXED, [8, 16, 5]), (DECODE, [16, 1, 40, 64]), ([(1, 0)], [8])])
def test_forward_matches_the_formula(ctx, dtype, k, n, pad, off, requests, ranks):
    check_forward(ctx, Batch(dtype, k, n, requests, ranks, pad=pad, off=off))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("ranks", [[128], [100, 128, 3], [65], [32, 31, 17]])
@pytest.mark.parametrize("requests", [[(200, 0), (70, -1)], [(3, 0), (1, 0), (2, -1)]])
def test_all_ranks_both_tile_heights(ctx, dtype, ranks, requests):
    requests = requests + [(5, i) for i in range(len(ranks))]
    check_forward(ctx, Batch(dtype, 520, 264, requests, ranks))
    check_backward(ctx, Batch(dtype, 520, 264, requests, ranks))


@pytest.mark.parametrize("dtype", TYPES)
@pytest.mark.parametrize("k,n,pad,off", [(128, 64, 0, 0), (1500, 600, 0, 0), (333, 97, 0, 0), (200, 130, 3, 1), (1, 1, 0, 0), (64, 1000, 8, 0)])
@pytest.mark.parametrize("requests,ranks", [(MIXED, [8, 16, 5]), (DECODE, [16, 1, 40, 64]), ([(1, 0)], [8])])
@pytest.mark.parametrize("accumulate", [False, True])
def test_backward_matches_the_formula(ctx, dtype, k, n, pad, off, requests, ranks, accumulate):
    check_backward(ctx, Batch(dtype, k, n, requests, ranks, pad=pad, off=off), accumulate)


@pytest.mark.parametrize("dtype", TYPES)
def test_long_batches_take_several_splits_and_launches(ctx, dtype):
    """Rows enough for several splits of an adapter; rows scattered enough that the lists need several launches."""
    check_backward(ctx, Batch(dtype, 256, 192, [(3000, 0), (1500, 1), (10, -1), (900, 0)], [16, 24]))
    scattered = [(1, i % 7 - 1) for i in range(3000)]
    check_forward(ctx, Batch(dtype, 128, 96, scattered, [8, 4, 16, 2, 8, 12]))
    check_backward(ctx, Batch(dtype, 128, 96, scattered, [8, 4, 16, 2, 8, 12]))


def test_many_adapters_and_unused_ones(ctx):
    torch = _torch()
    ranks = [1 + i % 16 for i in range(300)]
    B = Batch("bfloat16", 96, 80, [(2, (7 * i) % 290) for i in range(290)] + [(1, -1)], ranks)
    check_forward(ctx, B)
    check_backward(ctx, B)                      # (adapters 290.. have no rows: their gradients are zero)
    assert all(bool((g == 0).all()) for g in B.ga[290:] + B.gb[290:])
    B = Batch("bfloat16", 96, 80, [(5, 1)], [4, 4])
    keep = B.ga[0].clone()
    check_backward(ctx, B, accumulate=True)
    assert torch.equal(B.ga[0], keep)


def test_empty_batches(ctx):
    torch = _torch()
    B = Batch("bfloat16", 64, 32, [(3, -1), (0, 0)], [4])
    launches = ctx.launch_count()
    check_forward(ctx, B)
    assert ctx.launch_count() == launches
    check_backward(ctx, B)
    assert bool((B.ga[0] == 0).all()) and bool((B.gb[0] == 0).all())
    tab = B.table(False)
    none = np.zeros(0)
    ctx.adapter_forward(tab, none, none, torch.zeros(0, 64, dtype=B.t, device="cuda"), torch.zeros(0, 32, dtype=B.t, device="cuda"))


@pytest.mark.parametrize("dtype", TYPES)
def test_rows_do_not_meet(ctx, dtype):
    """Rows of NaN and infinities, with an adapter and without: the other rows of the same tile do not change."""
    torch = _torch()
    requests = [(3, 0), (1, 1), (2, -1), (4, 0), (1, 1)]
    A, B = Batch(dtype, 300, 200, requests, [9, 20], seed=3), Batch(dtype, 300, 200, requests, [9, 20], seed=3)
    B.x[1], B.x[4], B.y[5] = float("nan"), float("inf"), float("nan")       # an adapter's row; a row without; the same
    B.x[7, 10] = float("inf")
    for X in (A, B):
        ctx.adapter_forward(X.table(False), X.rows, X.which, X.x, X.y, X.h)
    torch.cuda.synchronize()
    same = [i for i in range(A.m) if i not in (1, 5, 7)]
    assert torch.equal(A.y[same], B.y[same]) and torch.equal(A.h[same], B.h[same])
    assert torch.isnan(B.y[1]).all() and torch.isnan(B.y[5]).all() and not torch.isfinite(B.y[7]).any()
    # (an infinity times the second part of an fp32 operand, which may be zero, is no number)
    assert (torch.isinf(B.h[7, :9]) if dtype != "float32" else ~torch.isfinite(B.h[7, :9])).all()


def test_an_idle_row_of_nan_leaves_the_gradients_alone(ctx):
    torch = _torch()
    requests = [(70, 0), (3, -1), (40, 0)]
    for dtype in TYPES:
        A, B = Batch(dtype, 130, 70, requests, [12], seed=3), Batch(dtype, 130, 70, requests, [12], seed=3)
        for t in (B.x, B.dy, B.h):
            t[70:73] = float("nan")
        for X in (A, B):
            X.h[:70] = 0.5
            X.h[73:] = -0.25
            ctx.adapter_backward(X.table(), X.rows, X.which, X.x, X.dy, X.h, X.dx)
        torch.cuda.synchronize()
        assert torch.equal(A.ga[0], B.ga[0]) and torch.equal(A.gb[0], B.gb[0]) and torch.equal(A.dx, B.dx)


def test_binary16_keeps_the_range_of_h_and_u(ctx):
    """h far beyond 65504 and u far below 6e-8: neither overflows nor vanishes on the way."""
    check_forward(ctx, Batch("float16", 512, 64, [(20, 0)], [8], xs=2000.0, scales=[1e-6]))
    B = Batch("float16", 64, 512, [(100, 0)], [8], dys=1e-5, scales=[1e-4])
    B.dx.zero_()
    check_backward(ctx, B)
    B = Batch("float16", 2000, 64, [(100, 0)], [8], xs=2000.0, scales=[1e-6])
    B.a[0].mul_(40.0)
    check_backward(ctx, B)


@pytest.mark.parametrize("dtype", TYPES)
def test_equal_calls_give_equal_bits(ctx, dtype):
    torch = _torch()
    args = (dtype, 1500, 700, [(900, 0), (411, 1), (900, 0)], [16, 33])
    A, B = Batch(*args), Batch(*args)
    for X in (A, B):
        ctx.adapter_forward(X.table(False), X.rows, X.which, X.x, X.y, X.h)
        ctx.adapter_backward(X.table(), X.rows, X.which, X.x, X.dy, X.h, X.dx)
    torch.cuda.synchronize()
    for p, q in zip([A.y, A.h, A.dx] + A.ga + A.gb, [B.y, B.h, B.dx] + B.ga + B.gb):
        assert torch.equal(p[:, :9], q[:, :9]) and (p is A.h or torch.equal(p, q))


def test_gradients_against_differences(ctx):
    """The loss sum(y * c) along a direction of every input, by central differences in fp32 of moderate size."""
    torch = _torch()
    requests = [(9, 0), (3, -1), (14, 1), (5, 0)]
    B = Batch("float32", 70, 50, requests, [6, 11], seed=5)
    rs = np.random.RandomState(8)
    c = torch.from_numpy(rs.standard_normal((B.m, B.n))).float().cuda()
    dirs = {"x": [torch.randn(B.m, B.k, device="cuda")], "a": [torch.randn_like(t) for t in B.a], "b": [torch.randn_like(t) for t in B.b]}
    B.dy.copy_(c)
    B.dx.zero_()

    def loss(name, e):
        held = {"x": [B.x], "a": B.a, "b": B.b}[name]
        old = [t.clone() for t in held]
        for t, d in zip(held, dirs[name]):
            t.add_(d, alpha=e)
        y = torch.zeros(B.m, B.n, device="cuda")
        ctx.adapter_forward(B.table(False), B.rows, B.which, B.x, y, B.h)
        for t, o in zip(held, old):
            t.copy_(o)
        return float((y.double() * c.double()).sum())
    loss("x", 0.0)                              # leaves h
    ctx.adapter_backward(B.table(), B.rows, B.which, B.x, B.dy, B.h, B.dx)
    got = {"x": float((B.dx.double() * dirs["x"][0].double()).sum()),
           "a": sum(float((g.double() * d.double()).sum()) for g, d in zip(B.ga, dirs["a"])),
           "b": sum(float((g.double() * d.double()).sum()) for g, d in zip(B.gb, dirs["b"]))}
    size = float((B.y.double().abs() * 0 + c.double().abs()).sum())
    for name in got:        # the loss is linear in each input alone: a difference has only rounding error, sum |c| |y| 2^-20 / e
        e = 0.5
        diff = (loss(name, e) - loss(name, -e)) / (2 * e)
        assert abs(diff - got[name]) <= size * 20 * 2.0 ** -19, (name, diff, got[name])


def test_streams_and_graphs(ctx):
    torch = _torch()
    args = ("bfloat16", 600, 320, [(300, 0), (200, 1), (411, 0)], [16, 24])
    want, A, Bs = Batch(*args), Batch(*args), [Batch(*args) for _ in range(4)]

    def both(X, stream):
        ctx.adapter_forward(X.table(False), X.rows, X.which, X.x, X.y, X.h, stream=stream)
        ctx.adapter_backward(X.table(), X.rows, X.which, X.x, X.dy, X.h, X.dx, stream=stream)
    both(want, None)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    for i, X in enumerate(Bs):
        both(X, streams[i % 2])
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        both(A, torch.cuda.current_stream())
    g.replay()
    torch.cuda.synchronize()
    for X in Bs + [A]:
        for p, q in zip([X.y, X.dx] + X.ga + X.gb, [want.y, want.dx] + want.ga + want.gb):
            assert torch.equal(p, q)


def test_refusals(ctx):
    """Nothing is launched and no buffer touched where an argument is wrong."""
    torch = _torch()
    from paper_1911_02497_b200 import cstep
    B = Batch("float16", 64, 48, [(3, 0), (2, 1)], [4, 8])
    before = [t.clone() for t in (B.x, B.y, B.dx, B.dy, B.h, *B.ga, *B.gb)]
    launches = ctx.launch_count()
    bad, no = cstep.ERR_INVALID_ARG, cstep.ERR_UNSUPPORTED

    def refused(code, change=None, rows=None, which=None, x=None, y=None, h=None):
        tab = B.table()
        if change:
            change(tab)
        args = (tab, B.rows if rows is None else rows, B.which if which is None else which)
        for call in (lambda: ctx.adapter_forward(*args, B.x if x is None else x, B.y if y is None else y, B.h if h is None else h),
                     lambda: ctx.adapter_backward(*args, B.x if x is None else x, B.y if y is None else y, B.h if h is None else h, B.dx)):
            with pytest.raises(cstep.CondensaError) as e:
                call()
            assert e.value.code == code, e.value

    refused(bad, lambda t: setattr(t.entries[0], "a", None))
    refused(bad, lambda t: setattr(t.entries[1], "b", None))
    refused(bad, lambda t: setattr(t.entries[0], "rank", 0))
    refused(no, lambda t: setattr(t.entries[0], "rank", 129))
    refused(bad, lambda t: setattr(t.entries[0], "scale", float("nan")))
    refused(bad, lambda t: setattr(t.entries[0], "a", t.entries[0].a + 1))
    refused(no, lambda t: setattr(t, "code", 3))
    refused(bad, lambda t: setattr(t, "address", None))
    refused(bad, which=[0, 2])
    refused(bad, which=[-2, 0])
    refused(bad, rows=[6, -1])
    for name in ("grad_a", "grad_b"):
        with pytest.raises(cstep.CondensaError):
            t = B.table()
            setattr(t.entries[0], name, B.dy.data_ptr())
            ctx.adapter_backward(t, B.rows, B.which, B.x, B.dy, B.h, B.dx)
    with pytest.raises(cstep.CondensaError):            # in place
        ctx.adapter_backward(B.table(), B.rows, B.which, B.x, B.dy, B.h, B.x)
    with pytest.raises(cstep.CondensaError):            # h is needed for the gradients
        ctx.adapter_backward(B.table(), B.rows, B.which, B.x, B.dy, None, B.dx)
    with pytest.raises(cstep.CondensaError):            # narrow h
        ctx.adapter_forward(B.table(), B.rows, B.which, B.x, B.y, torch.zeros(5, 4, device="cuda"))
    for x in (B.x.float(), B.x[:4], B.x[:, :63], B.x.t().contiguous().t()):
        with pytest.raises(ValueError):
            ctx.adapter_forward(B.table(), B.rows, B.which, x, B.y)
    with pytest.raises(ValueError):
        ctx.adapter_forward(B.table(), [5], B.which, B.x, B.y)
    refused(bad, rows=[3, 1])
    with pytest.raises((TypeError, ValueError)):
        cstep.adapter_table([B.a[0].float()], [B.b[0]], [1.0])
    with pytest.raises(ValueError):
        cstep.adapter_table([B.a[0]], [B.b[1]], [1.0])
    torch.cuda.synchronize()
    assert ctx.launch_count() == launches and B.guards_intact()
    for p, q in zip((B.x, B.y, B.dx, B.dy, B.h, *B.ga, *B.gb), before):
        assert torch.equal(p, q)
