"""Products with a projection in 8 bits against 64 bits.

Products of codes and powers of two are exact. A sum is formed 32 terms at a time by an instruction that cuts: measured, the 32 terms
and the sum so far at 2^-25 of the largest of them, their sum at 2^-23 of it, so a step loses at most (33 / 2 + 2) * 2^-24, less
than 33 * 2^-24, of the sum of magnitudes S; parts of a sum are joined with roundings. Over depth d that is at most
(33 d / 32 + 40) * 2^-24 * S. The result is rounded once."""
import numpy as np
import pytest

from coded_util import E, GROUP, HALF, LEAST, MOST, Room, f64, fill, read, values

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    from paper_1911_02497_b200 import cstep
    c = cstep.Context(0)
    yield c
    c.close()


class Case:
    def __init__(self, rows, k, n, dtype="bfloat16", back=False, pad=0, off=0, seed=0, more=0):
        rs = np.random.RandomState(seed)
        self.room, self.back, self.dtype = Room(), back, dtype
        self.w = fill(self.room.coded(n, k, GROUP, more), rs)
        self.x = fill(self.room.coded(rows, n if back else k, 1, more), rs)
        self.y = self.room.put(np.full((rows, k if back else n), 7.0), dtype, pad, off)

    def run(self, ctx, stream=None):
        (ctx.projection_backward if self.back else ctx.projection_forward)(self.w, self.x, self.y, stream=stream)

    def check(self):
        import torch
        w, x = torch.from_numpy(values(self.w)).cuda(), torch.from_numpy(values(self.x)).cuda()
        w = w if self.back else w.t()
        want, size = (x @ w).cpu().numpy(), (x.abs() @ w.abs()).cpu().numpy()
        got = f64(self.y)
        depth = x.shape[1]
        bound = HALF[self.dtype] * np.abs(want) + LEAST[self.dtype] + (33 * depth / 32 + 40) * E * size * (1 + HALF[self.dtype])
        top = MOST[self.dtype]
        off = np.abs(np.clip(got, -top, top) - np.clip(want, -top, top))
        assert not np.isnan(got).any() and np.all(off <= bound), float((off / bound).max())
        assert self.room.intact()


# one row to many, depths from 1 to long ones, and widths, at and around the tiles' edges
SHAPES = [(1, 1, 1), (1, 128, 128), (1, 1500, 6000), (2, 16, 300), (3, 130, 17), (8, 512, 128), (15, 640, 129), (16, 513, 256), (17, 127, 1000),
          (33, 700, 300), (64, 4096, 640), (100, 1500, 260), (127, 384, 384), (128, 1025, 130), (129, 256, 512), (145, 900, 140), (255, 2000, 70),
          (257, 129, 2000), (300, 5000, 33), (513, 1500, 1500), (700, 1500, 2100), (1025, 520, 777), (2049, 260, 1100)]


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("rows,k,n", SHAPES)
def test_shapes(ctx, rows, k, n, back):
    c = Case(rows, k, n, "bfloat16" if (rows + k) % 2 else "float16", back, seed=rows + k + n)
    c.run(ctx)
    c.check()


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("rows,k,n", [(1, 40000, 130), (130, 130, 40000), (700, 33278, 300), (40, 300, 33278)])
def test_long_sums_and_wide_results(ctx, rows, k, n, back):
    c = Case(rows, k, n, "float16", back, seed=2)
    c.run(ctx)
    c.check()


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("dtype", ["float16", "bfloat16"])
@pytest.mark.parametrize("rows", [5, 200, 1500])
@pytest.mark.parametrize("pad,off,more", [(4, 0, 1), (1, 1, 2), (2, 0, 0), (0, 3, 0)])
def test_strides(ctx, rows, back, dtype, pad, off, more):
    c = Case(rows, 620, 1000, dtype, back, pad, off, seed=rows, more=more)
    c.run(ctx)
    c.check()


@pytest.mark.parametrize("rows", [3, 90, 1030])
def test_whole_numbers_are_exact_and_backward_is_the_adjoint(ctx, rows):
    """Codes and scales that keep every sum a whole number below 2^11: no rounding anywhere."""
    import torch
    rs = np.random.RandomState(rows)
    room, k, n = Room(), 300, 420
    w, x, dy = room.coded(n, k, GROUP), room.coded(rows, k), room.coded(rows, n)
    for m in (w, x, dy):
        m.codes.copy_(torch.from_numpy(rs.choice([-2.0, -1.0, 0.0, 0.0, 1.0, 2.0], size=(m.rows, m.cols)) * (rs.uniform(size=(m.rows, m.cols)) < 0.3)))
        m.scales.view(torch.uint8).fill_(127)
    y, dx = room.put(np.zeros((rows, n)), "float16"), room.put(np.zeros((rows, k)), "float16")
    ctx.projection_forward(w, x, y)
    ctx.projection_backward(w, dy, dx)
    W, X, D = values(w), values(x), values(dy)
    assert np.array_equal(f64(y), X @ W.T) and np.array_equal(f64(dx), D @ W)
    assert (f64(y) * D).sum() == (f64(dx) * X).sum() and room.intact()


@pytest.mark.parametrize("rows", [7, 150, 1100])
@pytest.mark.parametrize("back", [False, True])
def test_every_scale_is_used_where_it_belongs(ctx, rows, back):
    """One code of 1 in each group, all scales different powers: a result is a sum of known powers of two, exact."""
    import torch
    k, n = 1150, 700
    c = Case(rows, k, n, "bfloat16", back)
    rs = np.random.RandomState(1)
    depth = n if back else k
    X = np.zeros((rows, depth))
    groups = -(-depth // GROUP)
    which = rs.randint(0, groups, size=rows)
    X[np.arange(rows), np.minimum(which * GROUP + rs.randint(0, GROUP, size=rows), depth - 1)] = 1.0
    c.x.codes.copy_(torch.from_numpy(X))
    c.x.scales.view(torch.uint8).copy_(torch.from_numpy(rs.randint(100, 150, size=(rows, groups)).astype(np.uint8)))
    c.w.codes.copy_(torch.ones(n, k))
    c.w.scales.view(torch.uint8).copy_(torch.from_numpy(rs.randint(100, 150, size=tuple(c.w.scales.shape)).astype(np.uint8)))
    c.run(ctx)
    w = values(c.w)
    assert np.array_equal(f64(c.y), values(c.x) @ (w if back else w.T)) and c.room.intact()


@pytest.mark.parametrize("rows", [6, 200, 1100])
def test_numbers_that_are_none_stay_in_their_rows(ctx, rows):
    import torch
    c = Case(rows, 700, 300, "float16")
    c.run(ctx)
    before = c.y.clone()
    c.x.codes.view(torch.uint8)[rows // 2, 650] = 0x7F
    c.run(ctx)
    same = torch.arange(rows, device="cuda") != rows // 2
    assert torch.isnan(c.y[rows // 2]).all() and torch.equal(c.y[same], before[same])


def test_sums_beyond_binary16_are_infinite(ctx):
    import torch
    c = Case(20, 256, 130, "float16")
    c.w.codes.copy_(torch.full((130, 256), 240.0))
    c.w.scales.view(torch.uint8).fill_(130)
    c.x.codes.copy_(torch.full((20, 256), 240.0) * torch.tensor([1.0, -1.0]).repeat(10)[:, None])
    c.x.scales.view(torch.uint8).fill_(130)
    c.run(ctx)
    assert torch.isinf(c.y).all() and torch.equal(c.y[:, 0] > 0, torch.tensor([True, False] * 10, device="cuda"))


@pytest.mark.parametrize("s", [1, 60, 127, 200, 254])
def test_ends_of_the_scales(ctx, s):
    """Scale bytes 1 .. 254 of one operand against the other's opposite ones: the product of powers is 1."""
    import torch
    c = Case(9, 200, 140, "bfloat16")
    c.w.scales.view(torch.uint8).fill_(s)
    c.x.scales.view(torch.uint8).fill_(254 - s if s < 254 else 1)
    c.run(ctx)
    if s < 254:
        c.check()
    else:                           # 2^127 * 2^-126
        want = f64(c.y)
        c.w.scales.view(torch.uint8).fill_(128)
        c.x.scales.view(torch.uint8).fill_(127)
        c.run(ctx)
        assert np.array_equal(want, f64(c.y))


def test_equal_calls_give_equal_bits_on_any_stream(ctx):
    import torch
    for rows in (1, 64, 700, 1500):
        c = Case(rows, 1500, 2000)
        c.run(ctx)
        torch.cuda.synchronize()
        before = c.y.clone()
        side = torch.cuda.Stream()
        for _ in range(3):
            c.y.fill_(7.0)
            side.wait_stream(torch.cuda.current_stream())
            c.run(ctx, side)
            side.synchronize()
            assert torch.equal(c.y, before)


def test_offsets_past_32_bits(ctx):
    """Codes, and results, whose last rows start beyond 2^32 bytes."""
    import torch
    from paper_1911_02497_b200 import cstep
    rs = np.random.RandomState(0)
    room = Room()
    w = fill(room.coded(40, 200, GROUP), rs)
    rows, ld = 1100, 1 << 22
    codes = torch.zeros(rows * ld, dtype=torch.uint8, device="cuda").view(rows, ld)[:, :200]
    x = fill(cstep.coded_rows(codes, torch.zeros(rows, 4, dtype=torch.uint8, device="cuda")[:, :2]), rs)
    y = torch.zeros(rows * (ld // 2), dtype=torch.bfloat16, device="cuda").view(rows, ld // 2)[:, :40]
    ctx.projection_forward(w, x, y)
    want, size = values(x) @ values(w).T, np.abs(values(x)) @ np.abs(values(w)).T
    assert np.all(np.abs(f64(y) - want) <= HALF["bfloat16"] * np.abs(want) + 250 * E * size * 1.01)


def test_no_rows(ctx):
    import torch
    from paper_1911_02497_b200 import cstep
    w = Room().coded(40, 200, GROUP)
    x = cstep.coded_rows(torch.zeros(0, 208, dtype=torch.uint8, device="cuda")[:, :200], torch.zeros(0, 4, dtype=torch.uint8, device="cuda")[:, :2])
    before = ctx.launch_count()
    ctx.projection_forward(w, x, torch.zeros(0, 40, dtype=torch.float16, device="cuda"))
    assert ctx.launch_count() == before


def test_refusals(ctx):
    import ctypes as C
    from paper_1911_02497_b200 import cstep
    c = Case(4, 256, 130, "bfloat16")
    d = Case(4, 256, 130, "bfloat16", back=True)

    def call(case, w={}, x={}, n=130, k=256, rows=4, y=None, ld=None, dtype=2, none=""):
        p = cstep.Projection(case.w.struct, n, k)
        for key, v in w.items():
            setattr(p.code, key, v)
        s = case.x.struct
        o = cstep.CodedMatrix(s.codes, s.scales, s.ld, s.ld_scales)
        for key, v in x.items():
            setattr(o, key, v)
        f = ctx._lib.condensa_projection_backward if case.back else ctx._lib.condensa_projection_forward
        return f(ctx._h, None if none == "w" else C.byref(p), None if none == "x" else C.byref(o), rows, case.y.data_ptr() if y is None else y,
                 case.y.stride(0) if ld is None else ld, dtype, None)

    bad, none, large = cstep.ERR_INVALID_ARG, cstep.ERR_UNSUPPORTED, cstep.ERR_TOO_LARGE
    before = ctx.launch_count()
    for case in (c, d):
        assert call(case, none="w") == bad and call(case, none="x") == bad and call(case, y=0) == bad
        assert call(case, dtype=0) == none and call(case, dtype=3) == none
        assert call(case, n=0) == bad and call(case, k=0) == bad and call(case, rows=-1) == bad
        assert call(case, n=(1 << 22) + 1) == large and call(case, k=(1 << 22) + 1) == large and call(case, rows=1 << 31) == large
        for m in ("w", "x"):
            s = case.w.struct if m == "w" else case.x.struct
            for kw in (dict(codes=None), dict(scales=None), dict(codes=s.codes + 4), dict(scales=s.scales + 2), dict(ld=s.ld + 8), dict(ld=16), dict(ld_scales=1),
                       dict(ld=-16)):
                assert call(case, **{m: kw}) == bad, (m, kw)
            assert call(case, y=s.codes) == bad
        assert call(case, ld=20) == bad and call(case, y=case.y.data_ptr() + 1) == bad and call(case, ld=1 << 60) == large
    assert ctx.launch_count() == before and c.room.intact() and d.room.intact()
    assert ctx._lib.condensa_projection_forward(None, None, None, 0, None, 0, 0, None) == bad


@pytest.mark.parametrize("rows", [9, 300])
def test_one_matrix_as_both_operands(ctx, rows):
    """Inputs may share memory: the codes of w's first rows as x, under scales of their own."""
    from paper_1911_02497_b200 import cstep
    c = Case(rows, 700, 400)
    scales = fill(c.room.coded(rows, 700), np.random.RandomState(9)).scales
    c.x = cstep.coded_rows(c.w.codes[:rows], scales)
    c.run(ctx)
    c.check()


def test_contexts_of_two_threads(ctx):
    """A context for each thread: calls at the same time, on streams of their own."""
    import threading

    import torch
    from paper_1911_02497_b200 import cstep
    cases = [Case(rows, 1500, 2000, seed=rows) for rows in (3, 700)]
    for c in cases:
        c.run(ctx)
    torch.cuda.synchronize()
    want, failed = [c.y.clone() for c in cases], []

    def work(c, expected):
        try:
            own, stream = cstep.Context(0), torch.cuda.Stream()
            for _ in range(50):
                c.run(own, stream)
            stream.synchronize()
            if not torch.equal(c.y, expected):
                failed.append("bits")
            own.close()
        except Exception as e:      # noqa: BLE001 - told by the test's own thread
            failed.append(e)

    threads = [threading.Thread(target=work, args=a) for a in zip(cases, want)]
    [t.start() for t in threads]
    [t.join() for t in threads]
    assert not failed
