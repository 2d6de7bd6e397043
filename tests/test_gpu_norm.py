"""RMS norm with the residual's addition, forward and backward, against the formulas in 64 bits.

Tolerances: E = 2^-24 is half a step of fp32. A row's sum takes at most 16 terms in a thread, then a tree over at most 1024
threads (10 levels; longer rows by fp64): 30 E of the sum of magnitudes covers it, rstd (a root, a quotient, half the sum's error) is within
20 E; a product of a few factors adds a rounding each. Results are rounded once, half a step of their type."""
import numpy as np
import pytest

from coded_util import E, HALF, LEAST, MOST, Room, f64, near_codes

pytestmark = pytest.mark.gpu
EPS = 1e-5


@pytest.fixture()
def ctx():
    from paper_1911_02497_b200 import cstep
    c = cstep.Context(0)
    yield c
    c.close()


def rounded(v, dtype):
    import torch
    return f64(torch.from_numpy(np.asarray(v, dtype=np.float32)).to(getattr(torch, dtype)))


def within(got, want, err, dtype):
    """got is want, known to within err, rounded to dtype once (beyond the largest value: infinite)."""
    fine = np.isfinite(want)
    assert np.array_equal(np.isnan(got), np.isnan(want))
    bound = np.abs(want) * HALF[dtype] + LEAST[dtype] + err * (1 + HALF[dtype])
    off = np.abs(np.clip(got, -MOST[dtype], MOST[dtype]) - np.clip(want, -MOST[dtype], MOST[dtype]))
    assert np.all(off[fine] <= bound[fine]), float((off / bound)[fine].max())


class Forward:
    def __init__(self, rows, cols, dtype, gain="float32", residual=True, pad=0, off=0, seed=0, scale=1.0):
        rs = np.random.RandomState(seed)
        self.room, self.dtype, self.shape = Room(), dtype, (rows, cols)
        draw = lambda: rs.standard_normal((rows, cols)) * np.exp(0.7 * rs.standard_normal(cols)) * np.exp(rs.standard_normal((rows, 1))) * scale
        new = lambda: self.room.put(np.full((rows, cols), 7.0), dtype, pad, off)
        self.x = self.room.put(draw(), dtype, pad, off)
        self.r = self.room.put(draw(), dtype, pad, off) if residual else None
        self.g = self.room.put(1 + 0.3 * rs.standard_normal(cols), gain, 0, off) if gain else None
        self.h, self.y = new(), new()
        self.rstd = self.room.put(np.full(rows, 7.0), "float32")
        self.code = self.room.coded(rows, cols, more=off)

    def want(self):
        x = f64(self.x)
        h = rounded(x + f64(self.r), self.dtype) if self.r is not None else x
        gain = f64(self.g) if self.g is not None else np.ones(self.shape[1])
        with np.errstate(invalid="ignore", over="ignore"):
            rstd = 1.0 / np.sqrt((h ** 2).mean(axis=1) + EPS)
            return h, rstd, h * rstd[:, None] * gain

    def check(self, h_too=True, y_too=True, code_too=True):
        h, rstd, y = self.want_kept if hasattr(self, "want_kept") else self.want()
        if h_too:
            assert np.array_equal(f64(self.h), h, equal_nan=True)
        got = f64(self.rstd)
        fine = np.isfinite(rstd)
        assert np.array_equal(np.isnan(got), np.isnan(rstd)) and np.all(np.abs(got - rstd)[fine] <= 20 * E * rstd[fine] + 2.0 ** -149)
        err = 24 * E * np.abs(y) + 2.0 ** -148
        if y_too:
            within(f64(self.y), y, err, self.dtype)
        if code_too:
            near_codes(self.code, y, err)
        assert self.room.intact()


COLS = [1, 3, 64, 127, 250, 256, 257, 500, 1000, 1500, 2048, 2100, 4096, 6001, 8192, 9000, 16384, 16385, 33278]


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype,gain", [("float32", "float32"), ("float16", "float16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
def test_forward(ctx, cols, dtype, gain):
    f = Forward(5, cols, dtype, gain, seed=cols)
    ctx.norm_forward(f.x, f.g, EPS, residual=f.r, h=f.h, y=f.y, code=f.code, rstd=f.rstd)
    f.check()


@pytest.mark.parametrize("cols", [40, 1500, 4100, 20000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad,off", [(4, 0), (3, 1), (0, 1)])
def test_forward_strides(ctx, cols, dtype, pad, off):
    f = Forward(9, cols, dtype, dtype, pad=pad, off=off)
    ctx.norm_forward(f.x, f.g, EPS, residual=f.r, h=f.h, y=f.y, code=f.code, rstd=f.rstd)
    f.check()


@pytest.mark.parametrize("cols", [200, 1500, 20000])
@pytest.mark.parametrize("place", ["h is x", "h is residual", "y is x", "y is residual", "both"])
def test_forward_in_place(ctx, cols, place):
    f = Forward(6, cols, "bfloat16")
    f.want_kept = f.want()
    if place in ("h is x", "both"):
        f.h = f.x
    elif place == "h is residual":
        f.h = f.r
    if place in ("y is residual", "both"):
        f.y = f.r
    elif place == "y is x":
        f.y = f.x
    ctx.norm_forward(f.x, f.g, EPS, residual=f.r, h=f.h if place[0] != "y" else None, y=f.y, code=f.code, rstd=f.rstd)
    f.check(h_too=place[0] != "y")


@pytest.mark.parametrize("cols", [200, 1500, 20000])
def test_forward_parts_left_out(ctx, cols):
    import torch
    f = Forward(4, cols, "float16", gain=None, residual=False)
    before = f.y.clone()
    ctx.norm_forward(f.x, None, EPS, code=f.code, rstd=f.rstd)
    f.check(h_too=False, y_too=False)
    assert torch.equal(f.y, before)
    ctx.norm_forward(f.x, None, EPS, y=f.y)
    f.check(h_too=False)
    f = Forward(4, cols, "float16", gain=None)
    ctx.norm_forward(f.x, None, EPS, residual=f.r, h=f.h, rstd=f.rstd)
    f.check(y_too=False, code_too=False)


@pytest.mark.parametrize("rows", [0, 1, 2, 130, 1027])
def test_forward_rows(ctx, rows):
    f = Forward(rows, 136, "bfloat16")
    ctx.norm_forward(f.x, f.g, EPS, residual=f.r, h=f.h, y=f.y, code=f.code, rstd=f.rstd)
    if rows:
        f.check()


@pytest.mark.parametrize("cols", [100, 1500, 20000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
def test_forward_values_out_of_the_ordinary(ctx, cols, dtype):
    """Rows of zeros, rows whose squares leave fp32 at either end, infinities and NaN stay in their rows."""
    import torch
    f = Forward(8, cols, dtype, gain=None, residual=False)
    f.x[0] = 0.0
    f.x[1] *= 1e30
    f.x[2] *= 1e-30
    f.x[3, cols // 2] = float("inf")
    f.x[4, cols - 1] = float("nan")
    ctx.norm_forward(f.x, None, EPS, h=f.h, y=f.y, code=f.code, rstd=f.rstd)
    f.check()
    assert torch.isnan(f.y[3]).sum() == 1 and torch.isnan(f.y[4]).all()


class Backward:
    def __init__(self, rows, cols, dtype, gain="float32", joined=True, pad=0, off=0, seed=0):
        rs = np.random.RandomState(seed)
        self.room, self.dtype, self.shape = Room(), dtype, (rows, cols)
        put = lambda v, t=dtype: self.room.put(v, t, pad, off)
        self.h = put(rs.standard_normal((rows, cols)) * np.exp(0.7 * rs.standard_normal(cols)))
        self.dy = put(rs.standard_normal((rows, cols)) * 0.1)
        self.dh = put(rs.standard_normal((rows, cols)) * 0.1) if joined else None
        self.g = self.room.put(1 + 0.3 * rs.standard_normal(cols), gain, 0, off) if gain else None
        self.rstd = self.room.put(1.0 / np.sqrt((f64(self.h) ** 2).mean(axis=1) + EPS) if rows else np.zeros(0), "float32")
        self.dx = put(np.full((rows, cols), 7.0))
        self.dgain = self.room.put(rs.standard_normal(cols), "float32")
        self.code = self.room.coded(rows, cols, more=off)
        self.start = f64(self.dgain)
        self.kept = self.want()

    def want(self):
        """dx, dgain, and what bounds their errors."""
        dy, h, R = f64(self.dy), f64(self.h), f64(self.rstd)[:, None]
        dh = f64(self.dh) if self.dh is not None else 0.0 * dy
        g = f64(self.g) if self.g is not None else np.ones(self.shape[1])
        unit, t = h * R, dy * g
        q, size = (t * unit).mean(axis=1, keepdims=True), np.abs(t * unit).mean(axis=1, keepdims=True)
        dx = dh + R * (t - unit * q)
        dx_err = E * (3 * np.abs(dh) + R * (6 * np.abs(t) + np.abs(unit) * (40 * size + 8 * np.abs(q))))
        return dx, dx_err, (dy * unit).sum(axis=0), (np.abs(dy * unit)).sum(axis=0)

    def check(self, accumulate=False, dx_too=True, code_too=True, dgain_too=True):
        dx, err, dg, size = self.kept
        if dx_too:
            within(f64(self.dx), dx, err, self.dtype)
        if code_too:
            near_codes(self.code, dx, err)
        if dgain_too:               # (a sum of all rows one after the other would be within rows * E of the magnitudes)
            base = self.start if accumulate else 0.0
            assert np.all(np.abs(f64(self.dgain) - dg - base) <= E * ((self.shape[0] + 8) * size + 2 * np.abs(base)) + 2.0 ** -148)
        assert self.room.intact()


@pytest.mark.parametrize("cols", COLS)
@pytest.mark.parametrize("dtype,gain", [("float32", "float32"), ("float16", "float16"), ("bfloat16", "float32"), ("bfloat16", "bfloat16")])
def test_backward(ctx, cols, dtype, gain):
    b = Backward(7, cols, dtype, gain, seed=cols)
    ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dh, dx=b.dx, code=b.code, dgain=b.dgain)
    b.check()


@pytest.mark.parametrize("rows,cols", [(1, 1500), (700, 72), (2100, 130), (650, 1500), (3000, 9), (700, 20000)])
@pytest.mark.parametrize("accumulate", [False, True])
def test_backward_rows(ctx, rows, cols, accumulate):
    b = Backward(rows, cols, "bfloat16")
    ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dh, dx=b.dx, code=b.code, dgain=b.dgain, accumulate=accumulate)
    b.check(accumulate)


@pytest.mark.parametrize("cols", [40, 1500, 4100, 20000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("pad,off", [(4, 0), (3, 1)])
def test_backward_strides(ctx, cols, dtype, pad, off):
    b = Backward(9, cols, dtype, dtype, pad=pad, off=off)
    ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dh, dx=b.dx, code=b.code, dgain=b.dgain)
    b.check()


@pytest.mark.parametrize("cols", [200, 1500, 20000])
@pytest.mark.parametrize("place", ["dy", "dh"])
def test_backward_in_place(ctx, cols, place):
    b = Backward(11, cols, "bfloat16")
    b.dx = b.dy if place == "dy" else b.dh
    ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dh, dx=b.dx, code=b.code, dgain=b.dgain)
    b.check()


@pytest.mark.parametrize("cols", [200, 1500, 20000])
def test_backward_parts_left_out(ctx, cols):
    b = Backward(6, cols, "float16", gain=None, joined=False)
    ctx.norm_backward(b.dy, b.h, None, b.rstd, dx=b.dx)
    b.check(code_too=False, dgain_too=False)
    assert np.array_equal(f64(b.dgain), b.start)
    ctx.norm_backward(b.dy, b.h, None, b.rstd, dgain=b.dgain)
    b.check(code_too=False)
    ctx.norm_backward(b.dy, b.h, None, b.rstd, code=b.code)
    b.check()


def test_backward_no_rows(ctx):
    import torch
    b = Backward(0, 300, "bfloat16")
    before = b.dgain.clone()
    ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dgain=b.dgain, accumulate=True)
    assert torch.equal(b.dgain, before)
    ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dgain=b.dgain)
    assert not b.dgain.any() and b.room.intact()


def test_backward_a_row_that_is_no_number_stays_alone(ctx):
    import torch
    b = Backward(8, 1500, "bfloat16")
    b.dy[3, 7] = float("nan")
    ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dh, dx=b.dx, code=b.code)
    assert torch.isnan(b.dx[3]).all() and not torch.isnan(b.dx[[0, 1, 2, 4, 5, 6, 7]]).any()


def test_equal_calls_give_equal_bits(ctx):
    import torch
    b = Backward(900, 1500, "bfloat16")
    ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dh, dx=b.dx, dgain=b.dgain)
    dx, dg = b.dx.clone(), b.dgain.clone()
    for _ in range(3):
        ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dh, dx=b.dx, dgain=b.dgain)
        assert torch.equal(dx, b.dx) and torch.equal(dg, b.dgain)


@pytest.mark.parametrize("cols", [37, 1500])
def test_gradient_against_differences(ctx, cols):
    """The backward call against differences of the forward call, fp32. Along a direction of length 1 per value, a step of d changes
    the objective by d g + O(d^3): with d = 2^-6 the third derivative's part is below d^2 = 2.5e-4 of sum |w gain| |direction|, the
    forward roundings below 30 E / d = 1.2e-4 of it."""
    import torch
    rs = np.random.RandomState(cols)
    f = Forward(3, cols, "float32", seed=cols)
    w = rs.standard_normal((3, cols))
    b = Backward(3, cols, "float32")
    ctx.norm_forward(f.x, f.g, EPS, residual=f.r, h=b.h, rstd=b.rstd)
    b.dy.copy_(torch.from_numpy(w))
    ctx.norm_backward(b.dy, b.h, f.g, b.rstd, dx=b.dx, dgain=b.dgain)

    def objective():
        ctx.norm_forward(f.x, f.g, EPS, residual=f.r, h=f.h, y=f.y)
        return float((f64(f.y) * w).sum())

    d = 2.0 ** -6
    size = float((np.abs(f64(f.y) * 0 + w) * np.abs(f64(f.g))).sum())
    unit = f64(b.rstd)[:, None]
    for target, grad, scale in ((f.x, b.dx, 1.0 / unit), (f.r, b.dx, 1.0 / unit), (f.g, b.dgain, 1.0)):
        v = rs.choice([-1.0, 1.0], size=tuple(target.shape)) * scale        # (rows of size 1 / rstd move by d of it)
        start = target.clone()
        at = []
        for sign in (1, -1):
            target.copy_(torch.from_numpy(f64(start) + sign * d * v))
            at.append((objective(), f64(target)))
        target.copy_(start)
        slope = (at[0][0] - at[1][0])
        want = float((f64(grad) * (at[0][1] - at[1][1])).sum())
        assert abs(slope - want) <= 2 * d * size * 1e-3, (slope, want, size)


def test_refusals(ctx):
    import ctypes as C
    from paper_1911_02497_b200 import cstep
    f, b = Forward(4, 256, "bfloat16", "bfloat16"), Backward(4, 256, "bfloat16", "bfloat16")
    x, r, h, y, g = (t.data_ptr() for t in (f.x, f.r, f.h, f.y, f.g))

    def forward(code=None, **kw):
        n = cstep.Norm(x, r, g, h, y, code or f.code.struct, f.rstd.data_ptr(), 256, 256, 256, 256, 4, 256, EPS, 2, 2, 0)
        for k, v in kw.items():
            setattr(n, k, v)
        return ctx._lib.condensa_norm_forward(ctx._h, C.byref(n), None)

    def backward(code=None, **kw):
        n = cstep.NormGradient(b.dy.data_ptr(), b.dh.data_ptr(), b.h.data_ptr(), b.g.data_ptr(), b.rstd.data_ptr(), b.dx.data_ptr(), code or b.code.struct,
                               b.dgain.data_ptr(), 256, 256, 256, 256, 4, 256, 2, 2, 0, 0)
        for k, v in kw.items():
            setattr(n, k, v)
        return ctx._lib.condensa_norm_backward(ctx._h, C.byref(n), None)

    bad, none, large = cstep.ERR_INVALID_ARG, cstep.ERR_UNSUPPORTED, cstep.ERR_TOO_LARGE
    before = ctx.launch_count()
    odd = cstep.CodedMatrix(f.code.struct.codes, f.code.struct.scales, 250, 4)
    for call in (forward, backward):
        assert call(dtype=3) == none and call(gain_dtype=1) == none and call(reserved=1) == bad
        assert call(rows=-1) == bad and call(cols=0) == bad and call(rows=1 << 31) == large and call(cols=(1 << 22) + 1) == large
        assert call(code=odd) == bad and call(ldh=255) == bad and call(ldh=1 << 60) == large
    assert forward(x=None) == bad and forward(x=x + 1) == bad and forward(eps=0.0) == bad and forward(eps=float("nan")) == bad
    assert forward(eps=float("inf")) == bad and forward(gain=g + 1) == bad
    assert forward(h=x + 2) == bad and forward(h=x, ldh=260) == bad and forward(y=h) == bad and forward(rstd=x) == bad and forward(h=g) == bad
    assert backward(dy=None) == bad and backward(h=None) == bad and backward(rstd=None) == bad
    assert backward(dx=b.h.data_ptr()) == bad and backward(dx=b.dy.data_ptr() + 2) == bad and backward(dgain=b.g.data_ptr()) == bad
    assert ctx.launch_count() == before
    assert ctx._lib.condensa_norm_forward(ctx._h, None, None) == bad and ctx._lib.condensa_norm_backward(ctx._h, None, None) == bad
    assert ctx._lib.condensa_norm_forward(None, None, None) == bad
    assert f.room.intact() and b.room.intact()


@pytest.mark.parametrize("cols", [100, 1500, 20000])
def test_one_buffer_in_several_places(ctx, cols):
    """x as its own residual, with the sum and the result over it; one gradient as dy, dh and dx."""
    f = Forward(5, cols, "bfloat16")
    f.r = f.x
    f.want_kept = f.want()
    f.h = f.x
    ctx.norm_forward(f.x, f.g, EPS, residual=f.x, h=f.x, y=f.y, code=f.code, rstd=f.rstd)
    f.check()
    b = Backward(5, cols, "bfloat16")
    b.dh = b.dy
    b.kept = b.want()
    b.dx = b.dy
    ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dy, dx=b.dy, code=b.code, dgain=b.dgain)
    b.check()


@pytest.mark.parametrize("cols,pad", [(99, 0), (99, 2), (1001, 0), (1001, 4), (5003, 1), (12345, 0)])
@pytest.mark.parametrize("dtype", ["float32", "float16"])
def test_rows_that_begin_anywhere(ctx, cols, pad, dtype):
    """Every operand at another place within its 16 bytes; neighbouring rows full of NaN, which no row may take over."""
    import torch
    for off in range(0, 8, 3):
        f = Forward(6, cols, dtype, dtype, pad=pad, off=off)
        f.y = f.room.put(np.full((6, cols), 7.0), dtype, pad + 3, off + 1)
        f.r = f.room.put(f64(f.r), dtype, pad + 1, off + 2)
        f.x[2], f.r[2] = float("nan"), float("nan")
        ctx.norm_forward(f.x, f.g, EPS, residual=f.r, h=f.h, y=f.y, code=f.code, rstd=f.rstd)
        f.check()
        b = Backward(6, cols, dtype, dtype, pad=pad, off=off)
        b.dy = b.room.put(f64(b.dy), dtype, pad + 5, off + 3)
        b.dh = b.room.put(f64(b.dh), dtype, pad, off + 1)
        b.dy[3] = float("nan")
        b.kept = b.want()
        ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dh, dx=b.dx, code=b.code)
        b.check(dgain_too=False)
        b.dy[3] = 0.0
        b.kept = b.want()
        ctx.norm_backward(b.dy, b.h, b.g, b.rstd, dh=b.dh, dx=b.dx, code=b.code, dgain=b.dgain)
        b.check()
