"""Encoders of rows and of weight blocks: codes and scales equal those of the definition."""
import numpy as np
import pytest

from coded_util import GROUP, Room, encode, f64, read, spread

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    from paper_1911_02497_b200 import cstep
    c = cstep.Context(0)
    yield c
    c.close()


def _inputs(rs, rows, cols, dtype):
    """Groups of very different size, groups of zeros, values at and next to the scales' borders, and subnormal ones."""
    v = rs.standard_normal((rows, cols)) * np.exp2(rs.uniform(-12, 12, size=(rows, -(-cols // 64))).repeat(64, axis=1)[:, :cols])
    v[rs.uniform(size=v.shape) < 0.1] = 0.0
    v[:, :min(cols, 3)] *= rs.uniform(size=(rows, 1)) < 0.5
    if rows > 2 and cols > 140:
        v[1, :GROUP] = 0.0
        v[2, :GROUP] *= 1e-3
        v[2, 5] = 1.75 * 2.0 ** 9                       # exactly 448 under its scale
        v[0, 130] = (1.75 + 2.0 ** -7) * 2.0 ** 12      # just above: the next scale
        if dtype != "float16":
            v[rows - 1, :GROUP] *= 2.0 ** -130          # below the least scale
            v[rows - 1, GROUP:] *= 2.0 ** 100
    return v


SIZES = [(1, 1), (1, 127), (1, 1500), (3, 128), (5, 129), (7, 1500), (33, 5), (130, 260), (2, 9217), (300, 640)]


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("pad,off", [(0, 0), (4, 0), (3, 1)])
def test_rows(ctx, dtype, rows, cols, pad, off):
    room = Room()
    x = room.put(_inputs(np.random.RandomState(rows + cols), rows, cols, dtype), dtype, pad, off)
    out = room.coded(rows, cols, more=off)
    ctx.encode_rows(x, out)
    q, s = encode(f64(x))
    got_q, got_s = read(out)
    assert np.array_equal(got_s, s) and np.array_equal(got_q, q) and room.intact()


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows,cols", SIZES)
@pytest.mark.parametrize("pad,off,theta", [(0, 0, None), (4, 0, "own"), (3, 1, "own"), (0, 0, "itself"), (1, 1, "itself")])
def test_blocks(ctx, dtype, rows, cols, pad, off, theta):
    if theta == "itself" and dtype != "float32":
        pytest.skip("only fp32 weights can hold their own theta")
    room = Room()
    w = room.put(_inputs(np.random.RandomState(rows + cols), rows, cols, dtype), dtype, pad, off)
    q, s = encode(f64(w), GROUP)
    out = room.coded(rows, cols, GROUP, more=off)
    th = None if theta is None else w if theta == "itself" else room.put(np.zeros((rows, cols)), "float32", pad, off)
    ctx.encode_blocks(w, out, theta=th)
    got_q, got_s = read(out)
    assert np.array_equal(got_s, s) and np.array_equal(got_q, q) and room.intact()
    if th is not None:
        assert np.array_equal(f64(th), q * 2.0 ** (spread(s, GROUP, q.shape) - 127.0))


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_values_that_are_not_finite(ctx, dtype):
    rs = np.random.RandomState(3)
    v = rs.standard_normal((260, 400))
    v[0, 0], v[0, 200], v[5, 399], v[200, 17] = np.inf, -np.inf, np.nan, -np.nan
    v[9, 128:256] = np.inf                              # a group without a finite value
    v[10, 128:256] = np.nan
    room = Room()
    x = room.put(v, dtype)
    rows, blocks = room.coded(260, 400), room.coded(260, 400, GROUP)
    theta = room.put(np.zeros((260, 400)), "float32")
    ctx.encode_rows(x, rows)
    ctx.encode_blocks(x, blocks, theta=theta)
    for out, high in ((rows, 1), (blocks, GROUP)):
        q, s = encode(f64(x), high)
        got_q, got_s = read(out)
        assert np.array_equal(got_s, s) and np.array_equal(got_q, q, equal_nan=True)
    assert np.array_equal(np.isnan(f64(theta)), ~np.isfinite(v)) and room.intact()


def test_largest_fp32_values(ctx):
    v = np.full((2, 256), 3.4028234663852886e38)
    v[1] = -1.5 * 2.0 ** 127
    room = Room()
    x, out = room.put(v, "float32"), room.coded(2, 256)
    ctx.encode_rows(x, out)
    q, s = encode(f64(x))
    got_q, got_s = read(out)
    assert np.array_equal(got_s, s) and np.array_equal(got_q, q) and s.max() == 247


def test_no_rows(ctx):
    import torch
    from paper_1911_02497_b200 import cstep
    x = torch.zeros(0, 200, device="cuda")
    out = cstep.coded_rows(torch.zeros(0, 208, dtype=torch.uint8, device="cuda")[:, :200], torch.zeros(0, 4, dtype=torch.uint8, device="cuda")[:, :2])
    before = ctx.launch_count()
    ctx.encode_rows(x, out)
    assert ctx.launch_count() == before


def test_offsets_past_32_bits(ctx):
    """Codes whose rows lie so far apart that the last ones start beyond 2^32 bytes."""
    import torch
    from paper_1911_02497_b200 import cstep
    rows, cols, ld = 1100, 200, 1 << 22
    x = torch.randn(rows, cols, device="cuda")
    codes = torch.zeros(rows * ld, dtype=torch.uint8, device="cuda").view(rows, ld)[:, :cols]
    out = cstep.coded_rows(codes, torch.zeros(rows, 4, dtype=torch.uint8, device="cuda")[:, :2])
    ctx.encode_rows(x, out)
    q, s = encode(f64(x))
    got_q, got_s = read(out)
    assert np.array_equal(got_s, s) and np.array_equal(got_q, q)


def test_refusals(ctx):
    import ctypes as C
    import torch
    from paper_1911_02497_b200 import cstep
    x = torch.zeros(4, 256, device="cuda")
    room = Room()
    out, blocks = room.coded(4, 256), room.coded(4, 256, GROUP)
    lib, h = ctx._lib, ctx._h

    def rows_call(p=x.data_ptr(), ld=256, rows=4, cols=256, dtype=0, o=out.struct):
        return lib.condensa_encode_rows(h, p, ld, rows, cols, dtype, C.byref(o) if o is not None else None, None)

    def blocks_call(p=x.data_ptr(), ld=256, n=4, k=256, dtype=0, o=blocks.struct, theta=None, ldt=0):
        return lib.condensa_encode_blocks(h, p, ld, n, k, dtype, C.byref(o) if o is not None else None, theta, ldt, None)

    def changed(s, **kw):
        c = cstep.CodedMatrix(s.codes, s.scales, s.ld, s.ld_scales)
        for k, v in kw.items():
            setattr(c, k, v)
        return c

    before = ctx.launch_count()
    for call, s in ((rows_call, out.struct), (blocks_call, blocks.struct)):
        assert call(p=None) == cstep.ERR_INVALID_ARG
        assert call(p=x.data_ptr() + 2) == cstep.ERR_INVALID_ARG
        assert call(ld=255) == cstep.ERR_INVALID_ARG
        assert call(ld=1 << 60) == cstep.ERR_TOO_LARGE
        assert call(dtype=3) == cstep.ERR_UNSUPPORTED
        assert call(o=None) == cstep.ERR_INVALID_ARG
        assert call(o=changed(s, codes=None)) == cstep.ERR_INVALID_ARG
        assert call(o=changed(s, scales=None)) == cstep.ERR_INVALID_ARG
        assert call(o=changed(s, codes=s.codes + 8)) == cstep.ERR_INVALID_ARG
        assert call(o=changed(s, scales=s.scales + 1)) == cstep.ERR_INVALID_ARG
        assert call(o=changed(s, ld=264)) == cstep.ERR_INVALID_ARG
        assert call(o=changed(s, ld=240)) == cstep.ERR_INVALID_ARG
        assert call(o=changed(s, ld_scales=2)) == cstep.ERR_INVALID_ARG
        assert call(o=changed(s, codes=x.data_ptr())) == cstep.ERR_INVALID_ARG              # output over the input
        assert call(o=changed(s, scales=s.codes)) == cstep.ERR_INVALID_ARG
    assert rows_call(rows=-1) == cstep.ERR_INVALID_ARG and rows_call(cols=0) == cstep.ERR_INVALID_ARG
    assert rows_call(rows=1 << 31) == cstep.ERR_TOO_LARGE and rows_call(cols=(1 << 22) + 1) == cstep.ERR_TOO_LARGE
    assert blocks_call(n=0) == cstep.ERR_INVALID_ARG and blocks_call(k=(1 << 22) + 1) == cstep.ERR_TOO_LARGE
    assert blocks_call(theta=x.data_ptr() + 4, ldt=256) == cstep.ERR_INVALID_ARG            # over the weights, but not they
    assert blocks_call(theta=x.data_ptr(), ldt=260) == cstep.ERR_INVALID_ARG
    assert ctx.launch_count() == before and room.intact()
    assert lib.condensa_encode_rows(None, None, 0, 0, 1, 0, None, None) == cstep.ERR_INVALID_ARG
