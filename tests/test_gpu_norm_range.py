"""The norm where squares, their mean or eps are at either end of fp32's range, against the formula in 64 bits.

Tolerances as for rows in the middle of the range: rstd is within 20 E, a result within 24 E ahead of its rounding."""
import numpy as np
import pytest

from coded_util import E, Room, f64, near_codes
from test_gpu_norm import ctx, within         # noqa: F401 - the fixture is used by its name

pytestmark = pytest.mark.gpu


def _check(ctx, v, dtype, eps):
    rows, cols = v.shape
    room = Room()
    x, y = room.put(v, dtype), room.put(np.full((rows, cols), 7.0), dtype)
    rstd, code = room.put(np.full(rows, 7.0), "float32"), room.coded(rows, cols)
    ctx.norm_forward(x, None, eps, y=y, code=code, rstd=rstd)
    h = f64(x)
    want = 1.0 / np.sqrt((h ** 2).mean(axis=1) + float(np.float32(eps)))
    got = f64(rstd)
    assert np.all(np.abs(got - want) <= 20 * E * want + 2.0 ** -149), (got / want - 1).tolist()
    r = h * want[:, None]
    err = 24 * E * np.abs(r) + 2.0 ** -148
    within(f64(y), r, err, dtype)
    near_codes(code, r, err)
    assert room.intact()


@pytest.mark.parametrize("cols", [100, 500, 1500, 4096, 20000])
@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("eps", [2.0 ** -149, 1e-43, 1e-38, 1e-30])
def test_squares_below_fp32(ctx, cols, dtype, eps):
    """Rows whose squares are subnormal in fp32 or vanish there, a row of zeros, and rows of sizes around where 64 bits are taken, under an eps
    that does not hide them."""
    rs = np.random.RandomState(cols)
    size = np.array([0.0, 1e-30, 1e-24, 3e-23, 1e-22, 1e-21, 1e-19, 5e-16, 2e-15, 1.0])
    _check(ctx, rs.standard_normal((len(size), cols)) * size[:, None], dtype, eps)


@pytest.mark.parametrize("cols", [1, 100, 1500, 20000])
def test_mean_and_eps_beyond_fp32(ctx, cols):
    """Squares that fit, with an eps that takes their mean beyond the largest value; squares that do not fit."""
    v = np.outer([0.0, 1.0, 1.5e19, 1.8e19, 1e25], np.where(np.arange(cols) % 3, 1.0, -0.9))
    _check(ctx, v, "float32", 3e38)
