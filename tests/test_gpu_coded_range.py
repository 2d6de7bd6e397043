"""The block encoder next to the largest value of fp32."""
import numpy as np
import pytest

from coded_util import GROUP, Room, encode, f64, read
from test_gpu_coded import ctx                # noqa: F401 - the fixture is used by its name

pytestmark = pytest.mark.gpu


def test_values_next_to_the_largest(ctx):
    """Under the scale 2^120 a code is a multiple of 16 from 128 on, and the next above 240 is 256. 1.9375 is half-way: to the even one, 256."""
    top = 2.0 ** 127
    v = np.array([[3.4028234663852886e38, 1.9375 * top, -1.9375 * top, 1.9374999 * top, -1.875 * top, 1.0, 0.0, -3.4028234663852886e38]])
    room = Room()
    w, out, theta = room.put(v, "float32"), room.coded(1, 8, GROUP), room.put(np.zeros((1, 8)), "float32")
    ctx.encode_blocks(w, out, theta=theta)
    q, s = encode(f64(w), GROUP)
    got_q, got_s = read(out)
    assert np.array_equal(got_s, s) and np.array_equal(got_q, q) and s[0, 0] == 247
    assert list(q[0]) == [256, 256, -256, 240, -240, 0, 0, -256]
    inf = float("inf")
    assert list(f64(theta)[0]) == [inf, inf, -inf, 1.875 * top, -1.875 * top, 0, 0, -inf] and room.intact()
