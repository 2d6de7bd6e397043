"""What the tests of the 8-bit operators share: guarded buffers, and the 8-bit form from its definition in 64 bits."""
import numpy as np

GROUP = 128


class Room:
    """Device buffers with guard bytes around and between their rows."""

    def __init__(self):
        self.held = []

    def _view(self, a, t, ld, off):
        import torch
        m, w = a.shape
        size = torch.zeros(0, dtype=t).element_size()
        room = torch.full(((off + max(m, 1) * ld + 64) * size,), 93, dtype=torch.uint8, device="cuda")
        mask = torch.ones(room.numel() // size, dtype=torch.bool, device="cuda")
        at = lambda x: torch.as_strided(x, (m, w), (ld, 1), off)
        at(mask)[:] = False
        self.held.append((room, mask, size))
        return at(room.view(t))

    def put(self, a, dtype, pad=0, off=0):
        """A matrix (or vector) of type `dtype`, rows `pad` elements further apart than they are long, `off` elements behind an aligned start."""
        import torch
        a = np.asarray(a, dtype=np.float64)
        t = getattr(torch, dtype)
        v = self._view(np.atleast_2d(a), t, np.atleast_2d(a).shape[1] + pad, off)
        v.copy_(torch.from_numpy(np.atleast_2d(a)))
        return v if a.ndim == 2 else v[0]

    def coded(self, rows, cols, high=1, more=0):
        """Buffers of an 8-bit matrix, `more` whole units wider apart than they have to be."""
        import torch
        from paper_1911_02497_b200 import cstep
        groups = -(-cols // GROUP)
        codes = self._view(np.zeros((rows, cols)), torch.uint8, (-(-cols // 16) + more) * 16, 16 * more)
        scales = self._view(np.zeros((-(-rows // high), groups)), torch.uint8, (-(-groups // 4) + more) * 4, 4 * more)
        return (cstep.coded_rows if high == 1 else cstep.coded_blocks)(codes.view(torch.float8_e4m3fn), scales)

    def intact(self):
        import torch
        return all(bool((room.view(-1, size)[mask] == 93).all()) for room, mask, size in self.held)


def f64(t):
    return t.detach().double().cpu().numpy()


def e4m3_value(codes):
    """Values of code bytes: sign, four exponent bits (bias 7), three fraction bits; S.1111.111 is no number."""
    c = np.asarray(codes, dtype=np.int64)
    e, f = (c >> 3) & 15, c & 7
    v = np.where(e == 0, f * 2.0 ** -9, (1 + f / 8.0) * 2.0 ** (e - 7.0))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c >> 7, -v, v)


def e4m3_round(q):
    """The nearest value of the format to |q| <= 448, of two the even one."""
    with np.errstate(invalid="ignore"):
        e = np.maximum(np.frexp(np.where(np.isfinite(q), q, 1.0))[1] - 1, -6)
        step = 2.0 ** (e - 3)
        return np.rint(q / step) * step


def spread(s, high, shape):
    return np.repeat(np.repeat(s, high, axis=0)[:shape[0]], GROUP, axis=1)[:, :shape[1]]


def group_most(v, high):
    """Largest finite magnitude of every group."""
    n, k = v.shape
    a = np.zeros((-(-n // high) * high, -(-k // GROUP) * GROUP))
    a[:n, :k] = np.where(np.isfinite(v), np.abs(v), 0.0)
    return a.reshape(a.shape[0] // high, high, -1, GROUP).max(axis=(1, 3))


def scale_bytes(most):
    """The least s >= 1 with most <= 448 * 2^(s - 127)."""
    m, e = np.frexp(most)
    return np.where(most > 0, np.maximum(e - 9 + 127 + (m > 0.875), 1), 1).astype(np.int64)


def encode(v, high=1):
    """(values of the codes, scale bytes)"""
    s = scale_bytes(group_most(v, high))
    q = e4m3_round(np.where(np.isfinite(v), v, np.nan) * 2.0 ** (127.0 - spread(s, high, v.shape)))
    return q, s


def read(coded):
    """(values of the codes, scale bytes) of a device matrix."""
    import torch
    return e4m3_value(coded.codes.view(torch.uint8).cpu().numpy()), coded.scales.view(torch.uint8).cpu().numpy().astype(np.int64)


def values(coded):
    q, s = read(coded)
    return q * 2.0 ** (spread(s, coded.high, q.shape) - 127.0)


def fill(coded, rs, spread_bits=3.0):
    """Random codes (no NaN) and scales around 1."""
    import torch
    c = rs.randint(0, 256, size=(coded.rows, coded.cols))
    c = np.where((c & 127) == 127, 0, c).astype(np.uint8)
    coded.codes.view(torch.uint8).copy_(torch.from_numpy(c))
    s = np.rint(127 + spread_bits * rs.standard_normal(tuple(coded.scales.shape))).astype(np.uint8)
    coded.scales.view(torch.uint8).copy_(torch.from_numpy(s))
    return coded


HALF = {"float32": 2.0 ** -24, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}        # half a step, relative
LEAST = {"float32": 2.0 ** -150, "float16": 2.0 ** -25, "bfloat16": 2.0 ** -134}    # half the least step
MOST = {"float32": 3.4028234663852886e38, "float16": 65504.0, "bfloat16": 3.3895313892515355e38}
E = 2.0 ** -24


def near_codes(coded, v, err):
    """Whether an 8-bit matrix holds v, known to within err: every scale follows from a value that near, every code is the
    nearest (half a step) to such a value under its scale."""
    q, s = read(coded)
    most, slack = group_most(v, 1), group_most(np.where(np.isfinite(v), err, 0.0), 1)
    assert np.all((s >= scale_bytes(np.maximum(most - slack, 0))) & (s <= scale_bytes(most + slack)))
    p = 2.0 ** (127.0 - spread(s, 1, v.shape))
    x, e = v * p, err * p
    assert np.array_equal(np.isnan(q), ~np.isfinite(v))
    fine = np.isfinite(v)
    lo, hi = e4m3_round(np.clip(x - e, -448, 448)), e4m3_round(np.clip(x + e, -448, 448))
    assert np.all((q >= lo) & (q <= hi) | ~fine)
