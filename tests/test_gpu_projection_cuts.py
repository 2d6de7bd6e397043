"""Products with a projection in 8 bits at shapes that reach the kernel by pairs of CTAs with its highest tiles, several tiles one after the other, and
the depth shared by several pairs, at every width of access to the result; against 64 bits, formed on the device.

Tolerance as in test_gpu_projection.py: (33 d / 32 + 40) * 2^-24 of the sum of magnitudes over depth d, and one rounding."""
import pytest

from coded_util import E, GROUP, HALF, LEAST
from test_gpu_projection import SHAPES, ctx         # noqa: F401 - the fixture is used by its name

pytestmark = pytest.mark.gpu

# rows, columns of the result, depth. Whole depths: a tile of 224 rows, of 192 with single accesses and with fours; several tiles of a pair
LARGE = [(6011, 2000, 700), (6011, 2049, 260), (2500, 1100, 1024), (9000, 4100, 300),
         # a depth in two to four parts, eights, fours and single accesses, the last with rows and columns that end inside a tile
         (700, 1504, 20000), (300, 2000, 12000), (900, 704, 20000), (400, 1500, 20000), (513, 1500, 33278), (1200, 701, 12000), (900, 1001, 9300),
         # single CTAs that share a depth, fours
         (33, 700, 9216)]


def _coded(rows, cols, high, g):
    """Random codes without NaN, scales around 1."""
    import torch
    from paper_1911_02497_b200 import cstep
    groups = -(-cols // GROUP)
    codes = torch.randint(0, 256, (rows, -(-cols // 16) * 16), dtype=torch.uint8, device="cuda", generator=g)
    codes[(codes & 127) == 127] = 0
    scales = torch.randint(122, 133, (-(-rows // high), -(-groups // 4) * 4), dtype=torch.uint8, device="cuda", generator=g)
    c = (cstep.coded_rows if high == 1 else cstep.coded_blocks)(codes[:, :cols].view(torch.float8_e4m3fn), scales[:, :groups])
    value = c.codes.double() * (c.scales.double() - 127).exp2().repeat_interleave(high, 0)[:rows].repeat_interleave(GROUP, 1)[:, :cols]
    return c, value


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("rows,width,depth", LARGE)
def test_large_products(ctx, rows, width, depth, back):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(rows + width)
    w, W = _coded(depth if back else width, width if back else depth, GROUP, g)
    x, X = _coded(rows, depth, 1, g)
    W = W if back else W.t()
    want, size = X @ W, X.abs() @ W.abs()
    for dtype in ("float16", "bfloat16"):
        t = getattr(torch, dtype)
        top = torch.finfo(t).max
        y = torch.full((rows + 1, width), 7.0, dtype=t, device="cuda")
        (ctx.projection_backward if back else ctx.projection_forward)(w, x, y[:rows])
        got = y[:rows].double()
        assert not bool(got.isnan().any()) and bool((y[rows] == 7).all())
        bound = HALF[dtype] * want.abs() + LEAST[dtype] + (33 * depth / 32 + 40) * E * size * (1 + HALF[dtype])
        assert bool(((got.clamp(-top, top) - want.clamp(-top, top)).abs() <= bound).all())


@pytest.mark.parametrize("back", [False, True])
@pytest.mark.parametrize("rows", [1, 40, 700])
@pytest.mark.parametrize("depth", [100, 200, 300, 500, 600, 800])
def test_what_fills_rows_up_has_no_part(ctx, rows, depth, back):
    """One to four groups in the last word of a row's scales; the bytes behind codes and scales are those of no number, then zeros."""
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(depth)
    width = 520
    results = []
    w, W = _coded(depth if back else width, width if back else depth, GROUP, g)
    x, X = _coded(rows, depth, 1, g)
    for fill in (255, 0):
        for c in (w, x):
            for part in (c.codes.view(torch.uint8), c.scales):
                n, apart = part.shape[0], part.stride(0)
                torch.as_strided(part, (n, apart), (apart, 1))[:, part.shape[1]:] = fill
        y = torch.zeros(rows, width, dtype=torch.bfloat16, device="cuda")
        (ctx.projection_backward if back else ctx.projection_forward)(w, x, y)
        results.append(y)
    want, size = X @ (W if back else W.t()), X.abs() @ (W if back else W.t()).abs()
    bound = HALF["bfloat16"] * want.abs() + (33 * depth / 32 + 40) * E * size * (1 + HALF["bfloat16"])
    assert torch.equal(*results) and bool(((results[0].double() - want).abs() <= bound).all())
