"""The norm and its gradient over so many rows that every CTA of the gradient takes several, at every number of threads that a row is given,
and over rows that lie far apart; against the formulas in 64 bits, formed on the device.

Tolerances are those of few rows (E = 2^-24: rstd within 20 E, a result within 24 E of its terms ahead of its rounding, sums of a row 40 E of
their magnitudes). A sum for the gain is formed by a thread over its rows, by a warp over every 32nd of what the threads left, then over
32 warps: as many roundings as those are at most, with the few of a product."""
import pytest

from coded_util import E, GROUP, HALF, LEAST
from test_gpu_norm import ctx                 # noqa: F401 - the fixture is used by its name

pytestmark = pytest.mark.gpu
EPS = 1e-5


def _matrix(v, dtype, access, apart=None):
    """A copy of v whose rows allow 8, 4 or single values at once: multiples of that many elements apart, and begun there."""
    import torch
    rows, cols = v.shape
    ld = apart or (-(-cols // 8) * 8 + {8: 8, 4: 4, 1: 3}[access])
    off = {8: 0, 4: 4, 1: 1}[access]
    m = torch.empty(off + (rows - 1) * ld + cols, dtype=getattr(torch, dtype), device="cuda")
    m = torch.as_strided(m, (rows, cols), (ld, 1), off)
    m.copy_(v)
    return m


def _coded(rows, cols):
    import torch
    from paper_1911_02497_b200 import cstep
    groups = -(-cols // GROUP)
    return cstep.coded_rows(torch.full((rows, -(-cols // 16) * 16), 93, dtype=torch.uint8, device="cuda")[:, :cols].view(torch.float8_e4m3fn),
                            torch.full((rows, -(-groups // 4) * 4), 93, dtype=torch.uint8, device="cuda")[:, :groups])


def _within(got, want, err, dtype):
    off = (got.double() - want).abs()
    assert bool((off <= want.abs() * HALF[dtype] + LEAST[dtype] + err * (1 + HALF[dtype])).all()), float((off / (want.abs() * HALF[dtype] + err)).max())


def _near(code, want, err):
    """A group's scale is the least that holds its largest magnitude (2^-20 either way), a code is off by half a step of E4M3: 2^-4 of its value,
    2^-10 of the scale at least."""
    import torch
    rows, cols = want.shape
    groups = -(-cols // GROUP)
    most = torch.zeros(rows, groups * GROUP, dtype=torch.float64, device="cuda")
    most[:, :cols] = want.abs()
    most = most.view(rows, groups, GROUP).amax(dim=2)
    scale = (code.scales.double() - 127).exp2()
    assert bool((most <= 448 * scale * (1 + 2.0 ** -20)).all()) and bool(((most >= 224 * scale * (1 - 2.0 ** -20)) | (code.scales == 1)).all())
    wide = scale.repeat_interleave(GROUP, dim=1)[:, :cols]
    off = (code.codes.double() * wide - want).abs()
    assert bool((off <= (2.0 ** -4 * want.abs()).maximum(2.0 ** -10 * wide) + 1.1 * err).all())


def _draw(rows, cols, seed, n):
    import torch
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return [torch.randn(rows, cols, device="cuda", generator=g) for _ in range(n)], 1 + 0.3 * torch.randn(cols, device="cuda", generator=g)


# columns for every number of threads of a row (and for rows that are read twice), with rows for at least seven rounds of a gradient's CTAs
# (148 SMs, eight CTAs of four warps, four or less of more threads)
WIDTHS = [(200, 36000), (480, 36000), (1000, 9000), (1496, 9000), (2000, 9000), (2600, 7000), (4088, 6000), (5640, 4000), (8000, 2500), (9000, 2100),
          (16000, 2100), (20000, 600)]


@pytest.mark.parametrize("dtype", ["float32", "bfloat16"])
@pytest.mark.parametrize("access", [8, 4, 1])
@pytest.mark.parametrize("cols,rows", WIDTHS)
def test_backward_many_rows(ctx, cols, rows, access, dtype):
    """dx beside its operands, over dy and over dh, with and without dh."""
    import torch
    cols -= {8: 0, 4: 4, 1: 3}[access]
    (h, dy, dh), gain = _draw(rows, cols, cols, 3)
    h, dy, dh = (_matrix(v, dtype, access) for v in (h, dy * 0.1, dh * 0.1))
    R = (1.0 / (h.double().square().mean(dim=1) + EPS).sqrt()).float()
    code, dgain = _coded(rows, cols), torch.zeros(cols, device="cuda")
    unit = h.double() * R.double()[:, None]
    t = dy.double() * gain.double()
    q, size = (t * unit).mean(dim=1, keepdim=True), (t * unit).abs().mean(dim=1, keepdim=True)
    back = R.double()[:, None] * (t - unit * q)
    err = E * R.double()[:, None] * (6 * t.abs() + unit.abs() * (40 * size + 8 * q.abs()))
    p = dy.double() * unit
    dg, dg_size = p.sum(dim=0), p.abs().sum(dim=0)
    # (a CTA has 128 threads or more, 16 of them fit an SM; up to 512 columns it has four rows under way)
    sms, under_way = torch.cuda.get_device_properties(0).multi_processor_count, 4 if cols <= 512 else 1
    roundings = -(-rows // (sms * under_way)) + -(-min(rows, sms * 16 * under_way) // 32) + 32 + 8
    for place in ("beside", "alone", "over dy", "over dh"):
        mine = [_matrix(v, dtype, access) for v in (dy, dh)]
        dx = {"over dy": mine[0], "over dh": mine[1]}.get(place)
        if dx is None:
            dx = _matrix(torch.full_like(dy, 7.0), dtype, access)
        ctx.norm_backward(mine[0], h, gain, R, dh=None if place == "alone" else mine[1], dx=dx, code=code, dgain=dgain)
        want = back if place == "alone" else back + dh.double()
        e = err if place == "alone" else err + 3 * E * dh.double().abs()
        _within(dx, want, e, dtype)
        _near(code, want, e)
        assert bool(((dgain.double() - dg).abs() <= roundings * E * dg_size).all())


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("access", [8, 4, 1])
@pytest.mark.parametrize("cols", [w for w, _ in WIDTHS] + [12000])
def test_forward_at_every_number_of_threads(ctx, cols, access, dtype):
    cols -= {8: 0, 4: 4, 1: 3}[access]
    rows = 37
    import torch
    (x, r), gain = _draw(rows, cols, cols, 2)
    x, r = (_matrix(v, dtype, access) for v in (x, r))
    h, y = (_matrix(torch.full_like(x, 7.0), dtype, access) for _ in range(2))
    rstd, code = torch.zeros(rows, device="cuda"), _coded(rows, cols)
    ctx.norm_forward(x, gain, EPS, residual=r, h=h, y=y, code=code, rstd=rstd)
    s = (x.float() + r.float()).to(x.dtype)
    R = 1.0 / (s.double().square().mean(dim=1) + EPS).sqrt()
    want = s.double() * R[:, None] * gain.double()
    assert torch.equal(h, s) and bool(((rstd.double() - R).abs() <= 20 * E * R).all())
    _within(y, want, 24 * E * want.abs(), dtype)
    _near(code, want, 24 * E * want.abs())


@pytest.mark.parametrize("access", [8, 1])
def test_offsets_past_32_bits(ctx, access):
    """Rows so far apart that the last ones begin more than 2^32 bytes behind the first."""
    import torch
    from paper_1911_02497_b200 import cstep
    rows, cols, apart = 1030, 200, (1 << 21) + 8 + (access == 1)
    (x, r, dh), gain = _draw(rows, cols, 1, 3)
    x, r = (_matrix(v, "bfloat16", access, apart) for v in (x, r))
    rstd = torch.zeros(rows, device="cuda")
    codes = torch.zeros(rows << 22, dtype=torch.uint8, device="cuda").view(rows, 1 << 22)[:, :cols].view(torch.float8_e4m3fn)
    code = cstep.coded_rows(codes, torch.zeros(rows, 4, dtype=torch.uint8, device="cuda")[:, :2])
    s = (x.float() + r.float()).bfloat16()
    ctx.norm_forward(x, gain, EPS, residual=r, h=x, y=r, code=code, rstd=rstd)
    R = 1.0 / (s.double().square().mean(dim=1) + EPS).sqrt()
    want = s.double() * R[:, None] * gain.double()
    assert torch.equal(x, s)
    _within(r, want, 24 * E * want.abs(), "bfloat16")
    _near(code, want, 24 * E * want.abs())
    dh = dh.bfloat16()
    r.copy_(dh)                                 # dy; dx goes over it
    ctx.norm_backward(r, x, gain, rstd, dx=r, code=code)
    unit, t, R = s.double() * rstd.double()[:, None], dh.double() * gain.double(), rstd.double()[:, None]
    q, size = (t * unit).mean(dim=1, keepdim=True), (t * unit).abs().mean(dim=1, keepdim=True)
    want, err = R * (t - unit * q), E * R * (6 * t.abs() + unit.abs() * (40 * size + 8 * q.abs()))
    _within(r, want, err, "bfloat16")
    _near(code, want, err)


@pytest.mark.parametrize("access", [8, 1])
def test_blocks_past_32_bits(ctx, access):
    """The same of a block encoder's weights, codes and values."""
    import torch
    from paper_1911_02497_b200 import cstep
    rows, cols, apart = 1030, 200, (1 << 21) + 8 + (access == 1)
    (w,), _ = _draw(rows, cols, 2, 1)
    w = _matrix(w, "float32", access, apart)
    codes = torch.zeros(rows << 22, dtype=torch.uint8, device="cuda").view(rows, 1 << 22)[:, :cols].view(torch.float8_e4m3fn)
    far = cstep.coded_blocks(codes, torch.zeros(-(-rows // GROUP), 4, dtype=torch.uint8, device="cuda")[:, :2])
    plain = torch.zeros(rows, 208, dtype=torch.uint8, device="cuda")[:, :cols].view(torch.float8_e4m3fn)
    near = cstep.coded_blocks(plain, torch.zeros(-(-rows // GROUP), 4, dtype=torch.uint8, device="cuda")[:, :2])
    theta = torch.zeros(rows, cols, device="cuda")
    ctx.encode_blocks(w.contiguous(), near, theta=theta)
    ctx.encode_blocks(w, far, theta=w)
    assert torch.equal(far.codes.view(torch.uint8), plain.view(torch.uint8)) and torch.equal(far.scales, near.scales) and torch.equal(w, theta)
    wide = (near.scales.double() - 127).exp2().repeat_interleave(GROUP, 0)[:rows].repeat_interleave(GROUP, 1)[:, :cols]
    assert torch.equal(theta.double(), plain.double() * wide)
