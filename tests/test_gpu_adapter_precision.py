"""Errors of the adapters that do not show where terms cancel: sums of one sign, against 64 bits.

The matrix instruction truncates its sums. Of the S products that follow one another in a sum, each loses at most 2^-23 of what
has been summed by then, half of the whole on average: S * 2^-24 of the sum. What is kept apart so is added with rounding, at random
signs. An fp32 operand is two TF32 parts, the second cut below 2^-22 of it: two operands and the product of both second parts are
3 * 2^-22 at most. These losses all go one way, so they show in the mean over many results; the largest error has the rounded
sums beside it (six standard deviations of N of them, each at most 2^-24)."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

EPS = 2.0 ** -24
PARTS = {"float32": 3 * 2.0 ** -22, "float16": 0.0, "bfloat16": 0.0}


def _torch():
    import torch
    return torch


@pytest.fixture()
def ctx():
    from paper_1911_02497_b200 import cstep
    c = cstep.Context(0)
    yield c
    c.close()


def matrix(rows, width, dtype, pad=0, low=0.5, high=1.0):
    """Values of one sign on the device, rows ``pad`` elements apart and one element off where there is a ``pad``."""
    torch = _torch()
    off = 1 if pad else 0
    room = torch.empty(off + rows * (width + pad), device="cuda", dtype=getattr(torch, dtype))
    v = torch.as_strided(room, (rows, width), (width + pad, 1), off)
    for i in range(0, rows, 4096):
        part = v[i:i + 4096]
        part.copy_(torch.rand(part.shape, device="cuda") * (high - low) + low)
    return v


def check(got, want, bias, largest, what):
    r = (got.double() - want) / want
    assert abs(float(r.mean())) <= bias, (what, float(r.mean()), bias)
    assert float(r.abs().max()) <= largest, (what, float(r.abs().max()), largest)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rank,pad", [(8, 0), (8, 1), (8, 4), (32, 0), (40, 0), (64, 2), (100, 0), (128, 0), (128, 3)])
def test_h_of_a_wide_row(ctx, dtype, rank, pad):
    """Whatever the rank and however the rows lie: rows enough that a CTA has the whole width of its tile."""
    torch = _torch()
    from paper_1911_02497_b200 import cstep
    k, n, rows = 9216, 64, 19200
    torch.manual_seed(rank + pad)
    x, y, h = matrix(rows, k, dtype, pad), matrix(rows, n, dtype, pad), torch.zeros(rows, rank, device="cuda")
    a, b = matrix(rank, k, dtype), matrix(n, rank, dtype)
    ctx.adapter_forward(cstep.adapter_table([a], [b], [1.0]), [rows], [0], x, y, h)
    torch.cuda.synchronize()
    want = torch.cat([x[i:i + 4096].double() @ a.double().t() for i in range(0, rows, 4096)])
    # a step is at most 128 bytes of a row: 4 products of 16 terms, or 4 times 3 of 8
    S = 12 if dtype == "float32" else 4
    loss, sums = S * EPS + PARTS[dtype], k * x.element_size() / 64
    check(h, want, loss + EPS / 4, 2 * loss + 6 * np.sqrt(sums) * EPS, (dtype, rank, pad))


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
def test_h_does_not_depend_on_the_other_adapters_of_the_call(ctx, dtype):
    """An adapter of rank 8 in a call with one of rank 128 is as exact as alone."""
    torch = _torch()
    from paper_1911_02497_b200 import cstep
    k, n, rows = 9216, 64, 9600
    torch.manual_seed(1)
    x, y, h = matrix(2 * rows, k, dtype), matrix(2 * rows, n, dtype), torch.zeros(2 * rows, 128, device="cuda")
    a, b = [matrix(r, k, dtype) for r in (8, 128)], [matrix(n, r, dtype) for r in (8, 128)]
    ctx.adapter_forward(cstep.adapter_table(a, b, [1.0, 1.0]), [rows, rows], [0, 1], x, y, h)
    torch.cuda.synchronize()
    S = 12 if dtype == "float32" else 4
    loss = S * EPS + PARTS[dtype]
    for i in (0, 1):
        at = slice(i * rows, (i + 1) * rows)
        want = torch.cat([x[at][j:j + 4096].double() @ a[i].double().t() for j in range(0, rows, 4096)])
        check(h[at][:, :a[i].shape[0]], want, loss + EPS / 4, 2 * loss + 6 * np.sqrt(k * x.element_size() / 64) * EPS, (dtype, i))


@pytest.mark.parametrize("rank", [8, 16, 17, 32, 64, 100, 128])
def test_expansion_in_fp32(ctx, rank):
    """y = B h and dx = A^T u at ranks up to the largest, beside the h and u that they were formed from."""
    torch = _torch()
    from paper_1911_02497_b200 import cstep
    k, n, rows = 64, 2048, 4096
    torch.manual_seed(rank)
    x, h = matrix(rows, k, "float32"), torch.zeros(rows, rank, device="cuda")
    y, dy, dx = torch.zeros(rows, n, device="cuda"), matrix(rows, n, "float32"), torch.zeros(rows, k, device="cuda")
    a, b, ga = matrix(rank, k, "float32"), matrix(n, rank, "float32"), torch.zeros(rank, k, device="cuda")
    tab = cstep.adapter_table([a], [b], [1.0], [ga])
    ctx.adapter_forward(tab, [rows], [0], x, y, h)
    ctx.adapter_backward(tab, [rows], [0], x, dy, None, dx)
    torch.cuda.synchronize()
    S, sums = 6, rank / 16 + 1              # 3 products of 8 terms, twice, before a rounded sum; y and dx start at 0
    most, mean = PARTS["float32"], 2.0 ** -22       # what is cut off an operand is half of the most on average, and 2 operands lose it
    loss = S * EPS + mean
    check(y, h.double() @ b.double().t(), loss, 2 * S * EPS + most + 6 * np.sqrt(sums) * EPS, ("y", rank))
    u_loss = 12 * EPS + mean                # (u is not handed out: its own loss comes first)
    want = (dy.double() @ b.double()) @ a.double()
    check(dx, want, loss + u_loss + EPS, 2 * (S + 12) * EPS + 2 * most + 12 * np.sqrt(sums + n / 16) * EPS, ("dx", rank))


def gradients(ctx, dtype, x, dy, a, b, h, scale=1.0):
    torch = _torch()
    from paper_1911_02497_b200 import cstep
    rank, k, n = a.shape[0], a.shape[1], b.shape[0]
    ga, gb = torch.zeros(rank, k, device="cuda"), torch.zeros(n, rank, device="cuda")
    ctx.adapter_backward(cstep.adapter_table([a], [b], [scale], [ga], [gb]), [x.shape[0]], [0], x, dy, h)
    torch.cuda.synchronize()
    return ga, gb


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rank,rows", [(4, 64), (16, 1000), (31, 130), (50, 700), (64, 64), (128, 300)])
def test_gradients_of_ranks_that_differ_by_powers_of_two(ctx, dtype, rank, rows):
    """Columns of B (which make u) and of h down to 2^-30 of one another: AdamW divides each by its own size."""
    torch = _torch()
    k, n = 264, 200
    torch.manual_seed(rank)
    size = 2.0 ** (10 - 10 * (torch.arange(rank, device="cuda") % 4).float())       # 2^10 .. 2^-20, as binary16 holds them
    x, dy, a = matrix(rows, k, dtype), matrix(rows, n, dtype), matrix(rank, k, dtype)
    # (values of B that binary16 holds exactly under every size: 1, 1.25 or 1.5, of 2^-20 too)
    b = ((1 + 0.25 * torch.randint(0, 3, (n, rank), device="cuda")) * size).to(getattr(torch, dtype))
    h = matrix(rows, rank, "float32") * size
    ga, gb = gradients(ctx, dtype, x, dy, a, b, h)
    u = dy.double() @ b.double()
    # per sum: the row kernel's u (dA only), then tiles of 64 rows, 8 products of 16-bit parts in a row (fp32: 12) each
    S, parts = (12, PARTS["float32"]) if dtype == "float32" else (12, 2.0 ** -21)
    largest = 2 * 2 * S * EPS + 2 * parts + 6 * np.sqrt(rows / 32 + n / 16 + 16) * EPS
    for name, got, want in (("dA", ga, u.t() @ x.double()), ("dB", gb, dy.double().t() @ h.double())):
        check(got, want, 2 * S * EPS + parts, largest, (name, dtype, rank))


@pytest.mark.parametrize("rank", [8, 24, 50, 100])
def test_an_infinite_coefficient_leaves_the_other_ranks_alone(ctx, rank):
    """binary16: beside it stand coefficients above 65504 and far below 6e-8."""
    torch = _torch()
    rows, k, n = 200, 72, 136
    torch.manual_seed(rank)
    x, dy, a, b = matrix(rows, k, "float16"), matrix(rows, n, "float16"), matrix(rank, k, "float16"), matrix(n, rank, "float16")
    h = matrix(rows, rank, "float32") * 10.0 ** (6 - 6 * (torch.arange(rank, device="cuda") % 3).float())
    bad = h.clone()
    bad[70, 0] = float("inf")
    _, want = gradients(ctx, "float16", x, dy, a, b, h)
    _, got = gradients(ctx, "float16", x, dy, a, b, bad)
    assert torch.isfinite(want).all() and not torch.isfinite(got[:, 0]).any()
    assert torch.equal(got[:, 1:], want[:, 1:])
    exact = dy.double().t() @ h.double()
    check(want, exact, 12 * EPS + 2.0 ** -21, 24 * EPS + 2.0 ** -20 + 6 * np.sqrt(rows / 32 + 16) * EPS, rank)


@pytest.mark.parametrize("dtype", ["float32", "float16", "bfloat16"])
@pytest.mark.parametrize("rows", [7, 300])
@pytest.mark.parametrize("rank", [6, 30, 64, 100])
def test_small_ranks_of_a_row_with_columns_of_their_own(ctx, dtype, rows, rank):
    """h of some ranks 2^-10 and 2^-20 of the others'; each column of y hangs on ranks of one size alone, and so does dx."""
    torch = _torch()
    from paper_1911_02497_b200 import cstep
    k = n = 240
    torch.manual_seed(rank)
    t = getattr(torch, dtype)
    kind = torch.arange(rank, device="cuda") % 3
    own = (torch.arange(n, device="cuda")[:, None] % 3 == kind[None, :]).float()
    down, up = 2.0 ** (5 - 10 * kind.float()), 2.0 ** (10 * kind.float() - 12)
    shrink, expand = (torch.rand(rank, k, device="cuda") * 0.5 + 0.5) * down[:, None], (torch.rand(n, rank, device="cuda") * 0.5 + 0.5) * up * own
    x, h = matrix(rows, k, dtype), torch.zeros(rows, rank, device="cuda")
    # forward with A = shrink, B = expand; backward with B^T = shrink, A^T = expand, so u takes h's part
    a, b, y = shrink.to(t), expand.to(t), torch.zeros(rows, n, device="cuda", dtype=t)
    ctx.adapter_forward(cstep.adapter_table([a], [b], [1.0]), [rows], [0], x, y, h)
    at, bt, dx = expand.t().contiguous().to(t), shrink.t().contiguous().to(t), torch.zeros(rows, n, device="cuda", dtype=t)
    ctx.adapter_backward(cstep.adapter_table([at], [bt], [1.0]), [rows], [0], x, x, None, dx)
    torch.cuda.synchronize()
    hw = x.double() @ a.double().t()
    want = hw @ b.double().t()
    # parts of h: 2^-16 (bfloat16) or 2^-21 of each, and 2^-38 of the row's largest in binary16; sums: S as above; one rounding to the type
    part = {"float32": 2.0 ** -21, "float16": 2.0 ** -21, "bfloat16": 2.0 ** -16}[dtype]
    floor = 2.0 ** -38 * hw.max(dim=1, keepdim=True).values * b.double().sum(dim=1)[None, :] if dtype == "float16" else 0.0
    half = {"float32": EPS, "float16": 2.0 ** -11, "bfloat16": 2.0 ** -8}[dtype]
    allowed = (2 * part + 48 * EPS + half) * want + floor
    for name, got in (("y", y), ("dx", dx)):
        off = (got.double() - want).abs()
        assert bool((off <= allowed).all()), (name, float((off / allowed).max()))


@pytest.mark.parametrize("dtype,top", [("float32", 0x7F7FEFFF), ("bfloat16", 0x7F7F7FFF), ("float16", 0x7F7FFFFF)])
def test_values_at_the_top_of_fp32_that_are_still_numbers(ctx, dtype, top):
    """The largest fp32 operand, and the largest h beside 16-bit operands, that the header calls a number; under a small factor."""
    torch = _torch()
    from paper_1911_02497_b200 import cstep
    rows, k, n, rank = 70, 40, 24, 3
    value = float(np.array([top], np.uint32).view(np.float32)[0])
    t = getattr(torch, dtype)
    a, b = torch.full((rank, k), 2.0 ** -8, device="cuda", dtype=t), torch.full((n, rank), 2.0 ** -8, device="cuda", dtype=t)
    dy, h = torch.full((rows, n), 2.0 ** -8, device="cuda", dtype=t), torch.zeros(rows, rank, device="cuda")
    h[:, 1], h[66] = -2.0, 0.25
    h[:, 0] = torch.where(torch.arange(rows, device="cuda") == 66, value, 1.0)
    x = torch.zeros(rows, k, device="cuda", dtype=t)
    if dtype == "float32":
        x[5, 7] = value
        y, hx = torch.zeros(rows, n, device="cuda"), torch.zeros(rows, rank, device="cuda")
        ctx.adapter_forward(cstep.adapter_table([a], [b], [1.0]), [rows], [0], x, y, hx)
        torch.cuda.synchronize()
        check(hx[5], torch.full((rank,), value * 2.0 ** -8, device="cuda").double(), 2.0 ** -21, 2.0 ** -21, "h")
        check(y[5], torch.full((n,), 3 * value * 2.0 ** -16, device="cuda").double(), 2.0 ** -19, 2.0 ** -19, "y")
        assert bool((y[:5] == 0).all()) and bool((y[6:] == 0).all())
    _, gb = gradients(ctx, dtype, x, dy, a, b, h)
    want = 2.0 ** -8 * h.double().sum(dim=0).expand(n, rank)
    check(gb, want, 2.0 ** -19, 2.0 ** -19, "dB")
