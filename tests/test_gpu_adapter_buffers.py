"""Where the adapters' matrices may lie: slices of one buffer, and sizes that no buffer has."""
import ctypes as C

import numpy as np
import pytest

pytestmark = pytest.mark.gpu


@pytest.fixture()
def ctx():
    from paper_1911_02497_b200 import cstep
    c = cstep.Context(0)
    yield c
    c.close()


def test_column_slices_of_one_buffer(ctx):
    """x and y, dy and dx side by side in the rows of one buffer, as a fused projection writes them."""
    import torch
    from paper_1911_02497_b200 import cstep
    m, k, n, r = 70, 64, 128, 8
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0)
    draw = lambda *s: torch.randn(*s, device="cuda", generator=gen).bfloat16()
    a, b, wide, back = draw(r, k), draw(n, r), draw(m, k + n + 16), draw(m, k + n)
    ga, gb = [[torch.zeros(s, device="cuda") for _ in range(2)] for s in ((r, k), (n, r))]
    tabs = [cstep.adapter_table([a], [b], [0.5], [ga[i]], [gb[i]]) for i in (0, 1)]
    x, y, dy, dx = wide[:, :k].clone(), wide[:, k:k + n].clone(), back[:, :n].clone(), back[:, n:].clone()
    hs = [torch.zeros(m, r, device="cuda") for _ in range(2)]
    rest = wide[:, k + n:].clone()
    ctx.adapter_forward(tabs[0], [m], [0], x, y, hs[0])
    ctx.adapter_backward(tabs[0], [m], [0], x, dy, hs[0], dx)
    ctx.adapter_forward(tabs[1], [m], [0], wide[:, :k], wide[:, k:k + n], hs[1])
    ctx.adapter_backward(tabs[1], [m], [0], wide[:, :k], back[:, :n], hs[1], back[:, n:])
    torch.cuda.synchronize()
    assert torch.equal(wide[:, :k], x) and torch.equal(wide[:, k:k + n], y) and torch.equal(wide[:, k + n:], rest)
    assert torch.equal(back[:, :n], dy) and torch.equal(back[:, n:], dx) and torch.equal(hs[0], hs[1])
    assert torch.equal(ga[0], ga[1]) and torch.equal(gb[0], gb[1])
    launches = ctx.launch_count()
    with pytest.raises(cstep.CondensaError) as e:            # a column in common
        ctx.adapter_forward(tabs[1], [m], [0], wide[:, :k], wide[:, k - 1:k - 1 + n], hs[1])
    assert e.value.code == cstep.ERR_INVALID_ARG and ctx.launch_count() == launches


def test_rows_that_leave_the_address_space_are_refused(ctx):
    """Rows times stride beyond 63 bits must not wrap around in the overlap check."""
    import torch
    from paper_1911_02497_b200 import cstep
    a, b = torch.zeros(4, 64, device="cuda").half(), torch.zeros(32, 4, device="cuda").half()
    tab, some = cstep.adapter_table([a], [b], [1.0]), torch.zeros(4096, device="cuda")
    length, which = np.array([(1 << 31) - 1], dtype=np.int64), np.zeros(1, dtype=np.int32)
    batch = cstep.AdapterBatch(tab.address, 1, 1, length.ctypes.data, which.ctypes.data, int(length[0]), 64, 32, tab.code, 0)
    launches, p = ctx.launch_count(), some.data_ptr()
    for ldx, ldy in ((1 << 40, 32), (64, 1 << 40), (1 << 33, 1 << 33), ((1 << 40) + 1, 32)):
        rc = ctx._lib.condensa_adapter_forward(ctx._h, C.byref(batch), p, ldx, p + 8192, ldy, None, 0, None)
        assert rc == cstep.ERR_TOO_LARGE
    assert ctx.launch_count() == launches


def test_h_of_a_batch_without_adapters(ctx):
    """No row has an adapter: h has no column to keep, whatever stride it is given with."""
    import torch
    from paper_1911_02497_b200 import cstep
    a, b = torch.zeros(4, 64, device="cuda").half(), torch.zeros(32, 4, device="cuda").half()
    tab, some = cstep.adapter_table([a], [b], [1.0]), torch.zeros(4096, device="cuda")
    length, which = np.array([3], dtype=np.int64), np.full(1, -1, dtype=np.int32)
    batch = cstep.AdapterBatch(tab.address, 1, 1, length.ctypes.data, which.ctypes.data, 3, 64, 32, tab.code, 0)
    p = some.data_ptr()
    for ldh in (0, 1, 64):
        assert ctx._lib.condensa_adapter_forward(ctx._h, C.byref(batch), p, 64, p + 4096, 32, p + 8192, ldh, None) == cstep.OK
    torch.cuda.synchronize()
    assert bool((some == 0).all())


def test_the_longest_batch(ctx):
    """2^31 - 64 rows are taken (and then miss their x); one more is refused for its length: tiles count past the last row."""
    import torch
    from paper_1911_02497_b200 import cstep
    a, b = torch.zeros(1, 1, device="cuda").half(), torch.zeros(1, 1, device="cuda").half()
    tab, which = cstep.adapter_table([a], [b], [1.0]), np.zeros(2, dtype=np.int32)
    launches, most = ctx.launch_count(), (1 << 31) - 64
    for rows, code in (([most, 0], cstep.ERR_INVALID_ARG), ([most - 1, 1], cstep.ERR_INVALID_ARG), ([most, 1], cstep.ERR_TOO_LARGE),
                       ([(1 << 31) - 1, 0], cstep.ERR_TOO_LARGE), ([1, 1 << 62], cstep.ERR_TOO_LARGE)):
        length = np.array(rows, dtype=np.int64)
        batch = cstep.AdapterBatch(tab.address, 1, 2, length.ctypes.data, which.ctypes.data, int(sum(rows)), 1, 1, tab.code, 0)
        assert ctx._lib.condensa_adapter_forward(ctx._h, C.byref(batch), None, 1, None, 1, None, 0, None) == code
        assert ctx._lib.condensa_adapter_backward(ctx._h, C.byref(batch), None, 1, None, 1, None, 0, None, 0, 0, None) == code
    assert ctx.launch_count() == launches
