"""The ctypes mirrors of the list operators' and the adapters' structs have the layout that the header gives them, and the
tables refuse what they cannot describe (no GPU needed)."""
import ctypes
import os
import subprocess
import tempfile

import numpy as np
import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_mirrors_match_the_header():
    from paper_1911_02497_b200 import cstep
    fields = {"condensa_adamw_tensor": (cstep.AdamwTensor, ["w", "lambda", "m_scale", "w_h", "numel"]),
              "condensa_adamw": (cstep.Adamw, ["weight_decay", "grad_scale", "step", "w_h_dtype"]),
              "condensa_adapter": (cstep.Adapter, ["a", "grad_b", "scale", "rank"]),
              "condensa_adapter_batch": (cstep.AdapterBatch, ["adapters", "n_requests", "request_adapter", "rows", "k", "n", "dtype"])}
    mirror = {"lambda": "lam"}
    lines, want = [], []
    for name, (cls, members) in fields.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(ctypes.sizeof(cls))
        for m in members:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, m))
            want.append(getattr(cls, mirror.get(m, m)).offset)
    lines.append('printf("%zu\\n", sizeof(condensa_clip));')
    want.append(16)
    lines.append('printf("%d\\n", CONDENSA_STATE_BLOCK); printf("%d\\n", CONDENSA_ADAPTER_MAX_RANK); printf("%d\\n", CONDENSA_DTYPE_FP32);')
    want += [cstep.STATE_BLOCK, cstep.ADAPTER_MAX_RANK, cstep.DTYPE_FP32]
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "condensa_cstep.h"\nint main(void){%s return 0;}\n' % "".join(lines)
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "s.c"), os.path.join(d, "s")
        open(c, "w").write(src)
        subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", exe, c], check=True)
        got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == want


def test_adamw_table_describes_and_refuses():
    import torch
    from paper_1911_02497_b200 import cstep
    w, g = [torch.zeros(300), torch.zeros(5)], [torch.zeros(300, dtype=torch.bfloat16), torch.zeros(5, dtype=torch.bfloat16)]
    code = [torch.zeros(300, dtype=torch.uint8), torch.zeros(5, dtype=torch.uint8)]
    scale = [torch.zeros(2), torch.zeros(1)]
    tab = cstep.adamw_table(w, g, code, code, scale, scale, w_h=[torch.zeros(300, dtype=torch.float16), None])
    assert (tab.T, tab.grad_dtype, tab.state_dtype, tab.w_h_dtype) == (2, cstep.DTYPE_BF16, cstep.DTYPE_FP8_E4M3, cstep.DTYPE_FP16)
    assert tab.entries[0].w == w[0].data_ptr() and tab.entries[1].w_h is None and tab.entries[1].numel == 5
    with pytest.raises(ValueError):
        cstep.adamw_table(w, g, code, code, [torch.zeros(1), torch.zeros(1)], scale)        # 300 elements need two scales
    with pytest.raises(TypeError):
        cstep.adamw_table(w, [g[0], g[1].float()], code, code, scale, scale)                 # one type of gradient per list
    with pytest.raises(TypeError):
        cstep.adamw_table([x.half() for x in w], g)
    with pytest.raises(ValueError):
        cstep.adamw_table([torch.zeros(301), w[1]], g)


def test_adapter_table_describes_and_refuses():
    import torch
    from paper_1911_02497_b200 import cstep
    a, b = [torch.zeros(4, 32).half(), torch.zeros(7, 32).half()], [torch.zeros(48, 4).half(), torch.zeros(48, 7).half()]
    tab = cstep.adapter_table(a, b, [1.0, 0.5], None, [None, torch.zeros(48, 7)])
    assert (tab.count, tab.k, tab.n, tab.code) == (2, 32, 48, cstep.DTYPE_FP16)
    assert tab.entries[1].rank == 7 and tab.entries[1].scale == 0.5 and tab.entries[0].grad_b is None and tab.entries[0].grad_a is None
    for bad in ((a[:1], b, [1.0]), ([], [], []), (a, [b[0], b[0]], [1.0, 1.0]), ([a[0], a[1].t().contiguous().t()], b, [1.0, 1.0])):
        with pytest.raises(ValueError):
            cstep.adapter_table(*bad)
    with pytest.raises(TypeError):
        cstep.adapter_table([a[0], a[1].float()], b, [1.0, 1.0])
    with pytest.raises(TypeError):
        cstep.adapter_table(a, b, [1.0, 1.0], [torch.zeros(4, 32).half(), None])


def test_host_arrays_of_requests():
    from paper_1911_02497_b200 import cstep
    x = np.arange(4, dtype=np.int64)
    assert cstep._host_array(x, cstep._INT64) is x
    assert cstep._host_array([1, 2], cstep._INT32).dtype == np.int32
    assert cstep._host_array(x[::2], cstep._INT64).flags.c_contiguous


class _Recorder:
    """Stands in for the library: keeps the calls, launches nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


def _context():
    from paper_1911_02497_b200 import cstep
    ctx = cstep.Context.__new__(cstep.Context)
    ctx._lib, ctx._h = _Recorder(), None
    return ctx


def _adapter_calls(ctx, tab, rows, which, h):
    """Both calls with this h; the row stride of h that each passed on."""
    import torch
    m = int(sum(rows))
    x, y = (torch.zeros(m, w, dtype=torch.float16) for w in (tab.k, tab.n))
    ctx._lib.calls.clear()
    ctx.adapter_forward(tab, rows, which, x, y, h)
    ctx.adapter_backward(tab, rows, which, x, y, h, torch.zeros_like(x))
    (_, f), (_, b) = ctx._lib.calls
    return f[7], b[7]


def test_h_narrower_than_the_ranks_is_refused_before_the_library_is_called():
    """A view of few columns has the row stride of the matrix that it was taken from, which says nothing of its width."""
    import torch
    from paper_1911_02497_b200 import cstep
    ranks, k, n = [4, 8, 100], 64, 48
    a, b = [torch.zeros(r, k).half() for r in ranks], [torch.zeros(n, r).half() for r in ranks]
    tab = cstep.adapter_table(a, b, [1.0] * 3, [torch.zeros(r, k) for r in ranks], [torch.zeros(n, r) for r in ranks])
    big, ctx = torch.zeros(5, 64), _context()
    for rows, which, h in (([3, 2], [0, 1], big[:, :4]), ([3, 2], [0, 1], big[:, 57:]), ([3, 2], [0, 1], torch.zeros(5, 4)),
                           ([1], [1], big[:1, :4]), ([1], [1], torch.zeros(1, 64)[:, 60:]), ([1, 0, 4], [0, 2, 2], big)):
        ctx._lib.calls.clear()
        x, y = (torch.zeros(sum(rows), w).half() for w in (k, n))
        for call in (lambda: ctx.adapter_forward(tab, rows, which, x, y, h), lambda: ctx.adapter_backward(tab, rows, which, x, y, h)):
            with pytest.raises(cstep.CondensaError) as e:
                call()
            assert e.value.code == cstep.ERR_INVALID_ARG
        assert not ctx._lib.calls
    # as wide as the adapters that have rows is enough
    assert _adapter_calls(ctx, tab, [3, 2], [0, 1], big[:, :8]) == (64, 64)
    assert _adapter_calls(ctx, tab, [3, 0, 2], [0, 2, -1], big[:, :4]) == (64, 64)
    assert _adapter_calls(ctx, tab, [1], [1], big[:1, :8])[0] >= 8
    assert _adapter_calls(ctx, tab, [3, 2], [0, 1], None) == (0, 0)
    # backward reads h for the gradients of B alone
    tab = cstep.adapter_table(a, b, [1.0] * 3, [torch.zeros(r, k) for r in ranks])
    x, y = torch.zeros(5, k).half(), torch.zeros(5, n).half()
    ctx._lib.calls.clear()
    ctx.adapter_backward(tab, [3, 2], [0, 1], x, y, big[:, :4])
    assert len(ctx._lib.calls) == 1
