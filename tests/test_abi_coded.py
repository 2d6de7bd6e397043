"""The ctypes mirrors of the 8-bit operators' structs, and what the binding refuses (no GPU needed)."""
import ctypes
import os
import subprocess
import tempfile

import numpy as np
import pytest

from coded_util import encode, e4m3_round, e4m3_value, scale_bytes

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


def test_struct_mirrors_match_the_header():
    from paper_1911_02497_b200 import cstep
    fields = {"condensa_coded": (cstep.CodedMatrix, ["codes", "scales", "ld", "ld_scales"]), "condensa_projection": (cstep.Projection, ["code", "n", "k"]),
              "condensa_norm": (cstep.Norm, ["residual", "code", "rstd", "ldy", "cols", "eps", "gain_dtype", "reserved"]),
              "condensa_norm_gradient": (cstep.NormGradient, ["rstd", "dx", "code", "dgain", "ld_dx", "cols", "accumulate", "reserved"])}
    lines, want = [], []
    for name, (cls, members) in fields.items():
        lines.append('printf("%%zu\\n", sizeof(%s));' % name)
        want.append(ctypes.sizeof(cls))
        for m in members:
            lines.append('printf("%%zu\\n", offsetof(%s, %s));' % (name, m))
            want.append(getattr(cls, m).offset)
    lines.append('printf("%d\\n", CONDENSA_CODE_GROUP);')
    want.append(cstep.CODE_GROUP)
    src = '#include <stdio.h>\n#include <stddef.h>\n#include "condensa_cstep.h"\nint main(void){%s return 0;}\n' % "".join(lines)
    with tempfile.TemporaryDirectory() as d:
        c, exe = os.path.join(d, "s.c"), os.path.join(d, "s")
        open(c, "w").write(src)
        subprocess.run(["gcc", "-std=c99", "-Wall", "-Werror", "-I", os.path.join(ROOT, "include"), "-o", exe, c], check=True)
        got = [int(x) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.split()]
    assert got == want


def test_the_8_bit_form_of_the_tests():
    """The definition that the GPU tests go by, against values taken by hand."""
    assert list(e4m3_value([0x00, 0x01, 0x08, 0x38, 0x7E, 0xFE])) == [0.0, 2.0 ** -9, 2.0 ** -6, 1.0, 448.0, -448.0] and np.isnan(e4m3_value([0x7F])).all()
    assert list(e4m3_round(np.array([1.0625, 1.1875, -447.0, 2.0 ** -10, 3 * 2.0 ** -10, 464.0 - 1e-9]))) == [1.0, 1.25, -448.0, 0.0, 2.0 ** -8, 448.0]
    assert list(scale_bytes(np.array([0.0, 448.0, 448.0001, 1.0, 2.0 ** -149, 2.0 ** -118, 3.4e38]))) == [1, 127, 128, 119, 1, 1, 247]
    q, s = encode(np.array([[1.0, np.nan, -2.0, np.inf]]))
    assert s[0, 0] == 120 and list(q[0, ::2]) == [128.0, -256.0] and np.isnan(q[0, 1]) and np.isnan(q[0, 3])


class _Recorder:
    """Stands in for the library: keeps the calls, launches nothing."""

    def __init__(self):
        self.calls = []

    def __getattr__(self, name):
        return lambda *args: self.calls.append((name, args)) or 0


def _context():
    from paper_1911_02497_b200 import cstep
    ctx = cstep.Context.__new__(cstep.Context)
    ctx._lib, ctx._h, ctx.device = _Recorder(), None, -1          # (tensors of the CPU are on "device" -1)
    return ctx


def _coded(rows, cols, high=1):
    import torch
    from paper_1911_02497_b200 import cstep
    codes = torch.zeros(rows, -(-cols // 16) * 16, dtype=torch.uint8)[:, :cols].view(torch.float8_e4m3fn)
    groups = -(-cols // 128)
    scales = torch.zeros(-(-rows // high), -(-groups // 4) * 4, dtype=torch.uint8)[:, :groups]
    return (cstep.coded_rows if high == 1 else cstep.coded_blocks)(codes, scales)


def test_coded_describes_and_refuses():
    import torch
    from paper_1911_02497_b200 import cstep
    c = _coded(300, 1500, 128)
    assert (c.struct.ld, c.struct.ld_scales, c.projection.n, c.projection.k) == (1504, 12, 300, 1500)
    one = cstep.coded_rows(torch.zeros(1, 1500, dtype=torch.uint8), torch.zeros(1, 12, dtype=torch.uint8))      # a single row's stride says nothing
    assert (one.struct.ld, one.struct.ld_scales) == (1504, 12)
    codes, scales = torch.zeros(4, 256, dtype=torch.uint8), torch.zeros(4, 4, dtype=torch.uint8)[:, :2]
    for bad in ((codes[:, :250], scales[:, :1]), (codes, torch.zeros(4, 2, dtype=torch.uint8)), (torch.zeros(4, 250, dtype=torch.uint8), scales),
                (codes.view(-1)[8:8 + 3 * 256].view(3, 256), scales[:3]), (codes.t(), scales), (codes[0], scales)):
        with pytest.raises(ValueError):
            cstep.coded_rows(*bad)
    with pytest.raises(TypeError):
        cstep.coded_rows(codes.float(), scales)
    with pytest.raises(TypeError):
        cstep.coded_rows(codes, scales.int())


def test_calls_refuse_what_does_not_fit():
    import torch
    from paper_1911_02497_b200 import cstep
    ctx, w, x = _context(), _coded(40, 200, 128), _coded(5, 200)
    y, dy, dx = torch.zeros(5, 40).half(), _coded(5, 40), torch.zeros(5, 200).half()
    ctx.projection_forward(w, x, y)
    ctx.projection_backward(w, dy, dx)
    assert [c[0] for c in ctx._lib.calls] == ["condensa_projection_forward", "condensa_projection_backward"]
    ctx._lib.calls.clear()
    g, f, v = torch.ones(200), torch.zeros(5, 200), torch.zeros(5)
    for call in (lambda: ctx.projection_forward(x, x, y), lambda: ctx.projection_forward(w, w, y), lambda: ctx.projection_forward(w, x, y.float()),
                 lambda: ctx.norm_forward(f.int(), g), lambda: ctx.norm_forward(f.half(), g.bfloat16()), lambda: ctx.norm_forward(f, g, code=w),
                 lambda: ctx.norm_backward(f, f, g, v.double()), lambda: ctx.encode_blocks(f, x), lambda: ctx.encode_rows(f.double(), x)):
        with pytest.raises(TypeError):
            call()
    for call in (lambda: ctx.projection_forward(w, dy, y), lambda: ctx.projection_forward(w, x, dx), lambda: ctx.projection_backward(w, x, dx),
                 lambda: ctx.norm_forward(f, g[:199]), lambda: ctx.norm_forward(f, g, residual=f[:4]), lambda: ctx.norm_forward(f, g, y=f.half()),
                 lambda: ctx.norm_forward(f, g, rstd=v[:4]), lambda: ctx.norm_forward(f.t().contiguous().t(), g), lambda: ctx.norm_forward(f, g, code=dy),
                 lambda: ctx.norm_backward(f, f[:, :100], g, v), lambda: ctx.norm_backward(f, f, g, v, dgain=v), lambda: ctx.encode_rows(f[:4], x),
                 lambda: ctx.encode_blocks(torch.zeros(40, 200), w, theta=torch.zeros(40, 100))):
        with pytest.raises(ValueError):
            call()
    ctx.device = 0                  # (the tensors are on another device now)
    for call in (lambda: ctx.projection_forward(w, x, y), lambda: ctx.norm_forward(f, g, y=f), lambda: ctx.norm_backward(f, f, g, v),
                 lambda: ctx.encode_rows(f, x), lambda: ctx.encode_blocks(torch.zeros(40, 200), w)):
        with pytest.raises(ValueError):
            call()
    assert not ctx._lib.calls
