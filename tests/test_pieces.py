"""Which aligned 16 bytes are read for the values of a row that begins anywhere (csrc/pieces.h). No GPU needed."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "pieces.h"
#include <cstdio>
int main()
{
    for (int by = 0; by < cs::PIECE; ++by)
        for (int cols = 1; cols <= 40; ++cols)
            for (int c = 0; c < cols; c += 8) printf("%d %d %d %d\n", by, cols, c, cs::second_piece(by, c, cols) ? 2 : 1);
    return 0;
}
"""


def test_every_piece_holds_a_value_of_the_row_and_every_value_has_its_piece(tmp_path):
    src, exe = str(tmp_path / "t.cpp"), str(tmp_path / "t")
    open(src, "w").write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1911_02497_b200", "csrc"), "-o", exe, src], check=True)
    lines = [tuple(map(int, x.split())) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines()]
    assert len(lines) == 8 * (8 + 16 + 24 + 32 + 40)
    for by, cols, c, n in lines:
        held = {(by + i) // 8 for i in range(8) if c + i < cols}
        assert held == set(range(n)), (by, cols, c, n)
