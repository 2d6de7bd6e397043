"""How the encoder of rows is cut (csrc/row_runs.h). No GPU needed."""
import os
import random
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "row_runs.h"
#include <cstdio>
int main()
{
    long long rows;
    unsigned groups;
    while (scanf("%lld %u", &rows, &groups) == 2) {
        cs::RowRuns p;
        const int fits = cs::plan_row_runs(rows, groups, 16, p);
        long long wrong = 0;
        const unsigned long long all = (unsigned long long)p.grid * 16 * (4 / p.groups_of_run), step = all / 5000 + 1;
        for (unsigned long long u = 0; fits && u < all; u += step)
            for (unsigned long long v = u; v < u + 2 && v < all; ++v) {
                unsigned row, run;
                cs::place_of_run((unsigned)v, p.runs, p.reciprocal, [](unsigned a, unsigned b) { return (unsigned)(((unsigned long long)a * b) >> 32); }, row, run);
                wrong += row != v / p.runs || run != v % p.runs;
            }
        printf("%d %d %u %lld %lld\n", fits, p.groups_of_run, p.runs, p.grid, wrong);
    }
    return 0;
}
"""


def test_places_and_what_is_refused(tmp_path):
    src, exe = str(tmp_path / "t.cpp"), str(tmp_path / "t")
    open(src, "w").write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1911_02497_b200", "csrc"), "-o", exe, src], check=True)
    rng = random.Random(2)
    most = 2 ** 31 - 256
    cases = [(1, 1), (most, 1), (most, 2), (most, 4), (most, 5), (most, 8), (most, 32768), (2 ** 30, 16), (2 ** 30 - 64, 16), (131072, 32768), (524288, 32768), (524287, 32768)]
    cases += [(int(2 ** rng.uniform(0, 31)) or 1, int(2 ** rng.uniform(0, 15))) for _ in range(300)]
    out = subprocess.run([exe], input="\n".join("%d %d" % c for c in cases), capture_output=True, text=True, check=True).stdout.split("\n")
    for (rows, groups), line in zip(cases, out):
        fits, length, runs, grid, wrong = (int(v) for v in line.split())
        assert length in (1, 2, 4) and runs == -(-groups // length) and not wrong
        assert length == 1 or 4 * (runs * length - groups) <= groups
        per = 16 * (4 // length)
        assert grid == -(-rows * runs // per) and bool(fits) == (grid * per < 2 ** 32) and (not fits or grid < 2 ** 31)
    assert {line.split()[0] for line in out[:12]} == {"0", "1"}
