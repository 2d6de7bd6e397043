"""Which copies of a ring are waited for when a kernel gives up (csrc/ring.h), against a model of the stages' barriers. No GPU needed."""
import os
import random
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "ring.h"
#include <cstdio>
int main()
{
    int issued, stages;
    while (scanf("%d %d", &issued, &stages) == 2) {
        cs::copies_under_way(issued, stages, [](int s, int parity) { printf("%d %d ", s, parity); });
        printf("\n");
    }
    return 0;
}
"""


def _waits(tmp_path, cases):
    src, exe = str(tmp_path / "t.cpp"), str(tmp_path / "t")
    open(src, "w").write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1911_02497_b200", "csrc"), "-o", exe, src], check=True)
    out = subprocess.run([exe], input="\n".join("%d %d" % c for c in cases), capture_output=True, text=True, check=True).stdout.split("\n")
    lines = [[int(x) for x in line.split()] for line in out[:len(cases)]]
    return [list(zip(v[::2], v[1::2])) for v in lines]


def test_waits_end_when_all_that_was_issued_has_landed_and_not_before(tmp_path):
    """A stage's barrier has completed as many phases as copies into it have landed; a wait for parity p ends when the phase under way has the other
    one. A copy is issued when the one before it in its stage has landed."""
    rng = random.Random(1)
    cases = [(issued, stages) for stages in (1, 2, 3, 8, 12) for issued in range(0, 5 * stages + 2)]
    for (issued, stages), waits in zip(cases, _waits(tmp_path, cases)):
        assert len(waits) == min(issued, stages) and len({s for s, _ in waits}) == len(waits)
        uses = [len(range(s, issued, stages)) for s in range(stages)]
        for missing in range(8):
            late = {s for s in range(stages) if uses[s] and missing and rng.random() < 0.4}
            completed = [uses[s] - (s in late) for s in range(stages)]
            assert all(((completed[s] & 1) != p) == (s not in late) for s, p in waits)


BATCHES = r"""
#include "ring.h"
#include <cstdio>
int main()
{
    for (int batch = 1; batch <= 3; ++batch)
        for (int items = 0; items <= 40; ++items) printf("%d %d\n", (int)cs::last_batch_commits(items, batch, 0), (int)cs::last_batch_commits(items, batch, 1));
    return 0;
}
"""


def test_the_last_commit_of_each_side(tmp_path):
    """Two sides fill batches in turn, each behind the commit of its batch before; what is committed and has not been waited for then."""
    src, exe = str(tmp_path / "b.cpp"), str(tmp_path / "b")
    open(src, "w").write(BATCHES)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1911_02497_b200", "csrc"), "-o", exe, src], check=True)
    lines = [tuple(map(int, x.split())) for x in subprocess.run([exe], capture_output=True, text=True, check=True).stdout.splitlines()]
    for (batch, items), got in zip(((b, n) for b in (1, 2, 3) for n in range(41)), lines):
        sizes = [min(batch, items - at) for at in range(0, items, batch)]
        for side in (0, 1):
            mine = sizes[side::2]
            committed, waited = sum(n == batch for n in mine), max(len(mine) - 1, 0)
            assert got[side] == committed - waited if mine else got[side] == 0
