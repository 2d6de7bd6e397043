"""The overlap check of a call's buffers (csrc/ranges.h) against sets of bytes. No GPU needed."""
import os
import random
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "ranges.h"
#include <cstdio>
int main()
{
    int n, m;
    while (scanf("%d %d", &n, &m) == 2) {
        std::vector<Interval> iv;
        std::vector<RowRange> rows;
        for (int i = 0; i < n; ++i) {
            unsigned long a, b; int o;
            if (scanf("%lu %lu %d", &a, &b, &o) != 3) return 1;
            iv.push_back({a, b, o != 0});
        }
        for (int i = 0; i < m; ++i) {
            unsigned long a, w, s, r; int o;
            if (scanf("%lu %lu %lu %lu %d", &a, &w, &s, &r, &o) != 5) return 1;
            rows.push_back({a, w, s, r, o != 0});
        }
        printf("%d\n", rows_clash(iv, rows) ? 1 : 0);
    }
    return 0;
}
"""


def _answers(tmp_path, cases):
    src, exe = str(tmp_path / "t.cpp"), str(tmp_path / "t")
    open(src, "w").write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1911_02497_b200", "csrc"), "-o", exe, src], check=True)
    text = "\n".join(" ".join(str(int(v)) for v in [len(iv), len(m)] + [x for e in iv + m for x in e]) for iv, m in cases)
    return [int(x) for x in subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split()]


def _bytes(e):
    if len(e) == 3:
        return set(range(e[0], e[1]))
    lo, width, stride, rows, _ = e
    return {lo + r * stride + i for r in range(rows) for i in range(width)}


def _overlap(iv, m):
    every = [(_bytes(e), e[-1]) for e in iv + m]
    return any((o or p) and x & y for i, (x, o) in enumerate(every) for y, p in every[:i])


def test_column_slices_of_one_buffer_do_not_clash(tmp_path):
    """x and y side by side in rows of 64 bytes; the same with one byte in common; y ahead of x; three slices."""
    cases = [([], [(100, 32, 64, 9, 0), (132, 32, 64, 9, 1)]), ([], [(100, 33, 64, 9, 0), (132, 32, 64, 9, 1)]),
             ([], [(132, 32, 64, 9, 0), (100, 32, 64, 9, 1)]), ([], [(100, 20, 64, 9, 1), (120, 20, 64, 9, 1), (140, 24, 64, 9, 1)]),
             ([], [(100, 20, 64, 9, 1), (120, 20, 64, 9, 1), (140, 25, 64, 9, 1)]), ([(150, 164, 1)], [(100, 32, 64, 9, 0)]),
             ([(150, 165, 1)], [(100, 32, 64, 9, 0)]), ([(131, 140, 1)], [(100, 32, 64, 9, 0)])]
    assert _answers(tmp_path, cases) == [0, 1, 0, 0, 1, 0, 1, 1]


def test_random_buffers(tmp_path):
    """Plain ranges and matrices of one stride: exact. Matrices of different strides: never missed."""
    rnd, exact, other = random.Random(5), [], []
    for i in range(6000):
        strides = [rnd.randint(4, 24)] * 4 if i % 3 else [rnd.randint(4, 24) for _ in range(4)]
        m = []
        for s in strides[:rnd.randint(0, 4)]:
            m.append((rnd.randint(0, 150), rnd.randint(1, s), s, rnd.randint(1, 6), rnd.randint(0, 1)))
        iv = []
        for _ in range(rnd.randint(0, 3)):
            a = rnd.randint(0, 250)
            iv.append((a, a + rnd.randint(1, 12), rnd.randint(0, 1)))
        (exact if len({e[2] for e in m}) < 2 else other).append((iv, m))
    got, want = _answers(tmp_path, exact), [_overlap(*c) for c in exact]
    assert [c for c, g, w in zip(exact, got, want) if g != w] == [] and 0.2 < sum(want) / len(want) < 0.95
    got, want = _answers(tmp_path, other), [_overlap(*c) for c in other]
    assert all(g or not w for g, w in zip(got, want))
