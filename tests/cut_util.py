"""The library's choice of a cut for a product with a projection in 8 bits (csrc/projection_cut.h), asked without a GPU."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

PROGRAM = r"""
#include "projection_cut.h"
#include <cstdio>
int main()
{
    long long rows, width, depth;
    int sms, fit[9];
    while (scanf("%lld %lld %lld %d", &rows, &width, &depth, &sms) == 4) {
        for (int n = 1; n <= 8; ++n)
            if (scanf("%d", fit + n) != 1) return 1;
        cs::ProjectionCut c = {};
        const int rc = cs::choose_cut(rows, width, (int)((depth + cs::PJ_GROUP - 1) / cs::PJ_GROUP), sms, [&](const cs::ProjectionCut &s, int n, int &count) {
            if (n < 1 || n > 8 || s.tile < 16) return 7;
            count = fit[n];
            return 0;
        }, c);
        printf("%d %d %d %d %lld\n", rc, (int)c.pair, c.tile, c.parts, c.clusters);
    }
    return 0;
}
"""

# multiprocessors, and clusters of 1 .. 8 CTAs with an SM each that a device holds at once: as one answered, one whose SMs lie otherwise, a smaller one
DEVICES = [(148, (148, 74, 45, 33, 26, 22, 15, 15)), (148, (148, 74, 48, 36, 28, 24, 20, 18)), (132, (132, 66, 40, 30, 24, 20, 16, 14))]


def cuts(folder, questions, device=DEVICES[0]):
    """For each (rows, width, depth) the chosen (pair, rows of a tile, parts, clusters)."""
    src, exe = os.path.join(str(folder), "cut.cpp"), os.path.join(str(folder), "cut")
    if not os.path.exists(exe):
        open(src, "w").write(PROGRAM)
        subprocess.run(["g++", "-std=c++17", "-Wall", "-Werror", "-I", os.path.join(ROOT, "paper_1911_02497_b200", "csrc"), "-o", exe, src], check=True)
    text = "\n".join(" ".join(str(v) for v in (*q, device[0], *device[1])) for q in questions)
    lines = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout.split("\n")[:len(questions)]
    answers = [tuple(int(v) for v in line.split()) for line in lines]
    assert len(answers) == len(questions) and all(a[0] == 0 for a in answers)
    return [(bool(a[1]), *a[2:]) for a in answers]
