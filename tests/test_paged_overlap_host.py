"""Rows read back must not be written over each other: which strides let two rows share an element, on the CPU, against
trying every pair."""
import itertools
import os
import random
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "ra_paged.h"
#include <stdio.h>

int main()
{
    long long row, head;
    int n_rows, heads, D;
    while (scanf("%lld %lld %d %d %d", &row, &head, &n_rows, &heads, &D) == 5)
        printf("%d\n", (int)ra::rows_overlap(row, head, n_rows, heads, D));
    return 0;
}
"""


def overlap(tmp_path, asked):
    src, exe = tmp_path / "overlap.cpp", tmp_path / "overlap"
    src.write_text(SOURCE)
    nvcc = subprocess.check_output(["bash", "-c", "command -v nvcc || echo /usr/local/cuda/bin/nvcc"], text=True).strip()
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    subprocess.check_call(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2609_03430_gb300", "csrc"),
                           "-I" + cuda, str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], input="".join("%d %d %d %d %d\n" % a for a in asked), text=True, capture_output=True, check=True).stdout
    return [line == "1" for line in out.split()]


def by_trying(row, head, n_rows, heads, D):
    at = sorted(r * row + h * head for r in range(n_rows) for h in range(heads))
    return any(b - a < D for a, b in zip(at, at[1:]))


def test_against_every_pair(tmp_path):
    rng = random.Random(3)
    asked = [(8 * r, 8 * h, n, k, 64) for r, h, n, k in itertools.product((0, 7, 8, 9, 16, 24, 64), (0, 7, 8, 12, 16, 40, 72), (1, 2, 3, 9), (1, 2, 8))]
    asked += [(8 * rng.randint(0, 90), 8 * rng.randint(0, 90), rng.randint(1, 30), rng.randint(1, 12), rng.choice([64, 128])) for _ in range(4000)]
    got = overlap(tmp_path, asked)
    for a, g in zip(asked, got):
        assert g == by_trying(*a), a
    assert 200 < sum(got) < len(got) - 200


def test_the_usual_layouts(tmp_path):
    """[rows][heads][D], [heads][rows][D], slices of fused projections; and both strides D, which is none."""
    D, n = 128, 2 ** 31 - 1
    fine = [(8 * D, D, n, 8, D), (D, n * D, n, 8, D), (48 * D, D, n, 8, D), (48 * D, 6 * D, n, 8, D), (8 * D, D, 1, 8, D), (0, D, 1, 8, D),
            (D, 0, n, 1, D), (2 ** 62, 2 ** 40, 2, 65535, D), (3 * D, 2 * D, 2, 2, D)]
    bad = [(D, D, 2, 2, D), (8 * D, D, 2, 9, D), (D, 8 * D, 9, 2, D), (2 ** 62, 2 ** 61, 3, 3, D), (3 * D, 2 * D, 3, 4, D)]
    assert overlap(tmp_path, fine + bad) == [False] * len(fine) + [True] * len(bad)
