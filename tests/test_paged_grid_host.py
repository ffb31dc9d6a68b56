"""How a launch of the paged cache's row kernels shares the reads it brings ahead, on the CPU: for every grid the host
may launch (its size follows n_rows, an upper bound of the caller's), the threads that take part are numbered from 0, each
once, and steps by their count never leave 32 bits."""
import os
import subprocess

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))

SOURCE = r"""
#include "ra_paged.h"
#include <stdio.h>

// prints grid_x grid_y x y threads thread -> i n for each line of arguments read
int main()
{
    unsigned gx, gy, x, y;
    int threads, thread;
    while (scanf("%u %u %u %u %d %d", &gx, &gy, &x, &y, &threads, &thread) == 6) {
        const ra::PrefetchShare s = ra::prefetch_share(gx, gy, x, y, threads, thread);
        printf("%d %d\n", s.i, s.n);
    }
    return 0;
}
"""


def shares(tmp_path, asked):
    src, exe = tmp_path / "share.cpp", tmp_path / "share"
    src.write_text(SOURCE)
    nvcc = subprocess.check_output(["bash", "-c", "command -v nvcc || echo /usr/local/cuda/bin/nvcc"], text=True).strip()
    cuda = os.path.join(os.path.dirname(os.path.dirname(os.path.realpath(nvcc))), "include")
    subprocess.check_call(["g++", "-std=c++17", "-I" + os.path.join(ROOT, "include"), "-I" + os.path.join(ROOT, "paper_2609_03430_gb300", "csrc"),
                           "-I" + cuda, str(src), "-o", str(exe)])
    out = subprocess.run([str(exe)], input="".join("%d %d %d %d %d %d\n" % a for a in asked), text=True, capture_output=True, check=True).stdout
    return [tuple(map(int, line.split())) for line in out.splitlines()]


def grids():
    """Grids as the host sizes them: the pages that n_rows rows may touch by the groups of heads."""
    for n_rows in (1, 2, 37, 4096, 10 ** 6, 2 ** 27, 2 ** 28 - 32, 2 ** 31 - 1):
        for shift in (4, 7):
            for batch in (1, 512):
                pages = min((n_rows >> shift) + 2 * batch, n_rows)
                for heads in (1, 2, 65535 // 2):
                    yield pages, heads


def test_no_grid_leaves_32_bits(tmp_path):
    asked = []
    for gx, gy in grids():
        for threads in (32, 160, 256):
            for x, y in ((0, 0), (gx - 1, 0), (0, gy - 1), (gx - 1, gy - 1)):
                asked += [(gx, gy, x, y, threads, 0), (gx, gy, x, y, threads, threads - 1)]
    lines = 512 * 65535 * 2  # the most that one call's threads step over: a line of a head of every sequence's row
    for (gx, gy, x, y, threads, thread), (i, n) in zip(asked, shares(tmp_path, asked)):
        at = (y * gx + x) * threads + thread
        assert n >= 1 and n <= gx * gy * threads and lines + n < 2 ** 31
        assert i == (at if at < n else -1), (gx, gy, x, y, threads, thread, i, n)


def test_small_launches_take_part_whole(tmp_path):
    """Every thread of a small grid has a number of its own."""
    asked = [(7, 3, x, y, 64, t) for y in range(3) for x in range(7) for t in range(64)]
    got = shares(tmp_path, asked)
    assert sorted(i for i, _ in got) == list(range(7 * 3 * 64)) and {n for _, n in got} == {7 * 3 * 64}
