"""The longest calls that the gated recurrence takes, the first that it refuses, and the grid of a long one."""
import ctypes
import os
import shutil
import subprocess

import pytest

import paper_2411_19460_amd as pk
from paper_2411_19460_amd import binding
from test_gated_scan_abi import NULL, SHAPE, bwd, fwd, shape, step
from test_gated_scan_places import CSRC

MOST = 2 ** 31 - 1


@pytest.mark.parametrize("batch,channels", [(1, 64), (65535, 1), (65535, 65), (64, 5120), (3, 2560), (1, 1 << 20), (7, 100)])
@pytest.mark.parametrize("back", [0, 1])
def test_the_longest_call(batch, channels, back):
    length = min(MOST // (batch * -(-channels // 64)) * 64, 1 << 32)
    call = bwd if back else fwd
    good, long = (shape(batch=batch, channels=channels, seqlen=n) for n in (length, length + 1))
    scratch = [binding.lib().ssd_gated_scan_workspace_bytes(ctypes.byref(s), back) for s in (good, long)]
    assert scratch[0] > 0 and call(good, x=None) == NULL and step(good, x=None) == NULL        # the shape is taken, and a pointer missed
    assert scratch[1] == 0 and call(long) == SHAPE and step(long) == SHAPE
    if back:
        assert call(long, flags=pk.SSD_FLAG_ACCUM_PARAM) == SHAPE


WALK = r"""
#include <cstdio>
#include <initializer_list>
#include "chunk_places.h"
using namespace ssdk;
int main() {
    for (uint64_t all : {1ull, 300ull, (1ull << 24) - 2, (1ull << 24) - 1, 1ull << 24, (1ull << 24) + 1, 257ull * 65535, (1ull << 25) - 16, (1ull << 31) - 1}) {
        const Grid g = grid_of((uint32_t)all);
        const uint64_t there = (uint64_t)g.x * g.y;
        bool good = there >= all && there - all < ROW && g.x * 256ull < 1ull << 32 && g.y < 65536 && there <= 1ull << 31;
        good = good && (g.y > 1 || there == all);
        // rows follow one another, and whole turns of the eight XCDs make a row
        for (uint32_t y = 1; y < g.y; ++y) good = good && number_of(0, y) == number_of(g.x - 1, y - 1) + 1 && number_of(0, y) % 8 == 0;
        good = good && number_of(0, 0) == 0 && number_of(g.x - 1, g.y - 1) == there - 1;
        if (!good) return std::printf("%u x %u workgroups for %llu\n", g.x, g.y, (unsigned long long)all), 1;
    }
    return 0;
}
"""


def test_the_grid_of_a_long_call(tmp_path):
    """Every workgroup once, in order, less than 2^32 threads along a dimension, and less than a row to spare."""
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "walk.cpp", os.path.join(tmp_path, "walk")
    src.write_text(WALK)
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-I", CSRC, str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
