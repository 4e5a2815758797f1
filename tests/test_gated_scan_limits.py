"""The longest calls that the gated recurrence takes, the first that it refuses, and the launches that a long one goes out in."""
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
    for (uint64_t all : {1ull, 300ull, (1ull << 24) - 9, (1ull << 24) - 8, (1ull << 24) - 7, 1ull << 24, 257ull * 65535, (1ull << 25) - 16, (1ull << 31) - 1}) {
        uint64_t sum = 0;
        uint32_t first = 0, launches = 0;
        for (uint32_t now; first < (uint32_t)all; first += now, ++launches) {
            now = workgroups_from(first, (uint32_t)all);
            if (!now || now * 256ull >= 1ull << 32 || first % 8) return std::printf("%u workgroups from %u of %llu\n", now, first, (unsigned long long)all), 1;
            sum += now;
        }
        if (sum != all || launches != (all + (1 << 24) - 9) / ((1 << 24) - 8)) return std::printf("%llu of %llu\n", (unsigned long long)sum, (unsigned long long)all), 1;
    }
    return 0;
}
"""


def test_launches_of_a_long_call(tmp_path):
    """Each carries less than 2^32 threads, and together they have every workgroup once."""
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "walk.cpp", os.path.join(tmp_path, "walk")
    src.write_text(WALK)
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-I", CSRC, str(src), "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
