"""What the adapters' narrow products ask for, walked on the host through the same header that the kernel is built from: no row of a factor
stored as [K][rank] beyond its last, whatever K, the ranks of a workgroup and its group of steps; and every row that exists is kept once."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_19460_amd", "csrc")
WALK = r"""
#include <cstdio>
#include <vector>
#include "low_steps.h"
using namespace ssdk;
int main() {
    const int rts[] = {1, 2, 4};
    long asked = 0;
    for (int rt : rts)
        for (int nr = 8; nr <= 16 * rt; nr += 8)
            for (int mt = 1; mt <= 2; ++mt)
                for (int K = 8; K <= 4352; K += K < 1100 ? 8 : 24) {
                    const int group = low_group(rt, mt), per_row = nr / 8;
                    std::vector<int> kept(K * per_row);
                    for (int w = 0; w < LWAVES; ++w) {
                        bool whole = true;
                        for (int k0 = LSTEP * w; k0 < K && whole; k0 += low_advance(group)) {
                            whole = low_whole(k0, group, K);
                            for (int s = 0; s < group; ++s)
                                for (int piece = 0; piece < 2 * rt * 64; ++piece) {
                                    const int ks = k0 + LSTEP * LWAVES * s, row = low_piece_row(piece, per_row);
                                    const int at = low_row_asked(ks, low_piece_asked(row), whole, K);
                                    ++asked;
                                    if (at < 0 || at >= K) return std::printf("rt %d, %d ranks, mt %d, K %d: row %d asked for\n", rt, nr, mt, K, at), 1;
                                    if (low_piece_there(row) && ks + row < K) {
                                        if (at != ks + row) return std::printf("rt %d, %d ranks, mt %d, K %d: row %d for %d\n", rt, nr, mt, K, at, ks + row), 1;
                                        ++kept[at * per_row + piece % per_row];
                                    }
                                }
                        }
                    }
                    for (int n : kept)
                        if (n != 1) return std::printf("rt %d, %d ranks, mt %d, K %d: a piece kept %d times\n", rt, nr, mt, K, n), 1;
                }
    std::printf("%ld\n", asked);
    return 0;
}
"""


def test_no_row_beyond_the_factor_is_asked_for(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(WALK)
    subprocess.run([cxx, "-std=c++17", "-O2", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout) > 0
