"""Which tile and chunk a workgroup of the gated recurrence works on, walked on the host through the header that the kernels are built from: alone on its
workspace a launch hands every chunk of
every tile out once, in order; beside another call on the same workspace it works on no chunk beyond the sequence."""
import os
import shutil
import subprocess

import pytest

CSRC = os.path.join(os.path.dirname(os.path.dirname(os.path.abspath(__file__))), "paper_2411_19460_amd", "csrc")
WALK = r"""
#include <cstdio>
#include <cstdlib>
#include <random>
#include <vector>
#include "chunk_places.h"
using namespace ssdk;

static void fail(const char* what, long a, long b, long c) {
    std::printf("%s: %ld %ld %ld\n", what, a, b, c);
    std::exit(1);
}

struct Launch {
    uint32_t side, chunks, next = 0;            // next: workgroups start in the order of their numbers
    long length, step;                          // tokens of a sequence and of a chunk
    bool left() const { return next < side * chunks; }
    uint32_t tile() { return tile_of(next++, side); }
    // the chunk's first token and its rows, as both directions work them out
    void check(uint32_t drawn) const {
        const long front = (long)drawn * step, back = (long)(chunks - 1 - (long)drawn) * step;
        if (front < 0 || front >= length || back < 0 || back >= length) fail("a chunk beyond the sequence", drawn, chunks, length);
    }
};

int main() {
    std::mt19937 rng(1);
    auto upto = [&](uint32_t n) { return (uint32_t)(rng() % n); };
    for (uint32_t side = 1; side <= 90; ++side)
        for (uint32_t chunks = 2; chunks <= 40; chunks += 1 + chunks / 8) {
            Launch a{side, chunks, 0, (long)chunks * 64 - 63, 64};
            std::vector<uint32_t> counter(side, 0);
            while (a.left()) {
                const uint32_t tile = a.tile();
                if (tile >= side) fail("tile", tile, side, chunks);
                const uint32_t drawn = counter[tile]++;
                if (!chunk_there(drawn, chunks)) fail("alone, a chunk is left out", drawn, chunks, side);
                a.check(drawn);
            }
            for (uint32_t n : counter)
                if (n != chunks) fail("alone, chunks of a tile", n, chunks, side);
        }
    long beyond = 0;
    for (int trial = 0; trial < 4000; ++trial) {
        // two calls, of other lengths and widths mostly; the second clears the counters when the first has begun, or lays other words there
        Launch call[2] = {{1 + upto(20), 2 + upto(30), 0, 0, 64}, {1 + upto(20), 2 + upto(30), 0, 0, trial & 1 ? 64 : 128}};
        if (trial % 3) call[1].side = call[0].side;
        for (Launch& c : call) c.length = (long)c.chunks * c.step - upto((uint32_t)c.step);
        std::vector<uint32_t> counter(20, 0);
        const uint32_t begun = upto(call[0].side * call[0].chunks + 1);
        bool clear = false;
        while (call[0].left() || call[1].left()) {
            if (!clear && call[0].next >= begun) {
                clear = true;
                for (uint32_t k = 0; k < 20; ++k)
                    if (k < call[1].side) counter[k] = 0;
                    else if (trial & 2) counter[k] = rng();
            }
            Launch& c = call[!call[0].left() || (clear && call[1].left() && upto(2))];
            if (!clear && &c == &call[1]) continue;
            const uint32_t drawn = counter[c.tile()]++;
            if (chunk_there(drawn, c.chunks)) c.check(drawn);
            else ++beyond;
        }
    }
    if (!beyond) fail("no call drew a number beyond its chunks", 0, 0, 0);
    std::printf("%ld\n", beyond);
    return 0;
}
"""


def test_no_chunk_beyond_the_sequence_is_worked_on(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    src, exe = tmp_path / "walk.cpp", tmp_path / "walk"
    src.write_text(WALK)
    subprocess.run([cxx, "-std=c++17", "-O2", "-Wall", "-I", CSRC, str(src), "-o", str(exe)], check=True)
    r = subprocess.run([str(exe)], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout
    assert int(r.stdout) > 0
