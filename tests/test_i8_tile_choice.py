"""Which tiles the 8-bit products of the GPU tests reach, whole and in parts of K (CPU: the library's
choices are compiled into a small program)."""
import os
import subprocess

import pytest

from paper_2607_23159_amd import build

from test_gemm_tile_choice import TILES as NAMES
from test_gpu_i8 import MM, PARTS, TILES

PROGRAM = """
#include <cstdio>
#include "gemm_tile.hpp"
int main() {
  long m, n, k;
  while (std::scanf("%ld %ld %ld", &m, &n, &k) == 3) {
    const auto s = cs::split_k_i8(m, n, k);
    std::printf("%d %d %d %d\\n", (int)cs::choose_tile_i8(m, n, k, false), s.parts, s.per, (int)s.tile);
  }
}
"""


@pytest.fixture(scope="module")
def choose(tmp_path_factory):
    d = tmp_path_factory.mktemp("choice")
    src, exe = str(d / "choice.cpp"), str(d / "choice")
    with open(src, "w") as f:
        f.write(PROGRAM)
    subprocess.run(["g++", "-std=c++17", "-O1", "-w", "-I", build.CSRC, src, "-o", exe], check=True)

    def run(shapes):
        text = "".join("%d %d %d\n" % s for s in shapes)
        out = subprocess.run([exe], input=text, capture_output=True, text=True, check=True).stdout
        return [tuple(map(int, line.split())) for line in out.splitlines()]
    return run


def test_every_tile_is_compared(choose):
    assert list(TILES) == NAMES
    for name, (tile, parts, _, _) in zip(NAMES, choose(TILES.values())):
        assert NAMES[tile] == name and parts == 1
    for name, (_, parts, _, tile) in zip(PARTS, choose(PARTS.values())):
        assert NAMES[tile] == name and parts > 1


def test_parts_cover_k_once(choose):
    shapes = [(m, n, k) for m in (17, 40, 64, 130, 500, 1024) for n in (16, 300, 1536, 5120) for k in range(6000, 65537, 1777)]
    found = choose(shapes + list(MM))
    for (m, n, k), (_, parts, per, tile) in zip(shapes + list(MM), found):
        slices = (k + 127) // 128
        assert parts * per >= slices > (parts - 1) * per and 1 <= parts <= 6
        assert parts == 1 or tile >= NAMES.index("RING_64x128")
    assert sum(f[1] > 1 for f in found) > 50
