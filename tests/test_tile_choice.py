"""The sizes of the tests of the products' tiles do reach each tile: the rule itself, compiled for the host, is asked."""
import os
import shutil
import subprocess

import pytest

from paper_1508_06904_amd import build

# tile (index in the rule's table) -> products M, N, K of more than one step of 128 channels for each group of
# waves, of which no tile divides a side; more than 32 tokens, so that the tiles run them
SHAPES = {
    0: [(2100, 4001, 300), (3900, 2705, 400)],                       # 256 x 256
    1: [(1500, 2701, 300), (2111, 2700, 400)],                       # 128 x 128
    2: [(1100, 1030, 390), (1777, 1003, 672)],                       # 64 x 64
    3: [(300, 301, 4100), (130, 511, 1680)],                         # 64 x 64, four groups of waves
}


def test_each_tile_is_reached(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    src = tmp_path / "ask.cpp"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "tile_choice.h"\n'
                   'int main(int n, char** v) { for (int i = 1; i + 2 < n; i += 3)\n'
                   '  printf("%d\\n", dss::pick_tile(atoll(v[i]), atoll(v[i + 1]), (atoi(v[i + 2]) + 15) / 16 * 16)); }\n')
    subprocess.run([cxx, "-std=c++17", "-I", build.CSRC, str(src), "-o", str(tmp_path / "ask")], check=True)
    for planar in (False, True):
        asked = [(t, (N, M, K) if planar else (M, N, K)) for t in SHAPES for M, N, K in SHAPES[t]]
        r = subprocess.run([str(tmp_path / "ask")] + [str(v) for _, s in asked for v in s], check=True, capture_output=True,
                           text=True)
        assert [int(v) for v in r.stdout.split()] == [t for t, _ in asked], (planar, asked, r.stdout)
    for t, shapes in SHAPES.items():
        side, groups = (256, 128, 64, 64)[t], (1, 1, 1, 4)[t]
        for M, N, K in shapes:
            assert M > 32 and M % side and N % side and K > 2 * 128 * groups
    assert any(K % 16 == 0 for t in SHAPES for _, _, K in SHAPES[t]) and any(K % 16 for t in SHAPES for _, _, K in SHAPES[t])
