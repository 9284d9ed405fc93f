"""The sizes of the tests of the 4-bit products' tiles do reach each tile: the rule itself, compiled for the host, is asked."""
import shutil
import subprocess

import pytest

from paper_1508_06904_amd import build

# tile (index in the rule's table) -> products M, N, K of more than one step of 256 channels, of which no tile divides a side
SHAPES = {
    0: [(4001, 2100, 600), (2705, 3900, 700)],                       # 256 x 256
    1: [(1500, 2701, 600), (100, 90, 29000)],                        # 128 x 128, also for rows whose scales do not fit LDS
    2: [(300, 301, 4100), (1030, 1100, 770), (17, 4001, 1000)],      # 64 x 64
}


def test_each_tile_is_reached(tmp_path):
    cxx = shutil.which("g++") or shutil.which("c++")
    if cxx is None:
        pytest.skip("no host compiler")
    src = tmp_path / "ask.cpp"
    src.write_text('#include <cstdio>\n#include <cstdlib>\n#include "tile_choice.h"\n'
                   'int main(int n, char** v) { for (int i = 1; i + 2 < n; i += 3)\n'
                   '  printf("%d\\n", dss::pick_mx4_tile(atoll(v[i]), atoll(v[i + 1]), (atoi(v[i + 2]) + 31) / 32)); }\n')
    subprocess.run([cxx, "-std=c++17", "-I", build.CSRC, str(src), "-o", str(tmp_path / "ask")], check=True)
    for planar in (False, True):
        asked = [(t, (N, M, K) if planar else (M, N, K)) for t in SHAPES for M, N, K in SHAPES[t]]
        r = subprocess.run([str(tmp_path / "ask")] + [str(v) for _, s in asked for v in s], check=True, capture_output=True,
                           text=True)
        assert [int(v) for v in r.stdout.split()] == [t for t, _ in asked], (planar, asked, r.stdout)
    for t, shapes in SHAPES.items():
        side = (256, 128, 64)[t]
        for M, N, K in shapes:
            assert M > 16 and N > 16 and M % side and N % side and K > 256
