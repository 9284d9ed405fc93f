"""Register and scratch budgets of the gradient-clipping and 8-bit token kernels (no GPU: compiles for
gfx950): no scratch, no spilled vector registers; the tiles' kernels keep two waves per SIMD."""
import concurrent.futures as cf
import os
import shutil

import pytest

from paper_1508_06904_amd import build
from tests.test_kernel_resources import _report

SOURCES = ["grad_clip.hip", "tokens.hip", "matmul_tokens.hip", "matmul_few.hip", "linear_tile.hip"]


@pytest.fixture(scope="module")
def reports():
    if not os.path.exists(build.HIPCC) and shutil.which(build.HIPCC) is None:
        pytest.skip("hipcc not available")
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        return dict(zip(SOURCES, ex.map(_report, SOURCES)))


@pytest.mark.parametrize("src", SOURCES)
def test_no_scratch_and_no_spills(reports, src):
    ks = reports[src]
    assert ks, "no kernels reported for %s" % src
    for name, r in ks.items():
        assert r.get("ScratchSize", 0) == 0, (name, r)
        assert r.get("VGPRs Spill", 0) == 0, (name, r)


def test_tiles_keep_two_waves_per_simd(reports):
    tiles = {n: r for n, r in reports["matmul_tokens.hip"].items() if "matmul_tile_kernel" in n}
    assert len(tiles) == 16                # four tiles, two output types, rows and maps
    for name, r in tiles.items():
        assert r["Occupancy"] >= 2, (name, r)
