"""Register, scratch and LDS budgets of the kernels of 4-bit tokens and of distillation (no GPU: compiles for gfx950): no
scratch, no spilled vector registers; the kernels fed by matrix instructions keep two waves per SIMD, the others that
wait for memory three; a kernel that may need more than 64 KB of LDS, for which the opt-in names the launch's own size,
declares none of a fixed size beside it."""
import concurrent.futures as cf
import os
import shutil

import pytest

from paper_1508_06904_amd import build
from tests.test_kernel_resources import _report

SOURCES = ["mx4.hip", "few_mx4.hip", "matmul_mx4.hip", "linear_mx4.hip", "distill.hip", "distill_map.hip"]
OVER_64_KB = [("few_mx4.hip", "matmul_few_mx4_kernel"), ("matmul_mx4.hip", "matmul_mx4_kernel"),
              ("matmul_mx4.hip", "matmul_mx4_deep_kernel"), ("linear_mx4.hip", "linear_mx4"),
              ("distill_map.hip", "distill_tile_kernel"), ("distill_map.hip", "distill_map_gradient_kernel")]


@pytest.fixture(scope="module")
def reports():
    if not os.path.exists(build.HIPCC) and shutil.which(build.HIPCC) is None:
        pytest.skip("hipcc not available")
    with cf.ThreadPoolExecutor(max_workers=len(SOURCES)) as ex:
        return dict(zip(SOURCES, ex.map(_report, SOURCES)))


@pytest.mark.parametrize("src", SOURCES)
def test_no_scratch_and_no_spills(reports, src):
    assert reports[src]
    for name, r in reports[src].items():
        assert r.get("ScratchSize", 0) == 0, (name, r)
        assert r.get("VGPRs Spill", 0) == 0, (name, r)
        assert r["Occupancy"] >= (2 if src in ("matmul_mx4.hip", "linear_mx4.hip", "few_mx4.hip") else 3), (name, r)


@pytest.mark.parametrize("src,kernel", OVER_64_KB)
def test_kernels_over_64_kb_have_all_of_it_in_the_launch(reports, src, kernel):
    ks = {n: r for n, r in reports[src].items() if kernel in n}
    assert ks
    for name, r in ks.items():
        assert r["LDS Size"] == 0, (name, r)
