"""LDS of the operators' kernels (no GPU: compiles for gfx950).  The opt-in for more than 64 KB is made for the size that
a launch names, so a kernel that may need it declares no LDS of a fixed size beside that."""
import os
import shutil

import pytest

from paper_1508_06904_amd import build
from tests.test_kernel_resources import _report


@pytest.mark.parametrize("src,kernel", [("linear_tile.hip", "linear_tile_kernel"), ("matmul_tokens.hip", "matmul_tile_kernel")])
def test_kernels_over_64_kb_have_all_of_it_in_the_launch(src, kernel):
    if not os.path.exists(build.HIPCC) and shutil.which(build.HIPCC) is None:
        pytest.skip("hipcc not available")
    ks = {n: r for n, r in _report(src).items() if kernel in n}
    assert ks
    for name, r in ks.items():
        assert r["LDS Size"] == 0, (name, r)
