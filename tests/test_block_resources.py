"""Registers and LDS of the kernels around the SSD layer, from the compiler's resource-usage remarks with the
library's own flags: no scratch memory and no VGPR spills; the tiles of the larger products within the
160 KB of LDS, the compile-time forms of the selective scan within two waves per SIMD (256 VGPRs)."""
import os
import shutil

import pytest

from paper_2608_21952_amd import build as libbuild
from test_build_resources import _resources

pytestmark = pytest.mark.skipif(shutil.which(libbuild.hipcc()) is None and
                                not os.path.exists(libbuild.hipcc()), reason="hipcc missing")


@pytest.mark.parametrize("src", ["conv.hip", "norm.hip", "linear.hip", "selective_scan.hip",
                                 "selective_scan_fast.hip"])
def test_no_register_spills(src):
    res = _resources(src)
    assert res, f"no kernels found in {src}"
    for name, r in res.items():
        assert r.get("VGPRs Spill", 0) == 0, f"{name}: {r}"
        assert r["ScratchSize"] == 0, f"{name}: {r}"
        assert r["LDS Size"] <= 160 * 1024, f"{name}: {r}"
        if src == "selective_scan_fast.hip":
            assert r["VGPRs"] + r.get("AGPRs", 0) <= 256, f"{name}: {r}"
