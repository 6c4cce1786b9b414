"""Registers and LDS of linear attention, the quantizing norm and the microscaled products, from the compiler's
resource-usage remarks with the library's own flags: no scratch memory and no VGPR spills, within the 160 KB of LDS."""
import os
import shutil

import pytest

from paper_2608_21952_amd import build as libbuild
from test_build_resources import _resources

pytestmark = pytest.mark.skipif(shutil.which(libbuild.hipcc()) is None and
                                not os.path.exists(libbuild.hipcc()), reason="hipcc missing")


@pytest.mark.parametrize("src", ["linear_attention.hip", "norm_quantize.hip", "quantize_mx.hip", "linear_mx.hip"])
def test_no_register_spills(src):
    res = _resources(src)
    assert res, f"no kernels found in {src}"
    for name, r in res.items():
        assert r.get("VGPRs Spill", 0) == 0, f"{name}: {r}"
        assert r["ScratchSize"] == 0, f"{name}: {r}"
        assert r["LDS Size"] <= 160 * 1024, f"{name}: {r}"
