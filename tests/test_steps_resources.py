"""The kernels of the verification and of the books keep no registers in scratch memory."""
import os

import pytest

from paper_2503_08640_amd import build
from test_kernel_resources import READELF, kernels


@pytest.mark.skipif(not (os.path.exists(READELF) and os.path.exists(build.LIB_PATH)), reason="needs the built library and llvm-readelf")
def test_no_scratch(tmp_path):
    found = [x for x in kernels(tmp_path) if "verify_" in x[0] or "pages_" in x[0]]
    assert sum("verify_draw_kernel" in name for name, _ in found) == 6 and sum("pages_" in name for name, _ in found) >= 8
    assert not {name for name, f in found if f[".vgpr_spill_count"] != "0" or f[".private_segment_fixed_size"] != "0"}
