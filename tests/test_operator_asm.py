"""The windowed attention's copies into LDS take their destination from M0, which
the compiler does not preserve across inline assembly: every instruction of the
kernels that names M0 is a copy's own write of it.  Their sums run in registers:
the loops of none of them spill."""
import os
import re
import subprocess

import pytest

from paper_2506_05345_amd import build
from test_kernel_asm import test_m0_is_only_the_lds_copy_destination as _m0_check


def test_m0_is_only_the_lds_copy_destination_in_windowed_attention(tmp_path):
    _m0_check(tmp_path, "dms_window.hip")


@pytest.mark.parametrize("src", ["dms_window.hip", "dms_rope.hip", "dms_pages.hip"])
def test_matrix_products_run_without_scratch_and_packed_float_math(tmp_path, src):
    out = str(tmp_path / "k.s")
    cmd = [build.hipcc(), *build.COMMON, *build.GPU_FLAGS, *build.PER_SOURCE.get(src, []), "-I", build.CSRC, "-S",
           "--cuda-device-only", os.path.join(build.CSRC, src), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True)
    text = open(out).read()
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    # between labels: no block with a matrix product touches scratch memory
    for block in re.split(r"\n(?:\.LBB\S+:|; %bb\S+)", text):
        if "v_mfma" in block:
            assert "scratch_" not in block
