"""What the compiler made of the tree attention and the sampling: every instruction
that names M0 is a copy's own write of its destination in LDS, no packed float
arithmetic, and no kernel touches scratch memory."""
import os
import re
import subprocess

import pytest

from paper_2506_05345_amd import build
from test_kernel_asm import test_m0_is_only_the_lds_copy_destination as _m0_check


def test_m0_is_only_the_lds_copy_destination_in_tree_attention(tmp_path):
    _m0_check(tmp_path, "dms_tree.hip")


@pytest.mark.parametrize("src", ["dms_tree.hip", "dms_sample.hip"])
def test_no_scratch_and_no_packed_float_math(tmp_path, src):
    out = str(tmp_path / "k.s")
    cmd = [build.hipcc(), *build.COMMON, *build.GPU_FLAGS, *build.PER_SOURCE.get(src, []), "-I", build.CSRC, "-S",
           "--cuda-device-only", os.path.join(build.CSRC, src), "-o", out]
    subprocess.run(cmd, check=True, capture_output=True)
    text = open(out).read()
    assert not re.search(r"\bv_pk_(add|mul|fma)_f32\b", text)
    sizes = re.findall(r"\.amdhsa_private_segment_fixed_size (\d+)", text)
    assert sizes and all(int(x) == 0 for x in sizes)
    assert "scratch_" not in re.sub(r"^\s*[;.].*$", "", text, flags=re.M)
