"""Limits of the rotary and windowed entry points at their border values: sizes
and scales past them are refused before any HIP call (no GPU needed)."""
import ctypes

import pytest

from paper_2506_05345_amd import dms

B = ctypes.byref
SOME = ctypes.c_void_p(4096)           # an aligned address that no call may read


@pytest.mark.parametrize("tokens", [(1 << 26) - 3, (1 << 26) - 2, (1 << 26) - 1, 1 << 26])
def test_rope_grids_stay_below_two_to_the_32_threads(tokens):
    """A wave per token, four to a workgroup of 256: 2^26 - 3 tokens already round up to 2^32 threads."""
    cfg = dms.make_rope_config(1, 1, 64, 64, [32])
    assert -(-tokens // 4) * 256 >= 1 << 32
    assert dms.lib().dms_rope_fwd(B(cfg), tokens, SOME, 64, None, 64, SOME, SOME, SOME, None, None, None,
                                  None) == dms.DMS_ERR_UNSUPPORTED
    assert dms.lib().dms_rope_bwd(B(cfg), tokens, SOME, None, SOME, SOME, None, SOME, 64, None, 64,
                                  None) == dms.DMS_ERR_UNSUPPORTED
