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


@pytest.mark.parametrize("scale", [1e-45, 1e-38, 2.0 ** -101])
def test_scales_whose_row_values_leave_float32_are_refused(scale):
    """The key-major gradients start from -lse / scale of each row: at scale 1e-38 the log of a few thousand equal
    weights, about 8, is already past float32, and every weight would be 0."""
    import numpy as np
    with np.errstate(over="ignore"):
        assert np.isinf(np.float32(8.0) / np.float32(1e-38))
    cfg = dms.make_window_config(1, 100, 100, 2, 3, 128, 16, 4, scale)
    assert dms.lib().dms_window_workspace(B(cfg), None) == dms.DMS_ERR_INVALID
    assert dms.lib().dms_window_attention_fwd(B(cfg), *[SOME] * 7, None) == dms.DMS_ERR_INVALID
    assert dms.lib().dms_window_attention_bwd(B(cfg), *[SOME] * 11, None) == dms.DMS_ERR_INVALID
    for fine in (2.0 ** -100, 0.0, -1.0):
        assert dms.dms_window_workspace(dms.make_window_config(1, 100, 100, 2, 3, 128, 16, 4, fine)) > 0


@pytest.mark.parametrize("tokens", [1777, 6000, 16384, 131072])
@pytest.mark.parametrize("H,g,d", [(2, 6, 128), (8, 5, 128), (2, 2, 64)])
def test_window_workspace_grows_with_the_tokens_alone(tokens, H, g, d):
    """Row values of each query head and at most 64 d bytes of dk's and of dv's sums per token and KV head, however
    many tokens are sinks."""
    for sinks in (0, 64, 200, 513, 1024, 4096, tokens // 2, tokens):
        cfg = dms.make_window_config(1, tokens, tokens, H, g, d, 256, sinks)
        rows = 2 * H * g * (tokens + 128) * 4
        assert dms.dms_window_workspace(cfg) <= rows + 2 * 64 * d * H * tokens + 65536, sinks
