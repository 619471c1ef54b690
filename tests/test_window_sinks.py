"""The windowed attention with hundreds of sinks, up to every token (full causal
attention), against the float64 oracle, and the forward's workspace."""
import numpy as np
import pytest

from test_window_attention import _check, _dev, _gpu, _inputs

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("lens, H, g, d, w, sinks", [
    ([1500], 1, 1, 64, 40, 300), ([900, 0, 300], 2, 1, 128, 30, 513), ([700], 1, 2, 128, 1, 700), ([1200], 1, 1, 64, 5, 10**9),
    # enough blocks to fill the chip
    ([1300], 24, 1, 64, 20, 600), ([1100, 150], 26, 1, 64, 100, 1100),
])
def test_many_sinks(lens, H, g, d, w, sinks):
    x = _inputs(sum(lens), H, g, d, 51, 2.0)
    _check(x, lens, H, g, d, w, min(sinks, max(lens)), _gpu(x, lens, H, g, d, w, sinks))


def test_the_forward_needs_no_workspace_of_the_backward_s_size():
    import torch
    from paper_2506_05345_amd import dms
    T, H, g, d, w, sinks = 300, 2, 3, 128, 40, 4
    x = {n: _dev(b) for n, b in _inputs(T, H, g, d, 52).items()}
    cfg = dms.make_window_config(1, T, T, H, g, d, w, sinks)
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    got = []
    for n in (dms.dms_window_workspace(cfg), 256):
        ws = torch.full((n,), 0x5A, dtype=torch.uint8, device="cuda")
        out, lse = torch.empty_like(x["q"]), torch.empty((H * g, T), device="cuda")
        dms.dms_window_attention_fwd(cfg, cu, x["q"], x["k"], x["v"], out, lse, ws)
        torch.cuda.synchronize()
        assert (ws == 0x5A).all()
        got.append((out, lse))
    assert all(torch.equal(a, b) for a, b in zip(*got))
    grads = [torch.empty_like(x[n]) for n in ("q", "k", "v")]
    with pytest.raises(dms.DmsError, match="workspace"):
        dms.dms_window_attention_bwd(cfg, cu, x["q"], x["k"], x["v"], *got[0], x["dout"], *grads, ws)
