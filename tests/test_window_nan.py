"""Infinite and NaN inputs of the windowed attention that leave the scores finite,
or whose first score is -Inf: what they reach is NaN, what they do not reach is as
without them, and a step on them is not hundreds of times as long as another."""
import numpy as np
import pytest

from test_window_attention import _bf16, _gpu, _inputs, _reference

pytestmark = pytest.mark.gpu
NAN = _bf16(np.array([float("nan")]))[0]


def _near(got, ref, slack, name, rows=slice(None)):
    at = (slice(None), rows) if name == "lse" else rows
    assert (np.abs(got[name][at] - ref[name][at]) <= slack[name][at]).all(), name


SHAPES = [(1, 64, 500), (32, 128, 500), (2, 128, 30)]


@pytest.mark.parametrize("H, d, w", SHAPES)
def test_nan_values(H, d, w):
    """Every value NaN: outputs, dQ and dK are NaN; the weights, and with them lse and dV, do not depend on values."""
    T, g, sinks = 1100, 2, 3
    x = _inputs(T, H, g, d, 41)
    ref, slack = _reference(x, [T], H, g, d, w, sinks)
    x["v"][:] = NAN
    got = _gpu(x, [T], H, g, d, w, sinks)
    assert all(np.isnan(got[n]).all() for n in ("out", "dq", "dk"))
    _near(got, ref, slack, "lse")
    _near(got, ref, slack, "dv")


@pytest.mark.parametrize("H, d, w", SHAPES)
def test_nan_output_gradients(H, d, w):
    """Every output gradient NaN (a loss that has diverged)."""
    T, g, sinks = 1100, 2, 3
    x = _inputs(T, H, g, d, 42)
    ref, slack = _reference(x, [T], H, g, d, w, sinks)
    x["dout"][:] = NAN
    got = _gpu(x, [T], H, g, d, w, sinks)
    assert all(np.isnan(got[n]).all() for n in ("dq", "dk", "dv"))
    _near(got, ref, slack, "out")
    _near(got, ref, slack, "lse")


@pytest.mark.parametrize("H, d, w", SHAPES)
def test_nan_in_one_element_of_the_rows(H, d, w):
    """One element of all values, or of all output gradients: the others of out and dV as without it."""
    T, g, sinks = 1100, 2, 3
    x = _inputs(T, H, g, d, 43)
    ref, slack = _reference(x, [T], H, g, d, w, sinks)
    other = np.arange(d) != 7
    for name, reached in (("v", "out"), ("dout", "dv")):
        y = {n: b.copy() for n, b in x.items()}
        y[name][:, :, 7] = NAN
        got = _gpu(y, [T], H, g, d, w, sinks)
        assert np.isnan(got[reached][:, :, 7]).all() and np.isnan(got["dq"]).all() and np.isnan(got["dk"]).all()
        assert (np.abs(got[reached] - ref[reached]) <= slack[reached])[:, :, other].all()


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
@pytest.mark.parametrize("H, d", [(1, 64), (29, 64), (2, 128)])
def test_queries_before_a_sink_in_its_tile(bad, H, d):
    """An Inf or NaN query and output gradient at position 2, or at 20: it reaches the keys up to its own and no
    later one, sinks with far queries among them."""
    T, g, w, sinks = 1100, 1, 20, 40
    x = _inputs(T, H, g, d, 44)
    ref, slack = _reference(x, [T], H, g, d, w, sinks)
    for at in (2, 20):
        y = {n: b.copy() for n, b in x.items()}
        y["q"][at] = y["dout"][at] = _bf16(np.array([bad]))[0]
        got = _gpu(y, [T], H, g, d, w, sinks)
        for n in ("dk", "dv"):
            _near(got, ref, slack, n, slice(at + 1, None))
            assert not np.isfinite(got[n][:at + 1]).any()


@pytest.mark.parametrize("d", [64, 128])
def test_a_first_score_of_minus_infinity(d):
    """Key 0, a sink, scores -Inf against every query (they are positive, it is -Inf): it has no weight, so that rows
    past its window are those of a call without sinks, rows beside a hidden NaN key included."""
    T, H, g, w, at = 400, 1, 2, 16, 300
    x = _inputs(T, H, g, d, 45)
    x["q"] &= 0x7FFF                                     # |q|
    ref, slack = _reference(x, [T], H, g, d, w, 0)
    x["k"][0] = _bf16(np.array([float("-inf")]))[0]
    x["k"][at] = x["v"][at] = NAN
    got = _gpu(x, [T], H, g, d, w, 1)
    rows = np.arange(T) >= w
    rows[at:at + w] = False
    _near(got, ref, slack, "out", rows)
    _near(got, ref, slack, "lse", rows)


@pytest.mark.parametrize("name", ["q", "k", "v", "dout"])
def test_a_step_on_nan_inputs_is_not_much_longer(name):
    """16384 tokens of 8 x 5 heads: at most 20 times the step on finite inputs (walks over every row's keys and
    every key's queries one by one took 200 times as long)."""
    import torch
    from paper_2506_05345_amd import dms
    T, H, g, d, w, sinks = 16384, 8, 5, 128, 256, 4
    cfg = dms.make_window_config(1, T, T, H, g, d, w, sinks)
    cu = torch.tensor([0, T], dtype=torch.int32, device="cuda")
    ws = torch.empty(dms.dms_window_workspace(cfg), dtype=torch.uint8, device="cuda")
    gen = torch.Generator(device="cuda").manual_seed(1)
    t = {n: torch.randn((T, h, d), generator=gen, device="cuda").bfloat16()
         for n, h in (("q", H * g), ("k", H), ("v", H), ("dout", H * g))}
    out, lse = torch.empty_like(t["q"]), torch.empty((H * g, T), device="cuda")
    dq, dk, dv = (torch.empty_like(t[n]) for n in ("q", "k", "v"))

    def step():
        a, b = torch.cuda.Event(enable_timing=True), torch.cuda.Event(enable_timing=True)
        a.record()
        dms.dms_window_attention_fwd(cfg, cu, t["q"], t["k"], t["v"], out, lse, ws)
        dms.dms_window_attention_bwd(cfg, cu, t["q"], t["k"], t["v"], out, lse, t["dout"], dq, dk, dv, ws)
        b.record()
        torch.cuda.synchronize()
        return a.elapsed_time(b)

    usual = sorted(step() for _ in range(7))[3]
    t[name][:] = float("nan")
    assert sorted(step() for _ in range(3))[1] <= 20 * usual
