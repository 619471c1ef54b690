"""How near the windowed attention's gradients come to float64 where dS = P (dP - D)
cancels: rows of few keys and rows whose weights lie on one key.  The row term D
has to be as exact as float32 sums make it; formed from the bf16 `out` it is off
by 2^-8 of |dO||out|, several times such a row's whole gradient."""
import numpy as np
import pytest

import dms_synth as sy
import oracle
from test_window_attention import _gpu, _inputs

pytestmark = pytest.mark.gpu

CASES = [
    # lens, H, g, d, w, sinks, scale of the queries
    ([500], 1, 2, 128, 256, 4, 8.0), ([130, 700], 2, 1, 64, 256, 0, 4.0), ([400], 1, 3, 128, 130, 2, 2.0),
    ([300, 50, 1, 2], 1, 1, 128, 1000, 0, 8.0), ([600], 1, 5, 64, 128, 64, 8.0), ([90], 2, 2, 128, 16, 2, 8.0),
]


def _grads(x, lens, H, g, d, w, sinks):
    """Float64 gradients of the packed sequences and their slacks with D summed in float32."""
    f = {n: sy.bf16_bits_to_f32_np(b).astype(np.float64) for n, b in x.items()}
    parts, a = [], 0
    for n in lens:
        q, k, v, do = (f[m][a:a + n] for m in ("q", "k", "v", "dout"))
        parts.append(oracle.window_attention_grads(q, k, v, do, w, sinks, g, summed_d=True))
        a += n
    return tuple({m: np.concatenate([p[i][m] for p in parts]) for m in ("dq", "dk", "dv")} for i in (0, 1))


@pytest.mark.parametrize("lens,H,g,d,w,sinks,q_scale", CASES)
def test_every_element_within_the_roundings_of_its_products(lens, H, g, d, w, sinks, q_scale):
    x = _inputs(sum(lens), H, g, d, 31, q_scale)
    ref, slack = _grads(x, lens, H, g, d, w, sinks)
    got = _gpu(x, lens, H, g, d, w, sinks)
    worst = {m: float((np.abs(got[m] - ref[m]) / slack[m]).max()) for m in ref}
    print(worst)
    assert all(o <= 1.0 for o in worst.values()), worst


@pytest.mark.parametrize("lens,H,g,d,w,sinks,q_scale", CASES)
def test_whole_gradients_are_off_by_two_roundings(lens, H, g, d, w, sinks, q_scale):
    """dS (P for dV) and the result are rounded to bf16, each by at most 2^-8 of the value and evenly spread, that
    is 2^-8 / sqrt(3) at most in the mean square; two of them together 2^-8 sqrt(2 / 3) = 0.0032, and float32 sums
    below a tenth of that in quadrature: 2^-8 in all."""
    x = _inputs(sum(lens), H, g, d, 32, q_scale)
    ref, _ = _grads(x, lens, H, g, d, w, sinks)
    got = _gpu(x, lens, H, g, d, w, sinks)
    off = {m: float(np.linalg.norm(got[m] - ref[m]) / np.linalg.norm(ref[m])) for m in ref}
    print(off)
    assert all(o <= 2.0 ** -8 for o in off.values()), off


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("w,sinks", [(256, 4), (1000, 0), (100, 40)])
def test_a_short_sequence_beside_longer_ones_gives_the_same_bits(d, w, sinks):
    lens, H, g = [100, 300, 20], 2, 3
    x = _inputs(sum(lens), H, g, d, 33, 4.0)
    whole = _gpu(x, lens, H, g, d, w, sinks)
    for a, b in ((0, 100), (400, 420)):
        one = _gpu({n: y[a:b] for n, y in x.items()}, [b - a], H, g, d, w, sinks)
        for n in ("out", "dq"):
            assert np.array_equal(whole[n][a:b], one[n]), (n, a)
        assert np.array_equal(whole["lse"][:, a:b], one["lse"]), a
