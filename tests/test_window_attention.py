"""GPU parity of the attention with a sliding window and sinks against the
float64 oracle: every element within the slack that the oracle derives from the
roundings of the products' operands and of the outputs.  NaN-filled outputs and
workspace, rows past the last sequence included."""
import numpy as np
import pytest

import dms_synth as sy
import oracle

pytestmark = pytest.mark.gpu


def _bf16(x):
    return sy.f32_to_bf16_bits_np(np.asarray(x, np.float32))


def _dev(bits):
    import torch
    return torch.from_numpy(np.ascontiguousarray(bits).view(np.int16)).cuda().view(torch.bfloat16)


def _inputs(T, H, g, d, seed, q_scale=1.0):
    rng = np.random.default_rng(seed)
    shapes = {"q": (T, H * g, d), "k": (T, H, d), "v": (T, H, d), "dout": (T, H * g, d)}
    return {n: _bf16(rng.normal(0, q_scale if n == "q" else 1.0, s)) for n, s in shapes.items()}


def _gpu(x, lens, H, g, d, w, sinks, max_len=None, stream=None, scale=0.0):
    """Forward and backward; outputs start as NaN."""
    import torch
    from paper_2506_05345_amd import dms
    T = x["q"].shape[0]
    cu = torch.tensor(np.concatenate([[0], np.cumsum(lens)]), dtype=torch.int32, device="cuda")
    cfg = dms.make_window_config(len(lens), T, max(lens) if max_len is None else max_len, H, g, d, w, sinks, scale)
    ws = torch.full((dms.dms_window_workspace(cfg),), 0xFF, dtype=torch.uint8, device="cuda")
    t = {n: _dev(b) for n, b in x.items()}
    nan = float("nan")
    r = {"out": torch.full_like(t["q"], nan), "lse": torch.full((H * g, T), nan, device="cuda"),
         "dq": torch.full_like(t["q"], nan), "dk": torch.full_like(t["k"], nan), "dv": torch.full_like(t["v"], nan)}
    torch.cuda.synchronize()
    dms.dms_window_attention_fwd(cfg, cu, t["q"], t["k"], t["v"], r["out"], r["lse"], ws, stream)
    ws2 = torch.full_like(ws, 0xFF)
    torch.cuda.synchronize()
    dms.dms_window_attention_bwd(cfg, cu, t["q"], t["k"], t["v"], r["out"], r["lse"], t["dout"], r["dq"], r["dk"],
                                 r["dv"], ws2, stream)
    torch.cuda.synchronize()
    return {n: y.double().cpu().numpy() for n, y in r.items()}


def _reference(x, lens, H, g, d, w, sinks, scale=None):
    """Float64 results of every packed sequence and their slacks, laid out as the library's."""
    f = {n: sy.bf16_bits_to_f32_np(b).astype(np.float64) for n, b in x.items()}
    T = x["q"].shape[0]
    shapes = {"out": (T, H * g, d), "lse": (H * g, T), "dq": (T, H * g, d), "dk": (T, H, d), "dv": (T, H, d)}
    ref, slack = ({n: np.zeros(s) for n, s in shapes.items()} for _ in range(2))
    a = 0
    for n in lens:
        b = a + n
        if n:
            q, k, v, do = (f[m][a:b] for m in ("q", "k", "v", "dout"))
            out, oslack, lse, lslack = oracle.window_attention(q, k, v, w, sinks, g, scale)
            r, sl = oracle.window_attention_grads(q, k, v, do, w, sinks, g, scale)
            for m, y, z in [("out", out, oslack), ("lse", lse, lslack)] + [(m, r[m], sl[m]) for m in r]:
                at = (slice(None), slice(a, b)) if m == "lse" else slice(a, b)
                ref[m][at], slack[m][at] = y, z
        a = b
    return ref, slack


def _check(x, lens, H, g, d, w, sinks, got, scale=None):
    ref, slack = _reference(x, lens, H, g, d, w, sinks, scale)
    n = sum(lens)
    worst = {}
    for m, y in got.items():
        here, past = ((slice(None), slice(0, n)), (slice(None), slice(n, None))) if m == "lse" else (slice(0, n), slice(n, None))
        off = np.abs(y[here] - ref[m][here]) / slack[m][here]
        assert not np.isnan(off).any(), m
        worst[m] = float(off.max())
        assert np.isnan(y[past]).all(), m     # rows of no sequence are untouched
    print({m: round(o, 3) for m, o in worst.items()})
    assert all(o <= 1.0 for o in worst.values()), worst


CASES = [
    # lens, H, g, d, w, sinks
    ([1], 1, 1, 64, 1, 0), ([1], 2, 16, 128, 5, 3), ([2, 1, 3], 2, 2, 64, 1, 0),
    ([33], 1, 2, 128, 32, 0), ([64], 2, 1, 64, 64, 4), ([65, 31], 1, 3, 128, 33, 1),
    ([200], 2, 5, 128, 16, 4), ([0, 77, 0, 128, 1], 2, 4, 64, 31, 2), ([150], 1, 7, 128, 1000, 8),
    ([129, 127], 2, 16, 64, 7, 0), ([300], 1, 6, 128, 256, 16), ([517], 1, 2, 64, 100, 33),
    ([260, 3, 90], 2, 8, 128, 128, 64), ([400], 1, 1, 128, 1, 200), ([90], 3, 5, 64, 20, 90),
    ([40, 500], 2, 5, 128, 64, 40), ([700], 1, 3, 128, 32, 1),
    # sinks with queries in several far shares, over more than one block of keys, among short sequences
    ([1500, 30, 0, 700], 1, 2, 64, 40, 140), ([1100], 2, 1, 128, 300, 5), ([512, 513, 514, 7], 1, 1, 64, 3, 1),
    ([9, 1025], 1, 3, 128, 1, 64),
]


@pytest.mark.parametrize("lens,H,g,d,w,sinks", CASES)
def test_forward_and_backward(lens, H, g, d, w, sinks):
    x = _inputs(sum(lens), H, g, d, hash((sum(lens), g, w)) % 1000, 2.0)
    _check(x, lens, H, g, d, w, sinks, _gpu(x, lens, H, g, d, w, sinks))


@pytest.mark.parametrize("lens, H, g, d, w, sinks", [
    ([1100], 29, 1, 64, 20, 3), ([700, 1, 0, 430], 29, 1, 128, 300, 37), ([1300], 26, 2, 64, 1200, 140),
    ([640, 600], 28, 1, 128, 1, 5),
])
def test_blocks_enough_to_fill_the_chip(lens, H, g, d, w, sinks):
    """256 blocks of 128 keys over the heads and more: no block's steps are shared out, sinks' far queries lie in
    longer pieces, and the near sums of sinks wait for them."""
    assert -(-sum(lens) // 128) * H >= 256
    x = _inputs(sum(lens), H, g, d, 12, 2.0)
    _check(x, lens, H, g, d, w, sinks, _gpu(x, lens, H, g, d, w, sinks))


@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_hidden_values_with_blocks_enough_to_fill_the_chip(bad):
    lens, H, g, d, w, sinks, T = [1100], 29, 1, 64, 20, 3, 1100
    x = _inputs(T, H, g, d, 13)
    ref, slack = _reference(x, lens, H, g, d, w, sinks)
    word, at = _bf16(np.array([bad]))[0], 800
    y = {n: b.copy() for n, b in x.items()}
    y["k"][at], y["v"][at] = word, word
    got = _gpu(y, lens, H, g, d, w, sinks)
    rows = np.ones(T, bool)             # queries that do not see key `at`
    rows[at:at + w] = False
    keys = np.ones(T, bool)             # keys that none of the others' gradients come from
    keys[at - w + 1:at + w] = False
    keys[:sinks] = False
    for n, where in (("out", rows), ("dq", rows), ("dk", keys), ("dv", keys)):
        assert (np.abs(got[n][where] - ref[n][where]) <= slack[n][where]).all(), n
    y = {n: b.copy() for n, b in x.items()}
    y["q"][at], y["dout"][at] = word, word
    got = _gpu(y, lens, H, g, d, w, sinks)
    keys = np.ones(T, bool)
    keys[at - w + 1:at + 1] = False
    keys[:sinks] = False
    for n in ("dk", "dv"):
        assert (np.abs(got[n][keys] - ref[n][keys]) <= slack[n][keys]).all(), n


def test_rows_past_the_last_sequence_and_a_longer_bound():
    """cu[n] below the tensors' rows, max_seqlen above the longest sequence."""
    x = _inputs(230, 2, 3, 128, 5)
    got = _gpu(x, [100, 61], 2, 3, 128, 40, 2, max_len=230)
    _check(x, [100, 61], 2, 3, 128, 40, 2, got)


@pytest.mark.parametrize("H", [1, 300])
def test_no_token_belongs_to_a_sequence(H):
    """Empty sequences alone, in a call of few blocks and of many: nothing is written."""
    x = _inputs(50, H, 2, 64, 14)
    got = _gpu(x, [0, 0, 0], H, 2, 64, 5, 2, max_len=50)
    assert all(np.isnan(y).all() for y in got.values())


@pytest.mark.parametrize("cu", [[40, 10, 130, 90], [-7, 60, 60, 2**31 - 1], [200, 200, 0, 200], [-2**31, 2**31 - 1, 5, 0]])
def test_bounds_that_break_the_rules_stay_inside(cu):
    """Offsets that fall, lie before or past the tensors: rows behind the tensors' last stay as they were."""
    import torch
    from paper_2506_05345_amd import dms
    T, H, g, d = 200, 2, 3, 128
    x = _inputs(T + 64, H, g, d, 15)
    cfg = dms.make_window_config(3, T, T, H, g, d, 30, 5)
    bounds = torch.tensor(cu, dtype=torch.int32, device="cuda")
    ws = torch.full((dms.dms_window_workspace(cfg) + 4096,), 0x5A, dtype=torch.uint8, device="cuda")
    t = {n: _dev(b) for n, b in x.items()}
    r = {n: torch.full_like(t[m], 7.0) for n, m in (("out", "q"), ("dq", "q"), ("dk", "k"), ("dv", "k"))}
    lse = torch.full((H * g * T + 64,), 7.0, device="cuda")
    dms.dms_window_attention_fwd(cfg, bounds, t["q"], t["k"], t["v"], r["out"], lse, ws)
    dms.dms_window_attention_bwd(cfg, bounds, t["q"], t["k"], t["v"], r["out"], lse, t["dout"], r["dq"], r["dk"], r["dv"], ws)
    torch.cuda.synchronize()
    assert all((y[T:] == 7).all() for y in r.values()) and (lse[H * g * T:] == 7).all() and (ws[-4096:] == 0x5A).all()


@pytest.mark.parametrize("d", [64, 128])
def test_many_short_sequences(d):
    lens = [(7 * i) % 23 for i in range(150)]
    x = _inputs(sum(lens), 1, 2, d, 6)
    _check(x, lens, 1, 2, d, 9, 3, _gpu(x, lens, 1, 2, d, 9, 3))


def test_peaked_scores_and_a_given_scale():
    x = _inputs(180, 1, 4, 128, 7, 8.0)
    _check(x, [180], 1, 4, 128, 50, 4, _gpu(x, [180], 1, 4, 128, 50, 4))
    x = _inputs(100, 1, 2, 64, 8)
    _check(x, [100], 1, 2, 64, 30, 0, _gpu(x, [100], 1, 2, 64, 30, 0, scale=0.5), scale=0.5)


@pytest.mark.parametrize("d", [64, 128])
@pytest.mark.parametrize("bad", [float("inf"), float("nan")])
def test_hidden_keys_of_any_value_change_nothing(bad, d):
    """Infinite or NaN keys and values reach the queries that see them and no others; an Inf or NaN query
    or output gradient reaches the gradients of the keys it sees and no others.  Results that they do not
    reach stay within the slack of the results without them."""
    lens, H, g, w, sinks, T = [130, 700], 1, 2, 20, 2, 830
    x = _inputs(T, H, g, d, 9)
    ref, slack = _reference(x, lens, H, g, d, w, sinks)

    def near(got, name, rows):
        at = (slice(None), rows) if name == "lse" else rows
        assert (np.abs(got[name][at] - ref[name][at]) <= slack[name][at]).all(), name

    word = _bf16(np.array([bad]))[0]
    at = 130 + 600                      # token 600 of the second sequence
    y = {n: b.copy() for n, b in x.items()}
    y["k"][at], y["v"][at] = word, word
    got = _gpu(y, lens, H, g, d, w, sinks)
    miss = np.ones(T, bool)
    miss[at:at + w] = False
    for n in ("out", "lse", "dq"):
        near(got, n, miss)
    far = np.ones(T, bool)            # keys that no query of [at, at + w) sees
    far[at - w + 1:at + w] = False
    far[130:130 + sinks] = False
    for n in ("dk", "dv"):
        near(got, n, far)
    y = {n: b.copy() for n, b in x.items()}
    y["q"][at], y["dout"][at] = word, word
    got = _gpu(y, lens, H, g, d, w, sinks)
    unseen = np.ones(T, bool)
    unseen[at - w + 1:at + 1] = False
    unseen[130:130 + sinks] = False
    for n in ("dk", "dv"):
        near(got, n, unseen)
    others = np.arange(T) != at
    for n in ("out", "lse", "dq"):
        near(got, n, others)


@pytest.mark.parametrize("H, d, w", [(1, 64, 1500), (32, 128, 1500), (2, 128, 30)])
@pytest.mark.parametrize("name", ["q", "k"])
def test_nan_scores_make_nan(name, H, d, w):
    """Queries, or keys, that are all NaN (a step that has diverged): every result that a score reaches is NaN."""
    T, g, sinks = 2500, 2, 3
    x = _inputs(T, H, g, d, 16)
    x[name][:] = _bf16(np.array([float("nan")]))[0]
    got = _gpu(x, [T], H, g, d, w, sinks)
    assert all(np.isnan(y).all() for y in got.values())


def test_results_do_not_depend_on_the_packing():
    """A sequence alone and between others gives the same bits (head dims 64 and 128)."""
    for d in (64, 128):
        lens, H, g, w, sinks = [70, 333, 20], 2, 3, 50, 5
        x = _inputs(sum(lens), H, g, d, 10)
        whole = _gpu(x, lens, H, g, d, w, sinks)
        one = _gpu({n: b[70:403] for n, b in x.items()}, [333], H, g, d, w, sinks)
        for n in ("out", "dq"):
            assert np.array_equal(whole[n][70:403], one[n]), (d, n)
        again = _gpu(x, lens, H, g, d, w, sinks)
        for n in whole:
            assert np.array_equal(whole[n], again[n]), (d, n)


def test_captured_step_replays():
    """Forward and backward in a captured graph, replayed with new inputs and eager work in between."""
    import torch
    from paper_2506_05345_amd import dms
    lens, H, g, d, w, sinks = [300, 57], 2, 3, 128, 64, 4
    T = sum(lens)
    cu = torch.tensor([0, 300, 357], dtype=torch.int32, device="cuda")
    cfg = dms.make_window_config(2, T, 300, H, g, d, w, sinks)
    ws = torch.empty(dms.dms_window_workspace(cfg), dtype=torch.uint8, device="cuda")
    t = {n: _dev(b) for n, b in _inputs(T, H, g, d, 11).items()}
    r = {"out": torch.empty_like(t["q"]), "lse": torch.empty((H * g, T), device="cuda"),
         "dq": torch.empty_like(t["q"]), "dk": torch.empty_like(t["k"]), "dv": torch.empty_like(t["v"])}

    def step():
        dms.dms_window_attention_fwd(cfg, cu, t["q"], t["k"], t["v"], r["out"], r["lse"], ws)
        dms.dms_window_attention_bwd(cfg, cu, t["q"], t["k"], t["v"], r["out"], r["lse"], t["dout"], r["dq"], r["dk"],
                                     r["dv"], ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for i in range(4):
        for n, b in _inputs(T, H, g, d, 20 + i).items():
            t[n].copy_(_dev(b))
        for y in r.values():
            y.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = {n: y.clone() for n, y in r.items()}
        step()
        torch.cuda.synchronize()
        for n in r:
            assert torch.equal(got[n], r[n]), (i, n)
        assert torch.ones(1000, device="cuda").sum().item() == 1000
    # another stream, given explicitly
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    again = _gpu(_inputs(T, H, g, d, 23), lens, H, g, d, w, sinks, stream=side)
    for n in r:
        assert np.array_equal(again[n], r[n].double().cpu().numpy()), n
