"""The oracles of the windowed attention, the rotary positions, forks and
compaction against definitions, differences and each other (CPU)."""
import math

import numpy as np
import pytest

import oracle
from oracle import OutOfPages, PagedKVOracle


@pytest.mark.parametrize("T,w,sinks", [(1, 1, 0), (7, 3, 0), (9, 4, 2), (6, 20, 1), (8, 1, 8)])
def test_window_mask_is_the_dms_mask_of_its_decisions(T, w, sinks):
    flags = (np.arange(T) >= sinks).astype(np.uint8)
    assert np.array_equal(oracle.window_mask(T, w, sinks), oracle.visibility_mask(flags, w))


def test_window_gradients_against_differences():
    rng = np.random.default_rng(0)
    T, H, g, d, w, sinks = 9, 2, 3, 4, 3, 2
    q, k, v, do = (rng.normal(size=(T, n, d)) for n in (H * g, H, H, H * g))
    grads, _ = oracle.window_attention_grads(q, k, v, do, w, sinks, g)

    def loss(q, k, v):
        return float((oracle.window_attention(q, k, v, w, sinks, g)[0] * do).sum())

    for name, x in (("dq", q), ("dk", k), ("dv", v)):
        for _ in range(12):
            i = tuple(rng.integers(0, n) for n in x.shape)
            old, h = x[i], 1e-5
            x[i] = old + h
            up = loss(q, k, v)
            x[i] = old - h
            down = loss(q, k, v)
            x[i] = old
            assert abs((up - down) / (2 * h) - grads[name][i]) < 1e-7, (name, i)


def test_window_attention_equals_training_attention_of_binary_decisions():
    rng = np.random.default_rng(1)
    T, H, g, d, w, sinks = 30, 2, 2, 8, 5, 3
    q, k, v = (rng.normal(size=(T, n, d)) for n in (H * g, H, H))
    alpha = np.broadcast_to((np.arange(T) >= sinks)[None, :, None], (1, T, H)).astype(np.float64)
    out, lse = oracle.train_attention(q[None], k[None], v[None], alpha, w, g)
    got, _, got_lse, _ = oracle.window_attention(q, k, v, w, sinks, g)
    assert np.abs(got - out[0]).max() < 1e-12 and np.abs(got_lse - lse[0]).max() < 1e-12


def test_rope_axes_cover_the_sections():
    assert oracle.rope_axes([2, 3], False) == [0, 0, 1, 1, 1]
    assert oracle.rope_axes([4, 2, 2], True) == [0, 1, 2, 0, 1, 2, 0, 0]
    for sec in ([5, 5, 5], [6, 4, 1], [3, 0], [7]):
        axes = oracle.rope_axes(sec, True)
        assert [axes.count(a) for a in range(len(sec))] == sec


def test_rope_turns_and_turns_back():
    rng = np.random.default_rng(2)
    x = rng.normal(size=(5, 3, 24))
    pos = rng.integers(-1000, 100000, (2, 5))
    inv = 10000.0 ** (-np.arange(8) / 8)
    axes = oracle.rope_axes([5, 3], False)
    for adjacent in (False, True):
        y = oracle.rope_rotate(x, pos, inv, axes, 16, 4, adjacent)
        assert np.abs(oracle.rope_rotate(y, pos, inv, axes, 16, 4, adjacent, back=True) - x).max() < 1e-10
        assert np.array_equal(y[..., :4], x[..., :4]) and np.array_equal(y[..., 20:], x[..., 20:])
        # pair 5 is the first of axis 1: a rotation matrix of its angle
        a, b = (4 + 10, 4 + 11) if adjacent else (4 + 5, 4 + 13)
        c, s = math.cos(pos[1, 2] * inv[5]), math.sin(pos[1, 2] * inv[5])
        assert abs(y[2, 1, a] - (x[2, 1, a] * c - x[2, 1, b] * s)) < 1e-9
        assert abs(y[2, 1, b] - (x[2, 1, a] * s + x[2, 1, b] * c)) < 1e-9


def _filled(seed, pages=60):
    rng = np.random.default_rng(seed)
    o = PagedKVOracle(8, 2, 5, 32, pages, 8, 4)
    o.append_chunk([1, 4], [(rng.random((n, 2)) < 0.7).astype(np.uint8) for n in (150, 90)],
                   [rng.normal(size=(n, 2, 4)) for n in (150, 90)], [rng.normal(size=(n, 2, 4)) for n in (150, 90)])
    return o, rng


def test_forked_sequences_decode_like_their_source_and_keep_pages_apart():
    o, rng = _filled(3)
    o.seq_fork([1, 1, 4, 6], [0, 7, 2, 5])        # sequence 6 is empty
    q = rng.normal(size=(1, 4, 4))
    for s, d in ((1, 0), (1, 7), (4, 2)):
        assert np.array_equal(o.decode([s], q, 2), o.decode([d], q, 2))
    assert o.pos[5] == 0 and not o.L[5].any()
    held = [int(p) for s in range(8) for h in range(2) for p in o.page_table[s, h, :-(-int(o.L[s, h]) // 32)]]
    assert len(set(held)) == len(held) and set(held) | set(map(int, o.free_stack())) == set(range(60))
    assert len(held) + o.top == 60
    # released in call order and forked again: the same pages
    table = o.page_table[[0, 7, 2]].copy()
    o.seq_reset([0, 7, 2])
    o.seq_fork([1, 1, 4], [0, 7, 2])
    for x, d in enumerate((0, 7, 2)):
        for h in range(2):
            n = -(-int(o.L[d, h]) // 32)
            assert np.array_equal(o.page_table[d, h, :n], table[x, h, :n])


def test_fork_refusals():
    o, _ = _filled(4)
    for src, dst in (([1], [4]), ([1], [1]), ([1, 1], [0, 0]), ([6, 1], [5, 6])):
        with pytest.raises(ValueError):
            o.seq_fork(src, dst)
    small, _ = _filled(4, pages=14)
    with pytest.raises(OutOfPages):
        small.seq_fork([1, 1, 1], [0, 2, 3])


def test_compaction_packs_the_pool_and_changes_no_output():
    o, rng = _filled(5)
    o.seq_fork([1, 4, 1], [0, 2, 3])
    o.seq_reset([1, 2])
    q = rng.normal(size=(1, 4, 4))
    before = [o.decode([s], q, 2) for s in (0, 3, 4)]
    used = o.compact()
    held = [int(p) for s in range(8) for h in range(2) for p in o.page_table[s, h, :-(-int(o.L[s, h]) // 32)]]
    assert sorted(held) == list(range(used)) and used + o.top == 60
    assert list(o.free_stack()) == list(range(59, used - 1, -1))
    for s, b in zip((0, 3, 4), before):
        assert np.array_equal(o.decode([s], q, 2), b)
