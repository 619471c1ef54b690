"""Pins of the tree and sampling oracles (CPU): closed forms, brute force, and
planted mistakes that each fail a pin."""
import math

import numpy as np
import pytest

import oracle


def _chain(rng, m, H, g, d):
    return (rng.normal(size=(m, H * g, d)), rng.normal(size=(m, H, d)), rng.normal(size=(m, H, d)),
            (rng.random((m, H)) < 0.5).astype(np.uint8))


@pytest.mark.parametrize("w", [1, 3, 50])
def test_a_chain_is_masked_attention_of_the_whole_history(w):
    rng = np.random.default_rng(w)
    m, H, g, d, past = 7, 2, 2, 8, 9
    q, k, v, f = _chain(rng, past + m, H, g, d)
    want = oracle.dense_dms_attention(q, k, v, f, w, g)
    held = [[j for j in range(past) if not f[j, h] or j > past - 1 - w] for h in range(H)]
    out, slack = oracle.tree_attention(q[past:], k[past:], v[past:], f[past:], np.arange(m) - 1, past, w, g,
                                       [k[held[h], h] for h in range(H)], [v[held[h], h] for h in range(H)], held,
                                       [f[held[h], h] for h in range(H)])
    assert np.abs(out - want[past:]).max() < 1e-12 and (slack > 0).all()


def test_a_branch_of_a_tree_is_a_chain_of_its_own():
    rng = np.random.default_rng(0)
    m, H, g, d = 9, 1, 2, 4
    q, k, v, f = _chain(rng, m, H, g, d)
    parents = [-1, 0, 0, 1, 2, 3, 3, 4, 0]
    none = [np.zeros((0, d))], [np.zeros((0, d))], [[]], [[]]
    out, _ = oracle.tree_attention(q, k, v, f, parents, 5, 2, g, *none)
    for path in oracle.tree_paths(parents):
        alone, _ = oracle.tree_attention(q[path], k[path], v[path], f[path], np.arange(len(path)) - 1, 5, 2, g, *none)
        assert np.allclose(out[path[-1]], alone[-1], atol=1e-13)


def test_accept_follows_the_targets():
    #        0
    #      1   2      tokens 7 under the root (twice), 8
    parents, tokens, targets = [-1, 0, 0, 2, 2, 4], [5, 7, 7, 9, 8, 3], [7, 9, 8, 1, 3, 6]
    assert oracle.tree_accept(parents, tokens, targets) == ([0, 1], 9)          # the lower of two equal siblings
    assert oracle.tree_accept(parents, tokens, [8] + targets[1:]) == ([0], 8)   # no child of the root has 8
    assert oracle.tree_accept(parents, [5, 1, 7, 9, 8, 3], targets) == ([0, 2, 4, 5], 6)
    assert oracle.tree_accept(parents, tokens, targets, first=4) == ([], 4)
    assert oracle.tree_accept([], [], []) == ([], -1)


def test_sampling_without_cuts_inverts_the_distribution():
    x = np.array([0.0, 1.0, -2.0, 0.5])
    p = np.exp(x / 0.7) / np.exp(x / 0.7).sum()
    edges = np.cumsum(p)
    for u in np.linspace(0, 0.999, 57):
        tok, lp = oracle.sample_token(x, float(np.float32(0.7)), u=u)
        assert tok == np.searchsorted(edges, np.float32(u), side="right") and abs(math.exp(lp) - p[tok]) < 1e-7


def test_cuts_by_hand():
    x = np.log([0.4, 0.3, 0.2, 0.1])
    tok = lambda **kw: {oracle.sample_token(x, u=u, **kw)[0] for u in np.linspace(0, 0.9999, 41)}
    assert tok() == {0, 1, 2, 3}
    assert tok(top_k=2) == {0, 1} and tok(top_k=-1) == tok(top_k=9) == {0, 1, 2, 3}
    assert tok(top_p=0.39) == {0} and tok(top_p=0.5) == {0, 1} and tok(top_p=0.95) == {0, 1, 2, 3}
    assert tok(top_k=2, top_p=0.5) == {0}          # 0.4 of the 0.7 that top-k left
    assert tok(min_p=0.5) == {0, 1, 2} and tok(min_p=0.76) == {0} and tok(top_p=0.0) == {0}
    assert tok(temperature=0.0) == {0}
    assert oracle.sample_token(np.zeros(5), top_k=2, u=0.6)[0] == 1            # equal ones by index
    assert oracle.sample_token(np.full(3, -np.inf))[0] == -1
    assert oracle.sample_token(np.array([np.nan, -np.inf, 1.0]), u=0.9)[0] == 2


@pytest.mark.parametrize("mistake", ["inclusive", "no_flag", "siblings"])
def test_planted_mistakes_of_the_tree_are_caught(mistake, monkeypatch):
    real = oracle.tree_attention

    def wrong(q, k, v, f, parents, pos, w, g, *cache):
        if mistake == "inclusive":
            w = w + 1
        elif mistake == "no_flag":
            f = np.zeros_like(f)
        else:
            parents = np.arange(len(parents)) - 1
        return real(q, k, v, f, parents, pos, w, g, *cache)

    monkeypatch.setattr(oracle, "tree_attention", wrong)
    with pytest.raises(AssertionError):
        if mistake != "siblings":
            test_a_chain_is_masked_attention_of_the_whole_history(3)
        test_a_branch_of_a_tree_is_a_chain_of_its_own()


@pytest.mark.parametrize("mistake", ["p_of_all", "strict", "ties"])
def test_planted_mistakes_of_sampling_are_caught(mistake, monkeypatch):
    real = oracle.sample_token

    def wrong(x, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, u=0.0):
        if mistake == "p_of_all" and top_k and top_p < 1:
            return real(x, temperature, 0, top_p, min_p, u)
        if mistake == "strict" and top_p < 1:
            return real(x, temperature, top_k, top_p + 0.15, min_p, u)
        if mistake == "ties" and len(set(x)) == 1:
            tok, lp = real(x[::-1], temperature, top_k, top_p, min_p, u)
            return len(x) - 1 - tok, lp
        return real(x, temperature, top_k, top_p, min_p, u)

    monkeypatch.setattr(oracle, "sample_token", wrong)
    with pytest.raises(AssertionError):
        test_cuts_by_hand()
