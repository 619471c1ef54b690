"""Trees of drafted tokens on the GPU: attention against the float64 definition,
accepted paths, and commits against the paged oracle, element by element."""
import numpy as np
import pytest

import dms_synth as sy
import oracle
from oracle import PagedKVOracle

pytestmark = pytest.mark.gpu


def bf(x):
    """float64 values of bf16 roundings."""
    return sy.bf16_bits_to_f32_np(sy.f32_to_bf16_bits_np(np.asarray(x, np.float32))).astype(np.float64)


def dev(x, kind=None):
    import torch
    x = np.ascontiguousarray(x)
    if kind == "bf16":
        return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().bfloat16()
    return torch.from_numpy(x).cuda()


def random_tree(rng, m, how):
    if how == "chain":
        return np.arange(m) - 1
    if how == "star":
        return np.where(np.arange(m) > 0, 0, -1)
    if how == "forest":
        return np.array([-1 if x == 0 or rng.random() < 0.3 else rng.integers(0, x) for x in range(m)])
    return np.array([-1 if x == 0 else max(0, x - 1 - rng.integers(0, 6)) for x in range(m)])


class Call:
    """A cache of one layer filled with random tokens, and a call's trees."""

    def __init__(self, seed, lens, nodes, H=2, g=2, d=64, w=16, P=64, kv="bf16", how="tree", p=0.6, query=False, quest=0,
                 immediate=False, layers=1, room=None):
        import torch
        from paper_2506_05345_amd import dms
        self.dms, self.rng = dms, np.random.default_rng(seed)
        rng = self.rng
        self.lens, self.H, self.g, self.d, self.w, self.kv = lens, H, g, d, w, kv
        n = self.n = len(lens)
        S = n + 1
        maxp = -(-(max(lens) + max(nodes) + 1) // P) if room is None else room
        self.cfg = dms.make_config(layers, S, H, g, d, w, P, S * H * maxp, maxp, max(sum(lens), sum(nodes)),
                                   eviction=int(immediate), decision_source=int(query), decision_bias=0.5,
                                   kv_format={"bf16": 0, "fp8": 1, "mla": 2}[kv], quest_page_budget=quest)
        self.cache = dms.DmsCache(self.cfg)
        self.ids = rng.permutation(S)[:n].astype(np.int32)
        T = sum(lens)
        self.cu_ctx = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        self.k0, self.v0 = bf(rng.normal(size=(T, H, d))), bf(rng.normal(size=(T, H, d)) + 0.3)
        self.f0 = (rng.random((T, H)) < p).astype(np.uint8)
        if T:
            dms.dms_append_chunk(self.cache.ctx, 0, n, dev(self.ids), dev(self.cu_ctx), T, max(lens), dev(self.k0, "bf16"),
                                 dev(self.v0, "bf16"), dev(self.f0))
        self.nodes, self.total, self.most = nodes, sum(nodes), max(nodes)
        self.cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
        self.parents = np.concatenate([random_tree(rng, m, how) for m in nodes] + [[]]).astype(np.int32)
        T = self.total
        self.q = bf(rng.normal(size=(T, H * g, d)) * 2)
        self.k, self.v = bf(rng.normal(size=(T, H, d))), bf(rng.normal(size=(T, H, d)) + 0.3)
        self.f = (rng.random((T, H)) < p).astype(np.uint8)
        self.ws = torch.full((dms.dms_tree_workspace(self.cfg, n, T, self.most),), 0xA5, dtype=torch.uint8, device="cuda")

    def tensors(self):
        return dict(ids=dev(self.ids), cu=dev(self.cu), parents=dev(self.parents), q=dev(self.q, "bf16"),
                    k=dev(self.k, "bf16"), v=dev(self.v, "bf16"), f=dev(self.f))

    def attend(self, t=None, out=None, stream=None):
        import torch
        t = t or self.tensors()
        if out is None:
            out = torch.full((self.total, self.H * self.g, self.d), 7.0, dtype=torch.bfloat16, device="cuda")
        self.dms.dms_tree_attention(self.cache.ctx, 0, self.n, t["ids"], t["cu"], self.total, self.most, t["parents"],
                                    t["q"], t["k"], t["v"], t["f"], out, self.ws, stream=stream)
        return out

    def expected(self, q=None, flags=None):
        held = (lambda x: oracle.fake_quantize_fp8(x)) if self.kv == "fp8" else (lambda x: x)
        q, flags = self.q if q is None else q, self.f if flags is None else flags
        view = self.cache.export(0)
        outs, slacks = [], []
        k0, v0, k, v = held(self.k0), held(self.v0), held(self.k), held(self.v)
        for i, s in enumerate(self.ids):
            a, b, c0 = self.cu[i], self.cu[i + 1], self.cu_ctx[i]
            if a == b:
                continue
            at = [view.slot_pos[s, h, :view.L[s, h]] for h in range(self.H)]
            o, sl = oracle.tree_attention(
                q[a:b], k[a:b], v[a:b], flags[a:b], self.parents[a:b], int(view.pos[s]), self.w, self.g,
                [k0[c0 + at[h], h] for h in range(self.H)], [v0[c0 + at[h], h] for h in range(self.H)], at,
                [view.slot_flag[s, h, :view.L[s, h]] for h in range(self.H)])
            outs.append(o)
            slacks.append(sl)
        return np.concatenate(outs), np.concatenate(slacks)

    def check(self, out, **kw):
        want, slack = self.expected(**kw)
        got = out.double().cpu().numpy()
        assert self.dms.dms_status(self.cache.ctx) == 0
        assert np.isfinite(got).all()
        bad = np.abs(got - want) > slack
        assert not bad.any(), (np.argwhere(bad)[:4], np.abs(got - want)[bad][:4], slack[bad][:4])


SIZES = [
    # lengths, nodes, KV heads, group, dims, window, page, tree
    ([0], [1], 1, 1, 64, 4, 32, "chain"),
    ([1], [1], 2, 2, 128, 16, 64, "chain"),
    ([40], [5], 2, 2, 64, 8, 32, "tree"),
    ([333, 0, 17], [7, 33, 1], 2, 6, 128, 16, 64, "tree"),
    ([700, 64, 129], [16, 0, 31], 4, 7, 128, 64, 64, "tree"),
    ([95, 31, 32, 33], [64, 65, 3, 32], 1, 5, 64, 7, 32, "forest"),
    ([1500], [100], 2, 3, 128, 256, 128, "chain"),
    ([260], [256], 1, 2, 64, 5, 256, "chain"),
    ([513, 200], [200, 129], 1, 16, 128, 32, 64, "tree"),
    ([64, 64], [12, 12], 8, 5, 128, 1, 64, "star"),
    ([3000], [9], 1, 4, 64, 30, 64, "forest"),
]


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("size", SIZES, ids=[f"{s[0]}x{s[1]}g{s[3]}d{s[4]}w{s[5]}" for s in SIZES])
def test_attention_matches_its_definition(size, kv):
    lens, nodes, H, g, d, w, P, how = size
    c = Call(len(str(size)), lens, nodes, H, g, d, w, P, kv, how)
    before = c.cache.export(0)
    out = c.attend()
    c.check(out)
    after = c.cache.export(0)       # nothing is appended
    for name in ("pos", "L", "ring_slot", "ring_flag", "page_table", "slot_pos", "slot_flag", "stack"):
        assert np.array_equal(getattr(before, name), getattr(after, name)), name


def test_a_chain_attends_as_decode_steps_do():
    """Nodes of a chain against dms_decode_step of the same tokens: both round weights to bf16 (decode: float32 out)."""
    import torch
    c = Call(3, [300], [20], 2, 3, 128, 9, 64, how="chain")
    out = c.attend().double().cpu().numpy()
    want, slack = c.expected()
    dms, H, g, d = c.dms, c.H, c.g, c.d
    step = torch.empty((1, H * g, d), device="cuda")
    for x in range(20):
        dms.dms_decode_step(c.cache.ctx, 0, 1, dev(c.ids), dev(c.q[x:x + 1], "bf16"), dev(c.k[x:x + 1], "bf16"),
                            dev(c.v[x:x + 1], "bf16"), dev(c.f[x:x + 1]), step)
        assert (np.abs(step.double().cpu().numpy()[0] - out[x]) <= 2 * slack[x]).all(), x


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_decisions_from_queries(kv):
    import torch
    c = Call(5, [200, 50], [12, 40], 2, 3, 128, 6, 64, kv, query=True, how="chain")
    t = c.tensors()
    out = torch.empty((c.total, c.H * c.g, c.d), dtype=torch.bfloat16, device="cuda")
    dec = torch.full((c.total, c.H), 9, dtype=torch.uint8, device="cuda")
    args = (c.cache.ctx, 0, c.n, t["ids"], t["cu"], c.total, c.most, t["parents"], t["q"], t["k"], t["v"])
    c.dms.dms_tree_attention_q(*args, dec, out, c.ws)
    flags = (c.q[:, ::c.g, 0] + 0.5 > 0).astype(np.uint8)
    assert np.array_equal(dec.cpu().numpy(), flags)
    q = c.q.copy()
    q[:, ::c.g, 0] = 0
    c.check(out, q=q, flags=flags)
    again = torch.empty_like(out)
    c.dms.dms_tree_attention_q(*args, None, again, c.ws)
    assert torch.equal(out, again)


def test_page_retrieval_contexts_attend_all_slots():
    c = Call(6, [400], [9], 2, 2, 64, 16, 32, quest=2)
    c.check(c.attend())


def test_large_scores():
    c = Call(7, [150, 3], [20, 5], 2, 4, 64, 20, 32)
    c.q *= 16          # scores of hundreds: one key takes nearly all the weight
    c.check(c.attend())


@pytest.mark.parametrize("value", [np.inf, -np.inf, np.nan])
@pytest.mark.parametrize("kv", ["bf16", "fp8"])
def test_hidden_infinities_reach_no_other_branch(value, kv):
    """Keys and values of a node that are not finite change its descendants and itself alone; slots past the live
    length hold anything."""
    import torch
    c = Call(8, [70, 100], [40, 9], 2, 3, 128, 8, 32, kv)
    base = c.attend()
    want, slack = c.expected()
    t = c.tensors()
    x = 11
    below = [y for y, p in enumerate(oracle.tree_paths(c.parents[:40])) if x in p]
    others = [y for y in range(c.total) if y not in below]
    assert len(below) < 30
    for name in ("k", "v"):
        bad = t[name].clone()
        bad[x, :, 5] = value
        out = c.attend(dict(t, **{name: bad}))
        assert torch.equal(out[others], base[others]), name
        if name == "v" and kv == "bf16":
            hit = out[below][..., 5].float()
            # a weight of 0 times an infinity is NaN, as in any sum of products
            assert (~torch.isfinite(hit)).all()
            keep = [e for e in range(c.d) if e != 5]
            got = out[below][..., keep].double().cpu().numpy()
            assert (np.abs(got - want[below][..., keep]) <= slack[below][..., keep]).all()


def test_expired_slots_with_infinite_values():
    """A flagged slot that the deeper nodes of a chain no longer see."""
    import torch
    w = 6
    c = Call(9, [50], [10], 1, 2, 64, w, 32, how="chain", p=1.0)
    base = c.attend()
    want, slack = c.expected()
    # the slot of position 48: visible to nodes at positions 50 .. 53, expired from 54 on
    view = c.cache.export(0)
    s = int(c.ids[0])
    slot = int(np.argwhere(view.slot_pos[s, 0, :view.L[s, 0]] == 48)[0, 0])
    page = int(view.page_table[s, 0, slot // 32])
    words = c.cache.pools[0].view(torch.int16).view(c.cfg.num_pages, -1)
    j, e = slot % 32, 3
    off = 32 * c.d + (((e // 16) * 4 + j // 8) * 16 + e % 16) * 8 + j % 8
    words[page, off] = 0x7F80      # +inf
    out = c.attend()
    assert (~torch.isfinite(out[:4, :, 3].float())).all()
    assert torch.equal(out[4:], base[4:])
    assert (np.abs(out[:4, :, 4:].double().cpu().numpy() - want[:4, :, 4:]) <= slack[:4, :, 4:]).all()


def test_results_do_not_depend_on_the_run_or_the_workspace():
    import torch
    c = Call(10, [2000, 900], [50, 31], 2, 6, 128, 64, 64)
    a = c.attend()
    c.ws.random_(0, 256)
    assert torch.equal(a, c.attend())
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    out = torch.empty_like(a)
    c.attend(out=out, stream=stream)
    torch.cuda.synchronize()
    assert torch.equal(a, out)


@pytest.mark.parametrize("how", ["ids", "twice", "cu", "order", "large", "parent", "self"])
def test_device_side_errors_leave_the_outputs(how):
    import torch
    c = Call(11, [60, 70], [8, 12], 2, 2, 64, 8, 32)
    t = c.tensors()
    code = c.dms.DMS_ERR_INVALID
    if how == "ids":
        t["ids"][1], code = c.cfg.max_seqs, c.dms.DMS_ERR_BAD_SEQ
    elif how == "twice":
        t["ids"][1], code = int(c.ids[0]), c.dms.DMS_ERR_BAD_SEQ
    elif how == "cu":
        t["cu"][2] = 19
    elif how == "order":
        t["cu"][1] = 21
    elif how == "large":
        t["cu"][1] = 7          # the second tree then has 13 nodes, more than max_nodes
    elif how == "parent":
        t["parents"][3] = -2
    else:
        t["parents"][9] = 1     # node 1 of the second tree: its own parent
    out = torch.full((c.total, c.H * c.g, c.d), 7.0, dtype=torch.bfloat16, device="cuda")
    c.attend(t, out)
    assert c.dms.dms_status(c.cache.ctx) == code
    assert (out == 7).all()
    c.dms.dms_clear_status(c.cache.ctx)
    c.check(c.attend())


# ---------------------------------------------------------------------------
# Accepted paths
# ---------------------------------------------------------------------------

@pytest.mark.parametrize("n,most,how", [(1, 1, "chain"), (1, 16, "tree"), (5, 33, "forest"), (300, 128, "tree"),
                                        (7, 256, "chain"), (64, 64, "star")])
@pytest.mark.parametrize("given", [True, False])
def test_accepted_paths(n, most, how, given):
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(n + most)
    nodes = rng.integers(0, most + 1, n)
    nodes[0] = most
    cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    T = int(cu[-1])
    parents = np.concatenate([random_tree(rng, m, how) for m in nodes]).astype(np.int32)
    tokens, targets = rng.integers(0, 4, T).astype(np.int32), rng.integers(0, 4, T).astype(np.int32)
    if how == "chain":
        agree = np.arange(T)[1:][rng.random(T - 1) < 0.97]
        tokens[agree] = targets[agree - 1]
    first = rng.integers(0, 4, n).astype(np.int32)
    path = torch.full((T + 3,), 77, dtype=torch.int32, device="cuda")
    length, nxt = (torch.full((n,), 77, dtype=torch.int32, device="cuda") for _ in range(2))
    dms.dms_tree_accept(n, dev(cu), T, most, dev(parents), dev(tokens), dev(targets), dev(first) if given else None, path,
                        length, nxt)
    path, length, nxt = path.cpu().numpy(), length.cpu().numpy(), nxt.cpu().numpy()
    for i in range(n):
        a, b = cu[i], cu[i + 1]
        want, token = oracle.tree_accept(parents[a:b], tokens[a:b], targets[a:b], first[i] if given else None)
        assert length[i] == len(want) and nxt[i] == token
        assert np.array_equal(path[a:b], want + [-1] * (b - a - len(want)))
    assert (path[T:] == 77).all()


def test_accepted_paths_of_broken_trees_stay_inside():
    import torch
    from paper_2506_05345_amd import dms
    cu = dev(np.array([-5, 9, 3, 4000], np.int32))
    parents = dev(np.array([5, 5, -7, 0, 1, 1, 9, 2**31 - 1, -1, -1, 3, 3], np.int32))
    same = dev(np.zeros(12, np.int32))
    guard = torch.full((64,), 77, dtype=torch.int32, device="cuda")
    dms.dms_tree_accept(3, cu, 12, 12, parents, same, same, None, guard[16:28], guard[32:35], guard[40:43])
    g = guard.cpu().numpy()
    assert (g[:16] == 77).all() and (g[28:32] == 77).all() and (g[35:40] == 77).all() and (g[43:] == 77).all()
    assert (g[32:35] >= 0).all() and (g[32:35] <= 12).all()


# ---------------------------------------------------------------------------
# Commits
# ---------------------------------------------------------------------------

def some_paths(rng, c, mode="mixed"):
    path, lens = np.full(c.total, -1, np.int32), []
    for i in range(c.n):
        a, m = c.cu[i], c.cu[i + 1] - c.cu[i]
        line = []
        if m and mode != "empty":
            lines = oracle.tree_paths(c.parents[a:a + m])
            line = max(lines, key=len) if mode == "longest" else lines[rng.integers(0, m)]
            if mode == "mixed" and rng.random() < 0.25:
                line = line[:rng.integers(0, len(line) + 1)]
        path[a:a + len(line)] = line
        lens.append(len(line))
    return path, np.array(lens, np.int32)


def pool_words(c):
    import torch
    torch.cuda.synchronize()
    return c.cache.pools[0].cpu().numpy().copy()


COMMITS = [
    ([40], [5], 2, 2, 64, 8, 32, "bf16", {}),
    ([0, 1], [3, 7], 2, 2, 64, 4, 32, "bf16", {}),
    ([333, 0, 17], [7, 33, 1], 2, 3, 128, 16, 64, "bf16", {}),
    ([100, 90], [256, 100], 1, 2, 64, 1, 32, "bf16", {"how": "chain"}),
    ([100, 90], [200, 100], 2, 2, 64, 7, 32, "fp8", {"how": "chain"}),
    ([200, 31, 64], [64, 0, 20], 2, 2, 128, 300, 64, "fp8", {}),
    ([70, 300], [20, 40], 1, 16, 576, 16, 64, "mla", {"how": "chain"}),
    ([150, 77], [30, 50], 2, 2, 64, 5, 32, "bf16", {"how": "chain", "immediate": True}),
    ([150, 77], [30, 50], 2, 2, 64, 5, 32, "bf16", {"how": "chain", "quest": 2}),
    ([30] * 40, [9] * 40, 4, 2, 64, 6, 32, "bf16", {}),
    ([60] * 9, [70, 3, 20] * 3, 2, 2, 64, 7, 32, "fp8", {"how": "chain"}),
    ([40, 3, 77] * 6, [9, 130, 0] * 6, 1, 16, 576, 5, 64, "mla", {"how": "chain"}),
    ([90] * 9, [30] * 9, 2, 2, 64, 5, 32, "bf16", {"how": "chain", "immediate": True}),
    ([20] * 16, [65] * 16, 1, 2, 64, 300, 32, "bf16", {"how": "chain"}),
]


@pytest.mark.parametrize("mode", ["mixed", "longest", "empty"])
@pytest.mark.parametrize("size", COMMITS, ids=[f"{s[0][:3]}x{s[1][:3]}d{s[4]}w{s[5]}{s[7]}{len(s[8])}" for s in COMMITS])
def test_commit_is_an_append_of_the_path(size, mode):
    """State and pool, byte by byte, against dms_append_chunk of the gathered rows in a second cache."""
    lens, nodes, H, g, d, w, P, kv, more = size
    a, b = (Call(21, lens, nodes, H, g, d, w, P, kv, **more) for _ in range(2))
    for c in (a, b):
        c.cache.pools[0].zero_()
        c.dms.dms_init_state(c.cache.ctx)
        T = sum(lens)
        if T:
            c.dms.dms_append_chunk(c.cache.ctx, 0, c.n, dev(c.ids), dev(c.cu_ctx), T, max(lens), dev(c.k0, "bf16"),
                                   dev(c.v0, "bf16"), dev(c.f0))
    path, plen = some_paths(np.random.default_rng(4), a, mode)
    t = a.tensors()
    a.dms.dms_tree_commit(a.cache.ctx, 0, a.n, t["ids"], t["cu"], a.total, a.most, dev(path), dev(plen), t["k"],
                          None if kv == "mla" else t["v"], t["f"], a.ws)
    rows = np.concatenate([a.cu[i] + path[a.cu[i]:a.cu[i] + plen[i]] for i in range(a.n)]).astype(np.int64)
    cu = np.concatenate([[0], np.cumsum(plen)]).astype(np.int32)
    if len(rows):
        b.dms.dms_append_chunk(b.cache.ctx, 0, b.n, dev(b.ids), dev(cu), len(rows), int(plen.max()),
                               dev(b.k[rows], "bf16"), dev(b.v[rows], "bf16"), dev(b.f[rows]))
    assert a.dms.dms_status(a.cache.ctx) == 0 and b.dms.dms_status(b.cache.ctx) == 0
    va, vb = a.cache.export(0), b.cache.export(0)
    assert np.array_equal(va.pos, vb.pos) and np.array_equal(va.L, vb.L) and va.top == vb.top
    assert np.array_equal(va.stack, vb.stack) and np.array_equal(va.page_table, vb.page_table)
    for s in a.ids:
        for h in range(H):
            L, t0 = int(va.L[s, h]), int(va.pos[s])
            e = [p % w for p in range(max(0, t0 - w), t0)]
            assert np.array_equal(va.ring_slot[s, h, e], vb.ring_slot[s, h, e])
            assert np.array_equal(va.ring_flag[s, h, e], vb.ring_flag[s, h, e])
            assert np.array_equal(va.slot_pos[s, h, :L], vb.slot_pos[s, h, :L])
            assert np.array_equal(va.slot_flag[s, h, :L], vb.slot_flag[s, h, :L])
    assert np.array_equal(pool_words(a), pool_words(b))
    if more.get("quest"):
        o = a.cache.offsets
        size = a.cfg.num_pages * 4 * d
        at = o.layer0 + o.page_bounds
        used = sorted(int(p) for s in a.ids for h in range(H) for p in va.page_table[s, h, :-(-int(va.L[s, h]) // P)])
        x, y = (c.cache.meta[at:at + size].cpu().numpy().reshape(a.cfg.num_pages, -1)[used] for c in (a, b))
        assert np.array_equal(x, y)


def test_commit_of_many_heads():
    """More heads than a workgroup sums for itself (2048): the summed form of the second pass."""
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(5)
    n, H, d, w, P = 300, 8, 64, 3, 32
    cfg = dms.make_config(1, n, H, 1, d, w, P, n * H * 2, 2, n * 6)
    caches = [dms.DmsCache(cfg) for _ in range(2)]
    nodes = rng.integers(1, 6, n)
    cu = np.concatenate([[0], np.cumsum(nodes)]).astype(np.int32)
    T = int(cu[-1])
    k, v = dev(rng.normal(size=(T, H, d)), "bf16"), dev(rng.normal(size=(T, H, d)), "bf16")
    f = dev((rng.random((T, H)) < 0.5).astype(np.uint8))
    ids = dev(rng.permutation(n).astype(np.int32))
    path = np.concatenate([np.arange(m) for m in nodes]).astype(np.int32)
    ws = torch.empty(dms.dms_tree_workspace(cfg, n, T, int(nodes.max())), dtype=torch.uint8, device="cuda")
    for c in caches:
        c.pools[0].zero_()
    for _ in range(6):
        dms.dms_tree_commit(caches[0].ctx, 0, n, ids, dev(cu), T, int(nodes.max()), dev(path),
                            dev(nodes.astype(np.int32)), k, v, f, ws)
        dms.dms_append_chunk(caches[1].ctx, 0, n, ids, dev(cu), T, int(nodes.max()), k, v, f)
    va, vb = (c.export(0) for c in caches)
    assert dms.dms_status(caches[0].ctx) == 0 and va.top == vb.top
    for name in ("pos", "L", "ring_slot", "ring_flag", "page_table", "stack"):
        assert np.array_equal(getattr(va, name), getattr(vb, name)), name
    assert torch.equal(caches[0].pools[0], caches[1].pools[0])


@pytest.mark.parametrize("how", ["ids", "twice", "cu", "node", "negative", "long", "short", "capacity", "pages"])
def test_refused_commits_change_nothing(how):
    c = Call(31, [60, 70], [12, 12], 2, 2, 64, 8, 32, how="chain", p=0.0, room=3 if how == "capacity" else None)
    dms = c.dms
    t = c.tensors()
    path, plen = some_paths(np.random.default_rng(1), c, "longest")
    code = dms.DMS_ERR_INVALID
    if how == "ids":
        t["ids"][0], code = -1, dms.DMS_ERR_BAD_SEQ
    elif how == "twice":
        t["ids"][0], code = int(c.ids[1]), dms.DMS_ERR_BAD_SEQ
    elif how == "cu":
        t["cu"][2] = 23
    elif how == "node":
        path[14] = 12
    elif how == "negative":
        path[3] = -1
    elif how == "long":
        plen[1] = 13
    elif how == "short":
        plen[0] = -1
    elif how == "capacity":
        # 3 pages of 32 slots a head, nothing evicted: 70, 82 and 94 tokens fit, 106 do not
        for _ in range(2):
            dms.dms_tree_commit(c.cache.ctx, 0, c.n, t["ids"], t["cu"], c.total, c.most, dev(path), dev(plen), t["k"],
                                t["v"], t["f"], c.ws)
        code = dms.DMS_ERR_CAPACITY
    elif how == "pages":
        # 2 heads x (2 + 3) pages of 11 are taken, and two heads of 72 tokens need one more each
        c.cache = dms.DmsCache(dms.make_config(1, 3, 2, 2, 64, 8, 32, 11, 6, 256))
        dms.dms_append_chunk(c.cache.ctx, 0, 2, dev(c.ids), dev(c.cu_ctx), 130, 70, dev(c.k0, "bf16"),
                             dev(c.v0, "bf16"), dev(c.f0))
        code = dms.DMS_ERR_OUT_OF_PAGES
    assert dms.dms_status(c.cache.ctx) == 0
    before, pool = c.cache.export(0), pool_words(c)
    dms.dms_tree_commit(c.cache.ctx, 0, c.n, t["ids"], t["cu"], c.total, c.most, dev(path), dev(plen), t["k"], t["v"],
                        t["f"], c.ws)
    assert dms.dms_status(c.cache.ctx) == code
    after = c.cache.export(0)
    for name in ("pos", "L", "ring_slot", "ring_flag", "page_table", "slot_pos", "slot_flag", "stack"):
        assert np.array_equal(getattr(before, name), getattr(after, name)), name
    assert before.top == after.top and np.array_equal(pool, pool_words(c))


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("byte", [0xFF, 0x7F, 0x00])
def test_slots_past_the_live_length_hold_anything(kv, byte):
    """A pool that held other bytes before its slots were written (0xFF and 0x7F: NaN keys, values and scales)."""
    import torch
    for lens, nodes, g in (([5, 40], [3, 9], 2), ([333], [40], 2), ([33, 95], [70, 5], 4), ([0, 500], [1, 100], 2),
                           ([45, 100], [20, 5], 3)):
        c = Call(41, lens, nodes, 2, g, 128, 16, 64, kv)
        c.cache.pools[0].view(torch.uint8).fill_(byte)
        c.dms.dms_init_state(c.cache.ctx)
        c.dms.dms_append_chunk(c.cache.ctx, 0, c.n, dev(c.ids), dev(c.cu_ctx), sum(lens), max(lens), dev(c.k0, "bf16"),
                               dev(c.v0, "bf16"), dev(c.f0))
        c.check(c.attend())


def test_commit_of_a_repeated_node():
    """A path may name a node more than once: its rows are appended as often."""
    for n in (2, 12):
        a, b = (Call(51, [40] * n, [6] * n, 2, 2, 64, 4, 32) for _ in range(2))
        path, plen = np.full(a.total, -1, np.int32), np.full(n, 4, np.int32)
        for i in range(n):
            path[a.cu[i]:a.cu[i] + 4] = [1, 1, 5, 1]
        t = a.tensors()
        a.dms.dms_tree_commit(a.cache.ctx, 0, n, t["ids"], t["cu"], a.total, a.most, dev(path), dev(plen), t["k"], t["v"], t["f"],
                              a.ws)
        rows = np.concatenate([a.cu[i] + np.array([1, 1, 5, 1]) for i in range(n)])
        cu = 4 * np.arange(n + 1, dtype=np.int32)
        b.dms.dms_append_chunk(b.cache.ctx, 0, n, dev(b.ids), dev(cu), 4 * n, 4, dev(b.k[rows], "bf16"), dev(b.v[rows], "bf16"),
                               dev(b.f[rows]))
        va, vb = a.cache.export(0), b.cache.export(0)
        assert a.dms.dms_status(a.cache.ctx) == 0
        for s in a.ids:
            for h in range(2):
                L = int(vb.L[s, h])
                assert va.L[s, h] == L and va.pos[s] == vb.pos[s]
                assert np.array_equal(va.slot_pos[s, h, :L], vb.slot_pos[s, h, :L])
                assert np.array_equal(va.page_table[s, h, :-(-L // 32)], vb.page_table[s, h, :-(-L // 32)])


def test_pages_past_four_gigabytes():
    """A pool of 6 GB whose last pages come first."""
    import torch
    from paper_2506_05345_amd import dms
    c = Call(52, [700, 90], [40, 7], 2, 3, 128, 16, 64)
    base = c.attend()
    cfg = dms.make_config(1, 3, 2, 3, 128, 16, 64, 190000, 16, 790)
    big = dms.DmsCache(cfg)
    o = big.offsets
    stack = big.meta[o.layer0 + o.stack:o.layer0 + o.stack + 4 * 190000].view(torch.int32)
    assert int(stack[-1]) == 0
    stack.copy_(stack.flip(0).clone())
    dms.dms_append_chunk(big.ctx, 0, 2, dev(c.ids), dev(c.cu_ctx), 790, 700, dev(c.k0, "bf16"), dev(c.v0, "bf16"), dev(c.f0))
    assert int(big.export(0).page_table[c.ids[0], 0, 0]) * 32768 > 1 << 32
    c.cache = big
    assert torch.equal(c.attend(), base)
    path, plen = some_paths(c.rng, c, "longest")
    t = c.tensors()
    dms.dms_tree_commit(big.ctx, 0, 2, t["ids"], t["cu"], c.total, c.most, dev(path), dev(plen), t["k"], t["v"], t["f"], c.ws)
    assert dms.dms_status(big.ctx) == 0
    out = torch.empty((2, 6, 128), device="cuda")
    step = lambda cache: dms.dms_decode_step(cache.ctx, 0, 2, dev(c.ids), t["q"][:2].contiguous(), t["k"][:2].contiguous(),
                                             t["v"][:2].contiguous(), t["f"][:2].contiguous(), out)
    step(big)
    got = out.clone()
    small = Call(52, [700, 90], [40, 7], 2, 3, 128, 16, 64)
    dms.dms_tree_commit(small.cache.ctx, 0, 2, t["ids"], t["cu"], c.total, c.most, dev(path), dev(plen), t["k"], t["v"], t["f"],
                        small.ws)
    step(small.cache)
    assert torch.equal(got, out)


def ragged(n, lens, nodes):
    """n sequences that take their lengths and trees from two cycles; the first and the last have no nodes."""
    a, b = [lens[i % len(lens)] for i in range(n)], [nodes[i % len(nodes)] for i in range(n)]
    b[0] = b[-1] = 0
    return a, b


LISTS = {
    # 12 heads, 400 columns of 25 units each at most: 16 parts, cut without regard to heads
    "units": ([700, 40, 333, 5, 64, 129], [200, 0, 130, 5, 0, 64], 2, 16, 64, 16, 64, 0.6),
    # four long heads in 16 parts: every head over several of them
    "long": ([3100, 2500], [200, 3], 2, 16, 64, 256, 64, 0.3),
    # many short heads, several to a part, of 32, 64 and 128 columns a unit
    "32": (*ragged(72, [300, 0, 40, 1, 95, 130, 33], [6, 1, 0, 3, 0]), 4, 5, 128, 16, 32, 0.6),
    "64": (*ragged(70, [260, 31, 0, 150, 64], [16, 0, 2, 7]), 4, 4, 64, 9, 64, 0.6),
    "128": (*ragged(66, [200, 90, 3, 0, 420], [18, 0, 0, 5, 1, 11]), 4, 7, 128, 20, 64, 0.5),
    # more heads than the plan holds in LDS (512)
    "heads": (*ragged(150, [120, 0, 33, 64], [2, 0, 1, 3, 0, 0]), 4, 2, 64, 8, 32, 0.6),
}


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("name", LISTS)
def test_tiles_cut_without_regard_to_heads(name, kv):
    """Calls of many heads or tiles: the tiles of all heads are one list in equal parts, which begin and end anywhere in a
    head and go on past heads without nodes."""
    import torch
    lens, nodes, H, g, d, w, P, p = LISTS[name]
    c = Call(61 + len(name), lens, nodes, H, g, d, w, P, kv, p=p)
    out = c.attend()
    c.check(out)
    # the sizes do ask for such a list: two workgroups a compute unit, at least eight tiles a part
    view = c.cache.export(0)
    tiles = sum(-(-int(view.L[s, h]) // 32) + -(-m // 32) for s, m in zip(c.ids, nodes) if m for h in range(H))
    cols = max(nodes) * g
    units = -(-cols // (32 if cols <= 32 else 64 if cols <= 64 else 128))
    most = 2 * torch.cuda.get_device_properties(0).multi_processor_count // 8 // units * 8
    assert c.n * H > 512 or c.n * H > most // 2 or tiles >= 16 * most
    assert tiles > 2 * 8
    c.ws.random_(0, 256)
    assert torch.equal(out, c.attend())


@pytest.mark.parametrize("kv", ["bf16", "fp8"])
@pytest.mark.parametrize("name", ["units", "32", "64", "128"])
def test_hidden_infinities_where_heads_share_a_part(name, kv):
    """Dead slots of NaN bytes, and a node of infinite values in one head: only its descendants and that head change,
    whatever else the workgroup attends before and after."""
    import torch
    lens, nodes, H, g, d, w, P, p = LISTS[name]
    c = Call(71 + len(name), lens, nodes, H, g, d, w, P, kv, p=p)
    c.cache.pools[0].view(torch.uint8).fill_(0xFF)
    c.dms.dms_init_state(c.cache.ctx)
    c.dms.dms_append_chunk(c.cache.ctx, 0, c.n, dev(c.ids), dev(c.cu_ctx), sum(lens), max(lens), dev(c.k0, "bf16"),
                           dev(c.v0, "bf16"), dev(c.f0))
    base = c.attend()
    c.check(base)
    t = c.tensors()
    i = int(np.argmax(c.nodes))
    x = c.cu[i] + 1
    below = [c.cu[i] + y for y, q in enumerate(oracle.tree_paths(c.parents[c.cu[i]:c.cu[i + 1]])) if 1 in q]
    bad = t["v"].clone()
    bad[x, 1, 9] = np.inf
    out = c.attend(dict(t, v=bad))
    changed = (out != base) | ~torch.isfinite(out.float())
    allowed = torch.zeros_like(changed)
    allowed[below, g:2 * g] = True
    assert not (changed & ~allowed).any()
    assert not torch.isfinite(out[x, g:2 * g, 9].float()).any()
