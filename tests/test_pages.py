"""GPU parity of sequence forks and pool compaction: state bit-exact against the
oracle's replay after every call, pool contents by owner, outputs of decode
steps on copies and after moves, device-side refusals that change nothing."""
import numpy as np
import pytest

from dms_testlib import ATOL, SeqInputs, bf16_to_f32, compare_pool, compare_pool_fp8, compare_state, to_dev
from oracle import PagedKVOracle

pytestmark = pytest.mark.gpu


class _Run:
    """A cache and the oracle's replay, taken through the same calls on every layer."""

    def __init__(self, S, H, g, d, w, P, pages, maxp, fmt="bf16", layers=1, budget=0, seed=0, mode="delayed"):
        import torch
        from paper_2506_05345_amd import dms
        self.dms, self.H, self.g, self.d = dms, H, g, d
        fmts = {"bf16": dms.DMS_KV_BF16, "fp8": dms.DMS_KV_FP8}
        self.cfg = dms.make_config(layers, S, H, g, d, w, P, pages, maxp, 4096, kv_format=fmts[fmt],
                                   quest_page_budget=budget,
                                   eviction=dms.DMS_EVICT_IMMEDIATE if mode == "immediate" else dms.DMS_EVICT_DELAYED)
        self.cache = dms.DmsCache(self.cfg)
        for p in self.cache.pools:
            p.fill_(0xFF)
        self.cache.workspace.fill_(0xFF)
        dms.dms_init_state(self.cache.ctx)
        self.orc = PagedKVOracle(S, H, w, P, pages, maxp, d, mode=mode, kv_format=fmt)
        self.inputs, self.seed, self.fmt, self.budget = {}, seed, fmt, budget

    def fill(self, seqs, lens, p=0.75):
        for s, n in zip(seqs, lens):
            self.inputs[s] = SeqInputs(self.seed, 0, s, n + 40, self.H, self.g, self.d, p)
        cat = lambda name: np.concatenate([getattr(self.inputs[s], name)[:n] for s, n in zip(seqs, lens)])
        cu = np.concatenate([[0], np.cumsum(lens)]).astype(np.int32)
        for y in range(self.cfg.num_layers):
            self.dms.dms_append_chunk(self.cache.ctx, y, len(seqs), to_dev(np.array(seqs, np.int32)), to_dev(cu),
                                      int(cu[-1]), int(max(lens)), to_dev(cat("k")), to_dev(cat("v")), to_dev(cat("flags")))
        self.orc.append_chunk(seqs, [self.inputs[s].flags[:n] for s, n in zip(seqs, lens)],
                              [bf16_to_f32(self.inputs[s].k[:n]) for s, n in zip(seqs, lens)],
                              [bf16_to_f32(self.inputs[s].v[:n]) for s, n in zip(seqs, lens)])

    def fork(self, src, dst, layer=-1):
        self.dms.dms_seq_fork(self.cache.ctx, layer, len(src), to_dev(np.array(src, np.int32)), to_dev(np.array(dst, np.int32)))
        self.orc.seq_fork(src, dst)
        for s, d in zip(src, dst):
            if s in self.inputs:
                self.inputs[d] = self.inputs[s]

    def reset(self, seqs):
        self.dms.dms_seq_reset(self.cache.ctx, -1, len(seqs), to_dev(np.array(seqs, np.int32)))
        self.orc.seq_reset(seqs)
        for s in seqs:
            self.inputs.pop(s, None)

    def compact(self):
        import torch
        used = torch.full((self.cfg.num_layers,), -1, dtype=torch.int32, device="cuda")
        self.dms.dms_compact(self.cache.ctx, -1, used)
        assert (used.cpu().numpy() == self.orc.compact()).all()

    def step(self, seqs, at):
        """Each sequence appends the token of position pos that input `at[s]` gives, and attends."""
        import torch
        pos = [int(self.orc.pos[s]) for s in seqs]
        pick = lambda name: np.stack([getattr(self.inputs[s], name)[p + a] for s, p, a in zip(seqs, pos, at)])
        q, k, v, f = (pick(n) for n in ("q", "k", "v", "flags"))
        out = torch.empty((len(seqs), self.H * self.g, self.d), device="cuda")
        for y in range(self.cfg.num_layers):
            out.fill_(float("nan"))
            self.dms.dms_decode_step(self.cache.ctx, y, len(seqs), to_dev(np.array(seqs, np.int32)), to_dev(q), to_dev(k),
                                     to_dev(v), to_dev(f), out)
        torch.cuda.synchronize()
        self.orc.append(seqs, f, bf16_to_f32(k), bf16_to_f32(v))
        if not self.budget:
            ref = self.orc.decode(seqs, bf16_to_f32(q), self.g)
            assert np.abs(out.cpu().numpy() - ref).max() <= ATOL

    def check(self, pool=True):
        import torch
        torch.cuda.synchronize()
        assert self.dms.dms_status(self.cache.ctx) == 0
        seqs = list(range(self.cfg.max_seqs))
        for y in range(self.cfg.num_layers):
            view = self.cache.export(y)
            compare_state(view, self.orc, seqs)
            if pool and self.fmt == "bf16":
                compare_pool(self.cache, y, view, [s for s in seqs if s in self.inputs], self.inputs)
            elif pool:
                compare_pool_fp8(self.cache, self.orc, [s for s in seqs if s in self.inputs], y)
            if self.budget:
                self.check_bounds(view, y)
        return view

    def check_bounds(self, view, y):
        """Channel-wise bounds of every live page against the keys stored in it."""
        import torch
        o, D, P = self.cache.offsets, self.d, self.cfg.page_size
        at = o.layer0 + y * o.layer_stride + o.page_bounds
        raw = self.cache.meta[at:at + self.cfg.num_pages * 4 * D].cpu().numpy().view(np.uint16)
        b = bf16_to_f32(raw.reshape(-1, 2, D))
        for s in range(self.cfg.max_seqs):
            for h in range(self.H):
                L = int(view.L[s, h])
                for i in range(-(-L // P)):
                    keys = self.orc.k_store[s, h, i * P:min(L, (i + 1) * P)]
                    pg = view.page_table[s, h, i]
                    assert np.array_equal(b[pg, 0], keys.min(0)) and np.array_equal(b[pg, 1], keys.max(0))


@pytest.mark.parametrize("fmt,P,d,budget", [("bf16", 64, 128, 0), ("fp8", 32, 64, 0), ("bf16", 256, 64, 2), ("fp8", 128, 128, 2)])
def test_chains_of_two_prompts(fmt, P, d, budget):
    """Prompts forked into chains that decode on their own ways, a release, a fork of a chain, compaction."""
    r = _Run(14, 2, 3, d, 16, P, 200, 8, fmt, layers=2, budget=budget)
    r.fill([3, 9], [333, 70])
    r.fork([3, 3, 3, 9, 3, 3], [0, 13, 5, 1, 2, 7])
    r.check()
    r.step([0, 13, 5, 1], [0, 0, 0, 0])
    r.step([13, 0, 3], [1, 0, 2])
    r.check(pool=False)
    r.reset([3, 5])
    r.fork([13, 0], [4, 10])
    r.check(pool=False)
    r.compact()
    r.check(pool=False)
    r.step([4, 13, 10, 1], [0, 1, 0, 0])
    r.fork([9], [5])
    r.compact()
    r.check(pool=False)


def test_empty_sources_window_of_one_and_immediate_eviction():
    r = _Run(6, 3, 1, 64, 1, 32, 60, 6, mode="immediate")
    r.fill([2], [90], p=0.5)
    r.fork([1, 2, 0], [3, 4, 5])       # sequences 0 and 1 hold nothing
    view = r.check()
    assert view.pos[3] == 0 and view.pos[4] == 90
    r.step([4, 2], [0, 0])
    r.reset([2])
    r.compact()
    r.check(pool=False)
    r.compact()                        # already compact: nothing moves
    r.check(pool=False)


def test_a_full_pool_forks_and_compacts():
    """Every page in use after the fork; compaction of a full and of an empty pool."""
    probe = _Run(5, 2, 2, 64, 8, 32, 100, 10)
    probe.compact()
    probe.fill([0], [200])
    held = 100 - probe.orc.top
    r = _Run(5, 2, 2, 64, 8, 32, 4 * held, 10)
    r.fill([0], [200])
    r.fork([0, 0, 0], [2, 1, 4])
    assert r.orc.top == 0
    r.compact()
    r.check()


def test_latent_rows_and_pages_of_many_sizes():
    """Latent rows: copies hold the source's rows; outputs equal the source's bit for bit."""
    import torch
    from paper_2506_05345_amd import dms
    for P in (32, 128):
        cfg = dms.make_config(1, 4, 1, 16, 576, 16, P, 64, 16, 1024, kv_format=dms.DMS_KV_MLA)
        c = dms.DmsCache(cfg)
        c.pools[0].fill_(0xFF)
        rng = np.random.default_rng(P)
        T = 300
        rows = torch.from_numpy(rng.normal(size=(T, 1, 576)).astype(np.float32)).cuda().bfloat16()
        flags = torch.from_numpy((rng.random((T, 1)) < 0.6).astype(np.uint8)).cuda()
        one = lambda *v: torch.tensor(v, dtype=torch.int32, device="cuda")
        dms.dms_append_chunk(c.ctx, 0, 1, one(2), one(0, T), T, T, rows, None, flags)
        dms.dms_seq_fork(c.ctx, 0, 2, one(2, 2), one(0, 3))
        dms.dms_seq_reset(c.ctx, 0, 1, one(0))
        q = torch.from_numpy(rng.normal(size=(1, 16, 576)).astype(np.float32)).cuda().bfloat16()
        outs = [torch.empty((1, 16, 512), device="cuda") for _ in range(3)]
        dms.dms_decode(c.ctx, 0, 1, one(2), q, outs[0])
        dms.dms_decode(c.ctx, 0, 1, one(3), q, outs[1])
        used = one(0)
        dms.dms_compact(c.ctx, 0, used)
        dms.dms_decode(c.ctx, 0, 1, one(3), q, outs[2])
        torch.cuda.synchronize()
        assert dms.dms_status(c.ctx) == 0
        assert torch.equal(outs[0], outs[1]) and torch.equal(outs[0], outs[2])
        view = c.export(0)
        assert int(used) == 64 - view.top == 2 * -(-int(view.L[2, 0]) // P)
        for i in range(-(-int(view.L[2, 0]) // P)):
            n = min(P, int(view.L[2, 0]) - i * P)
            a, b = (c.pool_page_kv(0, view.page_table[s, 0, i])[0][:n] for s in (2, 3))
            assert np.array_equal(a, b)
        c.close()


def test_refusals_change_no_layer():
    import torch
    from paper_2506_05345_amd import dms
    r = _Run(6, 2, 2, 64, 8, 32, 12, 10, layers=3)
    r.fill([0, 1], [150, 40])
    one = lambda v: to_dev(np.array(v, np.int32))
    r.dms.dms_seq_fork(r.cache.ctx, 1, 1, one([1]), one([5]))      # layer 1 alone
    torch.cuda.synchronize()
    state = r.cache.meta[256:].clone()
    pools = [p.clone() for p in r.cache.pools]
    cases = [([0], [6], dms.DMS_ERR_BAD_SEQ), ([-1], [3], dms.DMS_ERR_BAD_SEQ), ([0, 0], [3, 3], dms.DMS_ERR_BAD_SEQ),
             ([0], [1], dms.DMS_ERR_BAD_SEQ), ([2, 0], [3, 2], dms.DMS_ERR_BAD_SEQ),
             ([0, 1], [4, 5], dms.DMS_ERR_BAD_SEQ),                # 5 is empty in two layers of three
             ([0, 0, 0, 0], [2, 3, 4, 2], dms.DMS_ERR_BAD_SEQ), ([0, 0, 0], [2, 3, 4], dms.DMS_ERR_OUT_OF_PAGES)]
    for src, dst, code in cases:
        dms.dms_seq_fork(r.cache.ctx, -1, len(src), one(src), one(dst))
        assert dms.dms_status(r.cache.ctx) == code, (src, dst)
        # later calls do nothing until the status is cleared
        used = one([-7] * 3)
        dms.dms_compact(r.cache.ctx, -1, used)
        dms.dms_seq_fork(r.cache.ctx, -1, 1, one([1]), one([4]))
        torch.cuda.synchronize()
        assert (used == -7).all()
        assert torch.equal(r.cache.meta[256:], state) and all(torch.equal(a, b) for a, b in zip(r.cache.pools, pools))
        dms.dms_clear_status(r.cache.ctx)
    dms.dms_seq_fork(r.cache.ctx, 0, 1, one([1]), one([5]))        # empty in layer 0
    assert dms.dms_status(r.cache.ctx) == 0


def test_captured_release_and_fork_replays():
    """reset + fork + compact in a captured graph: every replay leaves the state of an eager run."""
    import torch
    r = _Run(7, 2, 2, 64, 16, 32, 120, 10, layers=2)
    e = _Run(7, 2, 2, 64, 16, 32, 120, 10, layers=2)
    for x in (r, e):
        x.fill([4, 1], [250, 100])
        x.fork([4, 1, 4], [0, 2, 6])
    dms = r.dms
    one = lambda v: to_dev(np.array(v, np.int32))
    src, dst, used = one([4, 1, 4]), one([0, 2, 6]), one([0, 0])

    def cycle(x):
        dms.dms_seq_reset(x.cache.ctx, -1, 3, dst)
        dms.dms_seq_fork(x.cache.ctx, -1, 3, src, dst)
        dms.dms_compact(x.cache.ctx, -1, used)

    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        cycle(r)
    for i in range(4):
        src.copy_(one([[4, 1, 4], [1, 1, 4], [4, 4, 4], [1, 1, 1]][i]))
        g.replay()
        torch.cuda.synchronize()
        cycle(e)
        torch.cuda.synchronize()
        for y in (0, 1):
            a, b = r.cache.export(y), e.cache.export(y)
            for f in ("pos", "L", "ring_slot", "ring_flag", "page_table", "stack"):
                assert np.array_equal(getattr(a, f), getattr(b, f)), (i, y, f)
        assert torch.ones(1000, device="cuda").sum().item() == 1000
        assert dms.dms_status(r.cache.ctx) == 0 and dms.dms_status(e.cache.ctx) == 0


def test_many_heads_and_layers():
    """More (pair, head) rows than a plan handles at once, more layers than one launch holds."""
    r = _Run(300, 5, 1, 64, 4, 32, 1700, 2)
    r.fill([7], [30])
    r.fork([7] * 299, [s for s in range(300) if s != 7])
    r.check(pool=False)
    r.reset([s for s in range(0, 300, 3)])
    r.compact()
    r.check(pool=False)
    m = _Run(3, 1, 2, 64, 4, 32, 8, 2, layers=67)
    m.fill([1], [40])
    m.fork([1], [2])
    m.reset([1])
    m.compact()
    m.step([2], [0])
    m.check(pool=False)
