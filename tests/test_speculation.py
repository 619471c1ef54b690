"""Speculative decoding over the cache: attention of drafted trees, choice of tokens,
accepted paths and commits together, against decoding token by token, eager and as a
captured graph; graphs that share a workspace, and calls on two streams."""
import numpy as np
import pytest

pytestmark = pytest.mark.gpu

PARENTS = [-1, 0, 0, 0, 1, 1, 2, 4, 6]       # of every tree: the last token, its continuations
RANKS = [0, 0, 1, 2, 0, 1, 0, 0, 0]          # a node's place among the likeliest followers of its parent


class Model:
    """Layers whose queries, keys, values and decisions follow from a token alone, so that both ways of decoding append the
    same rows; the logits add what the attention of every layer gives to a table of followers."""

    def __init__(self, seed, layers=2, H=2, g=2, d=64, vocab=500, w=8, kv=0, seqs=3):
        import torch
        from paper_2506_05345_amd import dms
        self.dms, self.torch = dms, torch
        rng = np.random.default_rng(seed)
        self.rng, self.layers, self.H, self.g, self.d, self.vocab, self.n = rng, layers, H, g, d, vocab, seqs
        P, S, maxp = 32, seqs + 1, 8
        self.cfg = dms.make_config(layers, S, H, g, d, w, P, S * H * maxp, maxp, 256, kv_format=kv)
        put = lambda x: torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda()
        self.q = [put(rng.normal(size=(vocab, H * g, d))).bfloat16() for _ in range(layers)]
        self.k = [put(rng.normal(size=(vocab, H, d))).bfloat16() for _ in range(layers)]
        self.v = [put(rng.normal(size=(vocab, H, d))).bfloat16() for _ in range(layers)]
        self.f = [torch.from_numpy((rng.random((vocab, H)) < 0.6).astype(np.uint8)).cuda() for _ in range(layers)]
        self.head = [put(rng.normal(size=(vocab, H * g * d)) * 0.02) for _ in range(layers)]
        table = rng.normal(size=(vocab, vocab)) + 7.0 * (rng.random((vocab, vocab)) < 3 / vocab)
        self.table = put(table)
        self.likely = torch.from_numpy(np.argsort(-table, axis=1)[:, :3].copy()).cuda()
        self.ids = torch.tensor(rng.permutation(S)[:seqs], dtype=torch.int32, device="cuda")
        self.sampling = dms.make_sample_config(vocab, temperature=0.7)
        m = len(PARENTS)
        self.cu = torch.arange(0, seqs * m + 1, m, dtype=torch.int32, device="cuda")
        self.parents = torch.tensor(PARENTS * seqs, dtype=torch.int32, device="cuda")
        depth = [0] * m
        for x, p in enumerate(PARENTS):
            depth[x] = 0 if p < 0 else depth[p] + 1
        self.depth = torch.tensor(depth, device="cuda")
        self.u = put(rng.random((seqs, 400)))
        self.prompt = rng.integers(0, vocab, (seqs, 30))

    def logits(self, tokens, outs):
        x = self.table[tokens]
        for head, o in zip(self.head, outs):
            x = x + (o.float().reshape(len(tokens), 1, -1) * head).sum(-1)
        return x

    def cache(self):
        torch, dms = self.torch, self.dms
        c = dms.DmsCache(self.cfg)
        t = torch.from_numpy(self.prompt.reshape(-1)).cuda()
        cu = torch.arange(0, t.numel() + 1, self.prompt.shape[1], dtype=torch.int32, device="cuda")
        for l in range(self.layers):
            dms.dms_append_chunk(c.ctx, l, self.n, self.ids, cu, t.numel(), self.prompt.shape[1], self.k[l][t].contiguous(),
                                 self.v[l][t].contiguous(), self.f[l][t].contiguous())
        return c


class Speculation:
    """State on the device between steps: the last token of every sequence and its position."""

    def __init__(self, model):
        torch, dms = model.torch, model.dms
        self.m, self.c = model, model.cache()
        n, T = model.n, model.n * len(PARENTS)
        self.last = torch.from_numpy(model.prompt[:, 0].astype(np.int32)).cuda()
        self.pos = torch.full((n,), model.prompt.shape[1], dtype=torch.int64, device="cuda")
        self.tokens = torch.zeros((n, len(PARENTS)), dtype=torch.int32, device="cuda")
        self.outs = [torch.zeros((T, model.H * model.g, model.d), dtype=torch.bfloat16, device="cuda") for _ in range(model.layers)]
        self.targets = torch.zeros(T, dtype=torch.int32, device="cuda")
        self.path, self.plen = torch.zeros_like(self.targets), torch.zeros(n, dtype=torch.int32, device="cuda")
        self.ws = torch.empty(dms.dms_tree_workspace(model.cfg, n, T, len(PARENTS)), dtype=torch.uint8, device="cuda")
        self.sws = torch.empty(dms.dms_sample_workspace(model.sampling, T), dtype=torch.uint8, device="cuda")

    def step(self):
        m, torch, dms, c = self.m, self.m.torch, self.m.dms, self.c
        n, M = m.n, len(PARENTS)
        T = n * M
        self.tokens[:, 0] = self.last
        for x in range(1, M):
            self.tokens[:, x] = m.likely[self.tokens[:, PARENTS[x]].long(), RANKS[x]].int()
        at = self.tokens.reshape(-1).long()
        rows = [[t[l].index_select(0, at) for t in (m.q, m.k, m.v, m.f)] for l in range(m.layers)]
        for l, (q, k, v, f) in enumerate(rows):
            dms.dms_tree_attention(c.ctx, l, n, m.ids, m.cu, T, M, m.parents, q, k, v, f, self.outs[l], self.ws)
        logits = m.logits(at, self.outs)
        u = torch.gather(m.u, 1, self.pos[:, None] + m.depth[None, :]).reshape(-1).contiguous()
        dms.dms_sample(m.sampling, T, logits, None, None, None, None, u, self.targets, None, self.sws)
        dms.dms_tree_accept(n, m.cu, T, M, m.parents, self.tokens, self.targets, self.last.clone(), self.path, self.plen, self.last)
        for l, (q, k, v, f) in enumerate(rows):
            dms.dms_tree_commit(c.ctx, l, n, m.ids, m.cu, T, M, self.path, self.plen, k, v, f, self.ws)
        self.pos += self.plen

    def state(self):
        return [x.clone() for x in (self.tokens, self.targets, self.path, self.plen, self.last, self.pos, *self.outs)]


def same_caches(m, a, b):
    for l in range(m.layers):
        x, y = a.export(l), b.export(l)
        assert np.array_equal(x.pos, y.pos) and np.array_equal(x.L, y.L)
        for s in m.ids.cpu().numpy():
            for h in range(m.H):
                L = int(x.L[s, h])
                assert np.array_equal(x.slot_pos[s, h, :L], y.slot_pos[s, h, :L])
                assert np.array_equal(x.slot_flag[s, h, :L], y.slot_flag[s, h, :L])


@pytest.mark.parametrize("kv", [0, 1], ids=["bf16", "fp8"])
def test_speculation_decodes_what_single_steps_do(kv):
    """Every accepted node against dms_decode_step of its token.  Outputs: both round weights to bf16, which moves a sum by at
    most 2^-8 / (1 - 2^-8) of the spread of the values, itself at most 2 max |v| (8-bit pages: and 2^-4 of the value more in
    both, the same stored one, so no more between them); the tree's are rounded to bf16 once: 5.1 2^-8 max |v| between them.
    Tokens: logits off by at most D move every border of the running probabilities by at most e^(2 D / T) - 1."""
    m = Model(11, kv=kv)
    torch, dms = m.torch, m.dms
    s, c = Speculation(m), m.cache()
    sws = torch.empty(dms.dms_sample_workspace(m.sampling, 1), dtype=torch.uint8, device="cuda")
    out = [torch.empty((1, m.H * m.g, m.d), device="cuda") for _ in range(m.layers)]
    token = torch.empty(1, dtype=torch.int32, device="cuda")
    most = 5.1 * 2.0 ** -8 * max(float(v.float().abs().max()) for v in m.v) * (1 + kv * 2.0 ** -4)
    committed = 0
    for _ in range(10):
        pos = s.pos.cpu().numpy().copy()
        s.step()
        assert dms.dms_status(s.c.ctx) == 0
        tokens, targets = s.tokens.cpu().numpy(), s.targets.cpu().numpy().reshape(m.n, -1)
        path, plen = s.path.cpu().numpy().reshape(m.n, -1), s.plen.cpu().numpy()
        nodes_logits = m.logits(s.tokens.reshape(-1).long(), s.outs).reshape(m.n, len(PARENTS), -1).double().cpu().numpy()
        assert (plen >= 1).all() and (path[:, 0] == 0).all()
        committed += int(plen.sum())
        for i in range(m.n):
            for z in range(plen[i]):
                x = path[i, z]
                t = torch.tensor([int(tokens[i, x])], device="cuda")
                for l in range(m.layers):
                    dms.dms_decode_step(c.ctx, l, 1, m.ids[i:i + 1], m.q[l][t], m.k[l][t], m.v[l][t], m.f[l][t], out[l])
                    diff = (out[l][0] - s.outs[l][i * len(PARENTS) + x].float()).abs().max()
                    assert float(diff) <= most
                logits = m.logits(t, out)
                u = m.u[i, pos[i] + z:pos[i] + z + 1].contiguous()
                dms.dms_sample(m.sampling, 1, logits, None, None, None, None, u, token, None, sws)
                one = logits[0].double().cpu().numpy()
                off = np.abs(one - nodes_logits[i, x]).max()
                e = np.exp((one - one.max()) / np.float32(0.7))
                F = np.concatenate([[0.0], np.cumsum(e) / e.sum()])
                for tok, eps in ((int(token), 1e-12), (int(targets[i, x]), 1e-12 + np.expm1(2 * off / np.float32(0.7)))):
                    assert F[tok] - eps <= float(u) <= F[tok + 1] + eps
                if z + 1 < plen[i]:
                    assert tokens[i, path[i, z + 1]] == targets[i, x]
            assert int(s.last[i]) == targets[i, path[i, plen[i] - 1]]
    assert committed > 10 * m.n      # some drafts were taken
    assert dms.dms_status(c.ctx) == 0
    same_caches(m, s.c, c)
    # and both caches answer alike
    q = torch.arange(m.n, device="cuda")
    got = [torch.empty((m.n, m.H * m.g, m.d), device="cuda") for _ in range(2)]
    for cache, o in zip((s.c, c), got):
        dms.dms_decode_step(cache.ctx, 0, m.n, m.ids, m.q[0][q], m.k[0][q], m.v[0][q], m.f[0][q], o)
    assert torch.equal(*got)


def test_a_captured_step_replays_as_it_runs():
    """One whole step as a graph; before each replay the same step runs eagerly over a second cache."""
    m = Model(12)
    torch, dms = m.torch, m.dms
    a, b = Speculation(m), Speculation(m)
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(stream):
        b.step()
    torch.cuda.current_stream().wait_stream(stream)
    a.step()
    for x, y in zip(a.state(), b.state()):
        assert torch.equal(x, y)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        b.step()
    for _ in range(8):
        a.step()
        torch.cuda.synchronize()
        b.ws.fill_(0xA5)             # contents of no meaning between calls
        b.sws.fill_(0x5A)
        graph.replay()
        for x, y in zip(a.state(), b.state()):
            assert torch.equal(x, y)
    assert dms.dms_status(a.c.ctx) == 0 and dms.dms_status(b.c.ctx) == 0
    same_caches(m, a.c, b.c)


def test_graphs_may_share_a_workspace_and_streams_may_not():
    """Two captured attentions of different sizes over one workspace, replayed in turn on one stream; and on two streams at
    once with a workspace each."""
    from test_tree import Call
    import torch
    x = Call(31, [900, 40], [50, 31], 2, 3, 128, 64, 64)
    y = Call(32, [333], [7], 1, 2, 64, 16, 32)
    tx, ty = x.tensors(), y.tensors()
    wx, wy = x.attend(tx), y.attend(ty)
    own = y.ws
    y.ws = x.ws
    ox, oy = torch.zeros_like(wx), torch.zeros_like(wy)
    graphs = []
    for c, t, o in ((x, tx, ox), (y, ty, oy)):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g):
            c.attend(t, o)
        graphs.append(g)
    for _ in range(4):
        ox.zero_(), oy.zero_()
        for g in graphs:
            g.replay()
        torch.cuda.synchronize()
        assert torch.equal(ox, wx) and torch.equal(oy, wy)
    y.ws = own
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(4):
        ox.zero_(), oy.zero_()
        torch.cuda.synchronize()
        for _ in range(5):
            x.attend(tx, ox, stream=streams[0])
            y.attend(ty, oy, stream=streams[1])
        torch.cuda.synchronize()
        assert torch.equal(ox, wx) and torch.equal(oy, wy)


def test_sampling_of_a_graph_reads_what_its_tensors_hold():
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(33)
    c = dms.make_sample_config(20000)
    rows = 7
    logits, u = torch.empty((rows, 20000), device="cuda"), torch.empty(rows, device="cuda")
    T, p = torch.empty(rows, device="cuda"), torch.empty(rows, device="cuda")
    k = torch.empty(rows, dtype=torch.int32, device="cuda")
    tokens, logp = torch.empty(rows, dtype=torch.int32, device="cuda"), torch.empty(rows, device="cuda")
    ws = torch.empty(dms.dms_sample_workspace(c, rows), dtype=torch.uint8, device="cuda")
    call = lambda tok, lp: dms.dms_sample(c, rows, logits, T, k, p, None, u, tok, lp, ws)

    def fill():
        for t, v in ((logits, rng.normal(size=(rows, 20000)) * rng.choice([0.1, 1, 5], (rows, 1))), (u, rng.random(rows)),
                     (T, rng.choice([0.0, 0.5, 1.0], rows)), (p, rng.choice([0.3, 0.9, 1.0], rows))):
            t.copy_(torch.from_numpy(v.astype(np.float32)))
        k.copy_(torch.from_numpy(rng.choice([0, 1, 50, 3000], rows).astype(np.int32)))

    fill()
    call(tokens, logp)
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call(tokens, logp)
    want_t, want_p = torch.empty_like(tokens), torch.empty_like(logp)
    for _ in range(6):
        fill()
        call(want_t, want_p)
        ws.random_(0, 256)
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(tokens, want_t) and torch.equal(logp, want_p)
