"""Performance cases of the operators that draft, check and choose tokens around the DMS cache.

Four kinds of call, each in a plain form (elementary torch operations) and, where
``own`` is true, as a program calls the library:

* ``tree``: attention of trees of drafted tokens over the paged cache and over
  their own ancestors, nothing appended (``dms_tree_attention``);
* ``commit``: the accepted path of every sequence's tree appended to the cache,
  in every layer of a call, from restored positions, lengths, rings and stacks
  (``dms_tree_commit``);
* ``accept``: the longest path of drafted tokens that agree with the tokens
  chosen for their predecessors (``dms_tree_accept``);
* ``sample``: one token per row of logits, with temperature, top-k, top-p and
  min-p, from given random numbers (``dms_sample``).

Layer shapes are those of the benchmark and of the tests: (KV heads, group,
head dim) of the 1.5B, 7B, 8B and 32B attention layers, latent rows, and a tiny
layer of 64 dims; vocabularies are theirs too.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
SHAPES = {"tiny": (2, 2, 64), "1.5b": (2, 6, 128), "7b": (4, 7, 128), "8b": (8, 4, 128),
          "32b": (8, 5, 128), "mla16": (1, 16, 576)}
PAGE = 64            # tokens of a cache page
TPP = PAGE // 32     # tiles of a page
TILE_BYTES = {"bf16": lambda d: 128 * d, "fp8": lambda d: 64 * d + 256, "mla": lambda d: 64 * d}
UNIT = 2.0 ** 43     # a sampling weight is a multiple of 1 / UNIT of the largest one


def _tree(shape, context, seqs, nodes, low=1.0, branch=True, ragged=False, window=256, evict=0.875, kv="bf16"):
    return {"kind": "tree", "shape": shape, "context": context, "seqs": seqs, "nodes": nodes, "low": low,
            "branch": branch, "ragged": ragged, "window": window, "evict": evict, "kv": kv, "layers": 1}


def _commit(shape, context, seqs, nodes, layers, low=1.0, ragged=False, window=256, evict=0.875, kv="bf16"):
    return {"kind": "commit", "shape": shape, "context": context, "seqs": seqs, "nodes": nodes, "low": low,
            "branch": True, "ragged": ragged, "window": window, "evict": evict, "kv": kv, "layers": layers}


def _accept(seqs, nodes, branch=True, ragged=False):
    return {"kind": "accept", "seqs": seqs, "nodes": nodes, "branch": branch, "ragged": ragged}


def _sample(rows, vocab, dtype="f32", temperature=0.6, top_k=0, top_p=1.0, min_p=0.0, mixed=False, spread=3.0):
    return {"kind": "sample", "rows": rows, "vocab": vocab, "dtype": dtype, "temperature": temperature,
            "top_k": top_k, "top_p": top_p, "min_p": min_p, "mixed": mixed, "spread": spread}


def listed():
    return [
        # a chain of four drafted tokens behind a short sequence of a small layer: a launch's latency
        dict(_tree("tiny", 300, 1, 4, branch=False, window=16), name="tree-tiny"),
        # eight chains of a small model, each checking a tree of 16 drafted tokens
        dict(_tree("1.5b", 32768, 8, 16, low=0.1), name="tree-1.5b"),
        # ragged trees of up to 33 nodes over a cache of 8-bit pages
        dict(_tree("7b", 24000, 5, 33, low=0.05, ragged=True, kv="fp8"), name="tree-7b-fp8-ragged"),
        # 48 chains at 32K tokens with short trees: the cache is read once for 60 columns
        dict(_tree("32b", 32768, 48, 12), name="tree-32b"),
        # large trees, 320 columns of each KV head: matrix products
        dict(_tree("32b", 32768, 8, 64), name="tree-32b-wide"),
        # the accepted paths of eight sequences, every layer of a small model
        dict(_commit("1.5b", 2000, 8, 16, 28), name="commit-1.5b"),
        # 64 sequences of the largest layer, two layers
        dict(_commit("32b", 16384, 64, 24, 2, low=0.5, ragged=True), name="commit-32b"),
        # one sequence's tree
        dict(_accept(1, 16), name="accept-1"),
        # a large batch of large trees
        dict(_accept(512, 128, ragged=True), name="accept-512"),
        # one row at the usual settings of a reasoning model: latency
        dict(_sample(1, 151936, top_p=0.95), name="sample-1"),
        # 128 chains, the settings of the benchmark's workload
        dict(_sample(128, 152064, top_p=0.95), name="sample-128"),
        # the rows of drafted trees, a setting of each row's own, bf16 logits
        dict(_sample(500, 151936, dtype="bf16", mixed=True), name="sample-tree-rows"),
    ]


def _log_int(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    kind = rng.choice(["tree", "tree", "tree", "commit", "accept", "sample", "sample"])
    if kind == "accept":
        return _accept(_log_int(rng, 1, 512), _log_int(rng, 1, 128), rng.random() < 0.7, rng.random() < 0.5)
    if kind == "sample":
        vocab = _log_int(rng, 2, 262144)
        rows = _log_int(rng, 1, min(500, 1 + 70000000 // vocab))
        how = rng.choice(["plain", "k", "p", "min", "all", "mixed"])
        return _sample(rows, vocab, rng.choice(["f32", "bf16"]), rng.choice([0.0, 0.3, 0.6, 0.8, 1.0, 1.7]),
                       rng.choice([1, 5, 20, 50, 400]) if how in ("k", "all") else 0,
                       rng.choice([0.3, 0.8, 0.95, 0.99]) if how in ("p", "all") else 1.0,
                       rng.choice([0.01, 0.05, 0.2]) if how in ("min", "all") else 0.0,
                       how == "mixed", rng.choice([0.5, 2.0, 3.0, 5.0]))
    window = rng.choice([4, 16, 64, 256])
    evict = rng.choice([0.5, 0.75, 0.875])
    context = _log_int(rng, 1, 32768)
    low, ragged = rng.uniform(0.02, 1.0), rng.random() < 0.5
    if kind == "commit":
        shape = rng.choice(["tiny", "1.5b", "7b", "8b", "32b", "mla16"])
        seqs, nodes = _log_int(rng, 1, 64), _log_int(rng, 1, 64)
        while seqs * context > 600000:
            context = context // 2
        layers = rng.choice([1, 2, 7]) if seqs * context < 100000 else 1
        return _commit(shape, context, seqs, nodes, layers, low, ragged, window, evict,
                       "mla" if shape == "mla16" else "bf16")
    shape = rng.choice(["tiny", "1.5b", "7b", "8b", "32b"])
    H, g, _ = SHAPES[shape]
    seqs, nodes = _log_int(rng, 1, 48), _log_int(rng, 1, 128)
    kept = min(context, window) + max(0, context - window) * (1 - evict)
    while seqs * H * (kept + nodes) * max(64, nodes * g) > 1.0e8 or seqs * H * kept > 1200000:
        seqs = max(1, seqs * 3 // 4)
        nodes = max(1, nodes * 4 // 5)
        context = context * 4 // 5 + 1
        kept = min(context, window) + max(0, context - window) * (1 - evict)
    return _tree(shape, context, seqs, nodes, low, rng.random() < 0.7, ragged, window, evict,
                 rng.choice(["bf16", "bf16", "fp8"]))


# ---------------------------------------------------------------------------
# Inputs
# ---------------------------------------------------------------------------

def _gen(seed, *ids):
    x = int(seed) + 1
    for i in ids:
        x = (x * 0x9E3779B1 + int(i) + 0x7F4A7C15) % (1 << 62)
    g = torch.Generator(device=DEV)
    g.manual_seed(x)
    return g


def _normal(gen, shape, dtype, scale=1.0):
    return (torch.randn(shape, generator=gen, device=DEV) * scale).to(dtype)


def _i32(a):
    return torch.as_tensor(np.ascontiguousarray(a), dtype=torch.int32, device=DEV)


def _dms():
    from paper_2506_05345_amd import dms
    return dms


def _trees(case, rng):
    """Node counts of the sequences (ragged: from 1 to the most, mixed) and every node's parent inside its tree (-1: the
    root, node 0).  A tree is a chain, or every node follows a random one of the last few."""
    i = np.arange(case["seqs"])
    m = case["nodes"] - ((case["nodes"] * (i * 0.6180339887498949 % 1.0)).astype(np.int64) if case["ragged"] else 0 * i)
    parents = []
    for k in m:
        x = np.arange(k)
        back = 1 + rng.integers(0, 1 + np.minimum(x, 8)) if case["branch"] else 1
        parents.append(np.maximum(x - back, np.where(x > 0, 0, -1)))
    return m, parents


def _shares(case):
    """Contexts of the sequences, from `low` of the longest to the longest."""
    n = case["seqs"]
    share = np.array([1.0 if n == 1 else case["low"] + (1 - case["low"]) * i / (n - 1) for i in range(n)])
    step = next(x for x in (7, 5, 3, 1) if math.gcd(x, n) == 1)
    return np.maximum(1, (case["context"] * share[(np.arange(n) * step) % n]).astype(np.int64))


def _most(case):
    """The most tokens that a head retains before the call, and the pages of its table (room for the tree too)."""
    most = min(case["context"], case["window"]) + \
        int(max(0, case["context"] - case["window"]) * min(1.0, 1.4 * (1 - case["evict"]))) + 1
    return most, -(-(most + case["nodes"]) // PAGE)


class _Context:
    """A context handle that is destroyed with the state that holds it."""

    def __init__(self, dms, handle):
        self.dms, self.handle = dms, handle

    def __del__(self):
        self.dms.dms_destroy(self.handle)


def _prepare_cache(case, seed):
    """The state arrays of every layer and its pool, as the library documents them: each head retains the last
    `window` tokens and a share of its own of the older ones, the recent tokens mostly in its later slots; pages lie
    scattered over the pool.  Sequence i of the call is sequence S - 1 - i of the cache."""
    H, g, d = SHAPES[case["shape"]]
    S, w, Ly = case["seqs"], case["window"], case["layers"]
    tile = TILE_BYTES[case["kv"]](d)
    most, maxp = _most(case)
    pages = S * H * maxp + 8
    rng = np.random.default_rng(seed)
    gen = _gen(seed, 1)
    m, parents = _trees(case, rng)
    pos = _shares(case)[::-1].copy()
    old = np.maximum(0, pos - w)[None, :, None]
    kept = np.minimum((old * np.minimum(1, (1 - case["evict"]) * rng.uniform(0.6, 1.4, (Ly, S, H)))).astype(np.int64),
                      np.maximum(0, most - np.minimum(pos, w))[None, :, None])
    recent = torch.as_tensor(np.broadcast_to(np.minimum(pos, w)[None, :, None], kept.shape).copy(), device=DEV)
    kept, posd = torch.as_tensor(kept, device=DEV), torch.as_tensor(pos, device=DEV)
    length = kept + recent
    Lmax = int(length.max())
    slot = torch.arange(Lmax, device=DEV)
    rand = lambda *shape: torch.rand(shape, generator=gen, device=DEV).clamp(min=1e-7)
    # slots of the last w tokens, and the rank of every slot among them and among the others
    key = slot / w - torch.log(-torch.log(rand(Ly, S, H, Lmax)))
    key = torch.where(slot < length[..., None], key, -math.inf)
    order = key.argsort(-1, descending=True)
    place = torch.empty_like(order).scatter_(-1, order, slot.expand_as(order).contiguous())
    new = place < recent[..., None]
    rank_old = (~new).cumsum(-1) - 1
    oldd = torch.as_tensor(old, device=DEV)[..., None]
    p_old = ((rank_old + rand(Ly, S, H, Lmax) * 0.999) * oldd / kept[..., None].clamp(min=1)).long()
    p_new = posd[None, :, None, None] - 1 - place
    flag = (torch.rand((Ly, S, H, Lmax), generator=gen, device=DEV) < case["evict"]) & new
    at = torch.where(new, p_new, torch.minimum(p_old, (oldd - 1).clamp(min=0)))
    meta = torch.zeros((Ly, S, H, maxp * PAGE), dtype=torch.int32, device=DEV)
    top_bit = -(1 << 31)
    meta[..., :Lmax] = torch.where(slot < length[..., None], at.int() | torch.where(flag, top_bit, 0).int(), 0)
    ring = torch.zeros((Ly, S, H, w + 1), dtype=torch.int64, device=DEV)
    ring.scatter_(-1, torch.where(new, at % w, w), torch.where(flag, slot + top_bit, slot))
    # page tables: scattered pages
    count = -(-length // PAGE)
    mine = torch.arange(maxp, device=DEV) < count[..., None]
    table = torch.full((Ly, S, H, maxp), -1, dtype=torch.int32, device=DEV)
    stack = torch.zeros((Ly, pages), dtype=torch.int32, device=DEV)
    top = torch.zeros((Ly, 1), dtype=torch.int32, device=DEV)
    for y in range(Ly):
        perm = torch.randperm(pages, generator=gen, device=DEV).int()
        used = int(mine[y].sum())
        table[y][mine[y]] = perm[:used]
        stack[y, :pages - used] = perm[used:]
        top[y] = pages - used
    t = {"pos": posd.int().expand(Ly, S).contiguous(), "len": length.int(), "ring": ring[..., :w].int().contiguous(),
         "page_table": table, "slot_meta": meta, "stack": stack, "top": top}
    # one page more than the cache has: the plain form's place for rows that are not there
    shape = (Ly, (pages + 1) * TPP, tile)
    if case["kv"] == "fp8":
        pool = torch.empty(shape, dtype=torch.uint8, device=DEV)
        codes = torch.randn((Ly, (pages + 1) * TPP, 64 * d), generator=gen, device=DEV, dtype=torch.bfloat16) * 110
        pool[..., :64 * d] = codes.clamp(-448, 448).to(torch.float8_e4m3fn).view(torch.uint8)
        scales = torch.exp2(torch.randint(-8, -5, (Ly, (pages + 1) * TPP, 64), generator=gen, device=DEV).float())
        pool[..., 64 * d:] = scales.view(torch.uint8)
    else:
        pool = torch.randn((Ly, (pages + 1) * TPP, tile // 2), generator=gen, device=DEV, dtype=torch.bfloat16).view(torch.uint8)
    total = int(m.sum())
    s = {"case": case, "pool": pool, "pages": pages, "Lmax": Lmax, "m": m, "total": total,
         "cu": _i32(np.concatenate([[0], np.cumsum(m)])), "parents": _i32(np.concatenate(parents)),
         "ids": _i32(np.arange(S)[::-1].copy()), "mmax": int(m.max())}
    bf = torch.bfloat16
    s["k"], s["v"] = _normal(gen, (Ly, total, H, d), bf), _normal(gen, (Ly, total, H, d), bf)
    s["flags"] = (torch.rand((Ly, total, H), generator=gen, device=DEV) < case["evict"]).to(torch.uint8)
    if case["kind"] == "tree":
        s["q"] = _normal(gen, (total, H * g, d), bf, 2.0)
        s["out"] = torch.empty((total, H * g, d), dtype=bf, device=DEV)
    else:
        # accepted paths: from the root to a node of the tree
        path, lens = np.full(total, -1), []
        a = 0
        for k, par in zip(m, parents):
            x, line = int(rng.integers(0, k)), []
            while x >= 0:
                line.append(x)
                x = int(par[x])
            line = line[::-1][:int(rng.integers(0, len(line) + 1))] if rng.random() < 0.3 else line[::-1]
            path[a:a + len(line)] = line
            lens.append(len(line))
            a += k
        s["path"], s["path_len"], s["longest"] = _i32(path), _i32(lens), max(lens)
    if own:
        dms = _dms()
        cfg = dms.make_config(Ly, S, H, g, d, w, PAGE, pages, maxp, kv_format={"bf16": 0, "fp8": 1, "mla": 2}[case["kv"]])
        meta_bytes, pool_bytes, ws_bytes, _ = dms.dms_layout(cfg)
        o = dms.dms_state_layout(cfg)
        assert pool_bytes + TPP * tile == pool[0].numel()
        buf = torch.zeros(meta_bytes, dtype=torch.uint8, device=DEV)
        s["cache_ws"] = torch.zeros(max(1, ws_bytes), dtype=torch.uint8, device=DEV)
        s["meta"] = buf
        s["ctx"] = _Context(dms, dms.dms_create(cfg, buf, [pool[y] for y in range(Ly)], s["cache_ws"]))
        dms.dms_init_state(s["ctx"].handle)
        s["ws"] = torch.empty(dms.dms_tree_workspace(cfg, S, total, s["mmax"]), dtype=torch.uint8, device=DEV)
        layers = buf[o.layer0:o.layer0 + Ly * o.layer_stride].view(Ly, o.layer_stride)
        for name, x in t.items():
            off, size = getattr(o, name), x[0].numel() * 4
            s[name] = layers[:, off:off + size].view(torch.int32).unflatten(1, x.shape[1:])
            s[name].copy_(x)
        if case["kind"] == "commit":    # positions, lengths and rings lie together
            s["front"] = layers[:, o.pos:o.page_table]
            s["saved"] = (s["front"].clone(), t["top"].clone())
    else:
        s.update(t)
        if case["kind"] == "commit":
            s["saved"] = tuple(t[x].clone() for x in ("pos", "len", "ring", "top"))
    return s


# ---------------------------------------------------------------------------
# Pages in their plain form
# ---------------------------------------------------------------------------

def _offsets(case):
    """Places of key and value element (row j, dim e) inside a tile: in 2-byte elements, for 8-bit pages in bytes."""
    _, _, d = SHAPES[case["shape"]]
    j, e = torch.arange(32, device=DEV)[:, None], torch.arange(d, device=DEV)
    h, r = (j // 4) % 2, 4 * (j // 8) + j % 4
    if case["kv"] == "fp8":
        return ((e // 64) * 2048 + h * 1024 + (16 * ((e // 8) % 4) + r) * 16 + 8 * ((e // 32) % 2) + e % 8,
                32 * d + (e // 32) * 1024 + (16 * (j // 8) + e % 16) * 16 + 8 * ((e // 16) % 2) + j % 8)
    return ((((e // 32) * 2 + h) * 4 + (e // 8) % 4) * 16 + r) * 8 + e % 8, \
        32 * d + (((e // 16) * 4 + j // 8) * 16 + e % 16) * 8 + j % 8


def _rows(s):
    """Keys and values of every slot of the pool, float32 [slots, d]."""
    case = s["case"]
    _, _, d = SHAPES[case["shape"]]
    ko, vo = _offsets(case)
    pool = s["pool"][0]
    if case["kv"] == "fp8":
        codes = pool[:, :64 * d].contiguous().view(torch.float8_e4m3fn).float()
        scale = pool[:, 64 * d:].contiguous().view(torch.float32).view(-1, 4, 2, 8)
        ks, vs = scale[:, :, 0].reshape(-1, 32, 1), scale[:, :, 1].reshape(-1, 32, 1)
        return (codes[:, ko] * ks).view(-1, d), (codes[:, vo] * vs).view(-1, d)
    x = pool.view(torch.bfloat16)
    return x[:, ko].float().view(-1, d), x[:, vo].float().view(-1, d)


def _stored(x, kv):
    """Rows of drafted tokens as the cache would hold them (8-bit pages: codes times a power of two)."""
    x = x.float()
    if kv != "fp8":
        return x
    mant, e = torch.frexp(x.abs().amax(-1, keepdim=True))
    e = torch.where(mant <= 0.875, e - 9, e - 8)
    scale = torch.where(mant > 0, torch.exp2(e.float()), 1.0)
    return (x / scale).to(torch.float8_e4m3fn).float() * scale


# ---------------------------------------------------------------------------
# Trees of drafted tokens
# ---------------------------------------------------------------------------

def _padded(s):
    """[n, mmax]: token row of every node (nodes that are not there: row 0) and whether it is there; its depth; which
    nodes are its ancestors or itself [n, mmax, mmax]."""
    n, M = s["case"]["seqs"], s["mmax"]
    cu = s["cu"].long()
    x = torch.arange(M, device=DEV)
    there = x < (cu[1:] - cu[:-1])[:, None]
    row = torch.where(there, cu[:-1, None] + x, 0)
    par = torch.where(there, s["parents"].long()[row], -1)
    line = torch.zeros((n, M, M), dtype=torch.bool, device=DEV)
    depth = torch.zeros((n, M), dtype=torch.long, device=DEV)
    i = torch.arange(n, device=DEV)
    for a in range(M):
        up = par[:, a]
        has = up >= 0
        line[:, a] = line[i, up.clamp(min=0)] & has[:, None]
        line[:, a, a] = True
        depth[:, a] = torch.where(has, depth[i, up.clamp(min=0)] + 1, 0)
    return row, there, depth, line


def _run_tree(s):
    case = s["case"]
    if own:
        _dms().dms_tree_attention(s["ctx"].handle, 0, case["seqs"], s["ids"], s["cu"], s["total"], s["mmax"], s["parents"],
                                  s["q"], s["k"], s["v"], s["flags"], s["out"], s["ws"])
        return {"out": s["out"]}
    H, g, d = SHAPES[case["shape"]]
    n, w, M, L = case["seqs"], case["window"], s["mmax"], s["Lmax"]
    row, there, depth, line = _padded(s)
    ids = s["ids"].long()
    slot = torch.arange(L, device=DEV)
    length = s["len"][0, ids].long()                                               # [n, H]
    page = s["page_table"][0, ids][..., slot // PAGE].clamp(min=0).long()          # [n, H, L]
    at = page * PAGE + slot % PAGE
    pool_k, pool_v = _rows(s)
    own_k = _stored(s["k"][0], case["kv"])[row].permute(0, 2, 1, 3)                # [n, H, M, d]
    own_v = _stored(s["v"][0], case["kv"])[row].permute(0, 2, 1, 3)
    k = torch.cat([pool_k[at], own_k], 2).reshape(n * H, L + M, d)
    v = torch.cat([pool_v[at], own_v], 2).reshape(n * H, L + M, d)
    meta = s["slot_meta"][0, ids][..., :L]
    held, flagged = (meta & 0x7FFFFFFF).long(), meta < 0
    t = s["pos"][0, ids].long()[:, None] + depth                                   # [n, M]
    see = (slot < length[..., None])[:, :, None] & ~(flagged[:, :, None] & (held[:, :, None] <= t[:, None, :, None] - w))
    flag = s["flags"][0][row].bool().permute(0, 2, 1)                              # [n, H, M]
    far = t[:, :, None] - t[:, None] >= w                                          # node behind ancestor
    see_own = line[:, None] & ~(far[:, None] & flag[:, :, None])
    see = torch.cat([see, see_own.expand(n, H, M, M)], -1)[:, :, :, None].expand(n, H, M, g, L + M).reshape(n * H, M * g, L + M)
    q = s["q"].float()[row].view(n, M, H, g, d).permute(0, 2, 1, 3, 4).reshape(n * H, M * g, d)
    p = (q @ k.transpose(-1, -2) / math.sqrt(d)).masked_fill_(~see, torch.finfo(torch.float32).min)
    p = (p - p.amax(-1, keepdim=True)).exp_() * see
    out = (p @ v) / p.sum(-1, keepdim=True)
    out = out.view(n, H, M, g, d).permute(0, 2, 1, 3, 4).reshape(n, M, H * g, d)
    s["out"][row[there]] = out[there].to(torch.bfloat16)
    return {"out": s["out"]}


def _exact_tree(case, seed):
    """Dense attention of one sequence and KV head at a time, tiles unfolded by their axes."""
    s = _prepare_cache(case, seed)
    H, g, d = SHAPES[case["shape"]]
    w, par = case["window"], s["parents"].tolist()
    out = torch.zeros((s["total"], H * g, d), dtype=torch.float64, device=DEV)

    def tile_rows(tiles):                                   # [x, bytes] -> keys, values [32 x, d]
        if case["kv"] == "fp8":
            c = tiles[:, :64 * d].contiguous().view(torch.float8_e4m3fn).double()
            # keys [d/64][h][G][r / 4][r % 4][2][8]: row 8 (r / 4) + 4 h + r % 4, dim 64 p + 32 j + 8 G + i
            k = c[:, :32 * d].view(-1, d // 64, 2, 4, 4, 4, 2, 8).permute(0, 4, 2, 5, 1, 6, 3, 7).reshape(-1, 32, d)
            # values [d/32][G][16][2][8]: row 8 G + i, dim 32 p + 16 j + r
            v = c[:, 32 * d:].view(-1, d // 32, 4, 16, 2, 8).permute(0, 2, 5, 1, 4, 3).reshape(-1, 32, d)
            sc = tiles[:, 64 * d:].contiguous().view(torch.float32).double().view(-1, 4, 2, 8)
            k, v = k * sc[:, :, 0].reshape(-1, 32, 1), v * sc[:, :, 1].reshape(-1, 32, 1)
        else:
            c = tiles.contiguous().view(torch.bfloat16).double()
            k = c[:, :32 * d].view(-1, d // 32, 2, 4, 4, 4, 8).permute(0, 4, 2, 5, 1, 3, 6).reshape(-1, 32, d)
            v = c[:, 32 * d:].view(-1, d // 16, 4, 16, 8).permute(0, 2, 4, 1, 3).reshape(-1, 32, d)
        return k.reshape(-1, d), v.reshape(-1, d)

    def as_held(x):
        x = x.double()
        if case["kv"] != "fp8":
            return x
        top = x.abs().amax(-1, keepdim=True)
        e = torch.ceil(torch.log2(torch.where(top > 0, top, 1.0) / 448))
        e = torch.where(top > 0, e, 0.0)
        e = torch.where(top * torch.exp2(-e) > 448, e + 1, torch.where((top > 0) & (top * torch.exp2(1 - e) <= 448), e - 1, e))
        return (x * torch.exp2(-e)).float().to(torch.float8_e4m3fn).double() * torch.exp2(e)

    pool = s["pool"][0].view(-1, TPP, s["pool"].shape[-1])
    a = 0
    for i, m in enumerate(s["m"].tolist()):
        sid = case["seqs"] - 1 - i
        pos = int(s["pos"][0, sid])
        lines = []
        for x in range(m):
            y, line = x, []
            while y >= 0:
                line.append(y)
                y = par[a + y]
            lines.append(line)
        t = torch.tensor([pos + len(x) - 1 for x in lines], device=DEV)
        up = torch.zeros((m, m), dtype=torch.bool, device=DEV)
        for x, line in enumerate(lines):
            up[x, line] = True
        for h in range(H):
            L = int(s["len"][0, sid, h])
            table = s["page_table"][0, sid, h, :-(-L // PAGE)].long()
            k, v = tile_rows(pool[table].flatten(0, 1))
            k, v = torch.cat([k[:L], as_held(s["k"][0, a:a + m, h])]), torch.cat([v[:L], as_held(s["v"][0, a:a + m, h])])
            meta = s["slot_meta"][0, sid, h, :L]
            kp = torch.cat([(meta & 0x7FFFFFFF).long(), t])
            fl = torch.cat([meta < 0, s["flags"][0, a:a + m, h].bool()])
            see = torch.ones((m, L + m), dtype=torch.bool, device=DEV)
            see[:, L:] = up
            see &= ~fl | (t[:, None] - kp < w)
            x = s["q"][a:a + m, h * g:(h + 1) * g].double().transpose(0, 1) @ k.T / math.sqrt(d)
            out[a:a + m, h * g:(h + 1) * g] = (torch.softmax(x.masked_fill(~see, -math.inf), -1) @ v).transpose(0, 1)
        a += m
    return {"out": out}


def _kept(case):
    """Expected retained tokens of a head, over the sequences."""
    pos = _shares(case)
    return float((np.minimum(pos, case["window"]) + np.maximum(0, pos - case["window"]) * (1 - case["evict"])).sum())


def _nodes(case):
    return case["seqs"] * ((case["nodes"] + 1) / 2 if case["ragged"] else case["nodes"])


def _work_tree(case):
    H, g, d = SHAPES[case["shape"]]
    row = TILE_BYTES[case["kv"]](d) / 32 + 4
    nodes, kept = _nodes(case), _kept(case)
    mean = nodes / case["seqs"]
    return {"bytes": H * kept * row + nodes * H * (4 * d + 1) + nodes * H * g * d * 4 + 4 * nodes,
            "flops": 4 * d * g * H * (kept * mean + nodes * min(mean, 4))}


# ---------------------------------------------------------------------------
# Accepted paths
# ---------------------------------------------------------------------------

def _run_commit(s):
    case = s["case"]
    n, H, Ly = case["seqs"], SHAPES[case["shape"]][0], case["layers"]
    names = ["pos", "len", "ring", "page_table", "slot_meta", "stack", "top"]
    if own:
        s["front"].copy_(s["saved"][0])
        s["top"].copy_(s["saved"][1])
        dms = _dms()
        for y in range(Ly):
            dms.dms_tree_commit(s["ctx"].handle, y, n, s["ids"], s["cu"], s["total"], s["mmax"], s["path"], s["path_len"],
                                s["k"][y], None if case["kv"] == "mla" else s["v"][y], s["flags"][y], s["ws"])
        return dict({x: s[x] for x in names}, pool=s["pool"][:, :s["pages"] * TPP])
    for x, saved in zip(("pos", "len", "ring", "top"), s["saved"]):
        s[x].copy_(saved)
    d, w = SHAPES[case["shape"]][2], case["window"]
    ids, steps = s["ids"].long(), s["longest"]
    cu, lens = s["cu"].long()[:-1], s["path_len"].long()
    c = torch.arange(steps, device=DEV)
    on = c < lens[:, None]                                                       # [n, steps]
    tok = torch.where(on, cu[:, None] + s["path"].long()[torch.where(on, cu[:, None] + c, 0)], 0)
    flag = s["flags"][:, tok].bool()                                             # [Ly, n, steps, H]
    ring, meta, length = s["ring"][:, ids], s["slot_meta"][:, ids], s["len"][:, ids].long()
    pos = s["pos"][:, ids].long()                                                # [Ly, n]
    first, slots = length.clone(), []
    for x in range(steps):
        t = pos + x
        e = ring.gather(-1, (t % w)[..., None, None].expand(Ly, n, H, 1))[..., 0]
        live = on[:, x][None, :, None]
        reuse = live & (t >= w)[..., None] & (e < 0)
        slot = torch.where(reuse, (e & 0x7FFFFFFF).long(), length)
        length = length + (live & ~reuse)
        mark = torch.where(flag[:, :, x], -(1 << 31), 0).int()
        ring.scatter_(-1, (t % w)[..., None, None].expand(Ly, n, H, 1), torch.where(live, slot.int() | mark, e)[..., None])
        spot = torch.where(live, slot, 0)[..., None]
        meta.scatter_(-1, spot, torch.where(live, t.int()[..., None] | mark, meta.gather(-1, spot)[..., 0])[..., None])
        slots.append(slot)
    # pages: sequences in call order, heads, positions
    had, need = -(-first // PAGE), -(-length // PAGE)
    pops = (need - had).view(Ly, n * H)
    before = (pops.cumsum(-1) - pops).view(Ly, n, H)
    table = s["page_table"][:, ids]
    x = torch.arange(table.shape[-1], device=DEV)
    new = (x >= had[..., None]) & (x < need[..., None])
    take = s["top"].long()[:, :, None, None] - 1 - (before[..., None] + x - had[..., None])
    layer = torch.arange(Ly, device=DEV)[:, None, None]
    table = torch.where(new, s["stack"][layer[..., None], torch.where(new, take, 0)], table)
    s["top"] -= pops.sum(-1, keepdim=True).int()
    s["pos"][:, ids] = (pos + lens).int()
    s["len"][:, ids], s["ring"][:, ids], s["slot_meta"][:, ids], s["page_table"][:, ids] = length.int(), ring, meta, table
    ko, vo = _offsets(case)
    pool = s["pool"].view(torch.int16)
    for i in range(steps):
        live = on[:, i][None, :, None]
        slot = slots[i]
        page = torch.where(live, table.gather(-1, torch.where(live, slot // PAGE, 0)[..., None])[..., 0].long(), s["pages"])
        tile = (page * TPP + slot % PAGE // 32)[..., None]
        pool[layer[..., None], tile, ko[slot % 32]] = s["k"][:, tok[:, i]].view(torch.int16)
        if case["kv"] != "mla":
            pool[layer[..., None], tile, vo[slot % 32]] = s["v"][:, tok[:, i]].view(torch.int16)
    return dict({x: s[x] for x in names}, pool=s["pool"][:, :s["pages"] * TPP])


def _work_commit(case):
    """Rows of the paths read and written once, with their ring and slot entries."""
    H, _, d = SHAPES[case["shape"]]
    mean = _nodes(case) / case["seqs"]
    path = case["seqs"] * min(mean, 2 + 0.2 * mean)
    row = 2 * d * (1 if case["kv"] == "mla" else 2)
    return {"bytes": case["layers"] * (H * path * (2 * row + 13) + case["seqs"] * (8 * H + 8)) + 4 * path, "flops": 0}


def _prepare_accept(case, seed):
    """Drafts that mostly agree with the chosen tokens along one path, and siblings that do not."""
    rng = np.random.default_rng(seed)
    m, parents = _trees(case, rng)
    total = int(m.sum())
    tokens, targets = rng.integers(0, 50, total), rng.integers(0, 50, total)
    a = 0
    for k, par in zip(m, parents):
        x = np.arange(1, k)
        agree = rng.random(k - 1) < 0.6
        tokens[a + x[agree]] = targets[a + par[1:][agree]]
        a += k
    first = tokens[np.cumsum(m) - m].copy()
    lost = rng.random(case["seqs"]) < 0.1
    first[lost] = 51
    s = {"case": case, "m": m, "total": total, "mmax": int(m.max()), "cu": _i32(np.concatenate([[0], np.cumsum(m)])),
         "parents": _i32(np.concatenate(parents)), "tokens": _i32(tokens), "targets": _i32(targets), "first": _i32(first)}
    for name, n in (("path", total), ("path_len", case["seqs"]), ("next", case["seqs"])):
        s[name] = torch.empty(n, dtype=torch.int32, device=DEV)
    return s


def _run_accept(s):
    case = s["case"]
    if own:
        _dms().dms_tree_accept(case["seqs"], s["cu"], s["total"], s["mmax"], s["parents"], s["tokens"], s["targets"],
                               s["first"], s["path"], s["path_len"], s["next"])
        return {x: s[x] for x in ("path", "path_len", "next")}
    n, M = case["seqs"], s["mmax"]
    cu = s["cu"].long()
    x = torch.arange(M, device=DEV)
    there = x < (cu[1:] - cu[:-1])[:, None]
    row = torch.where(there, cu[:-1, None] + x, 0)
    par, tok, tgt = s["parents"][row], s["tokens"][row], s["targets"][row]
    at = torch.full((n,), -1, dtype=torch.int32, device=DEV)
    want, count = s["first"].clone(), torch.zeros(n, dtype=torch.long, device=DEV)
    going = torch.ones(n, dtype=torch.bool, device=DEV)
    path = torch.full((n, M + 1), -1, dtype=torch.int32, device=DEV)
    for _ in range(M):
        hit = there & (par == at[:, None]) & (tok == want[:, None]) & going[:, None]
        going = hit.any(1)
        node = hit.int().argmax(1)           # the first
        path.scatter_(1, torch.where(going, count, M)[:, None], node.int()[:, None])
        count += going
        at = torch.where(going, node.int(), at)
        want = torch.where(going, tgt.gather(1, node[:, None])[:, 0], want)
    keep = x < count[:, None]
    s["path"].fill_(-1)                      # what a path leaves of its tree's entries
    s["path"][(cu[:-1, None] + x)[keep]] = path[:, :M][keep]
    s["path_len"].copy_(count)
    s["next"].copy_(want)
    return {x: s[x] for x in ("path", "path_len", "next")}


def _work_accept(case):
    nodes = _nodes(case)
    return {"bytes": 12 * nodes + 16 * case["seqs"], "flops": nodes}


# ---------------------------------------------------------------------------
# Sampling
# ---------------------------------------------------------------------------

def _prepare_sample(case, seed):
    gen = _gen(seed, 2)
    R, V = case["rows"], case["vocab"]
    x = torch.randn((R, V), generator=gen, device=DEV)
    x = x * case["spread"] + torch.where(torch.rand((R, V), generator=gen, device=DEV) < 8 / V, 6.0, 0.0)
    s = {"case": case, "logits": x.to(torch.float32 if case["dtype"] == "f32" else torch.bfloat16),
         "u": torch.rand(R, generator=gen, device=DEV), "tokens": torch.empty(R, dtype=torch.int32, device=DEV),
         "logprobs": torch.empty(R, device=DEV)}
    if case["mixed"]:        # every row its own setting
        pick = lambda *v: torch.tensor(v, device=DEV)[torch.randint(0, len(v), (R,), generator=gen, device=DEV)]
        s["temperature"], s["top_k"] = pick(0.0, 0.3, 0.6, 0.6, 1.0, 1.5), pick(0, 0, 0, 1, 20, 50, 1000).int()
        s["top_p"], s["min_p"] = pick(1.0, 1.0, 0.95, 0.9, 0.5), pick(0.0, 0.0, 0.05, 0.3)
    if own:
        dms = _dms()
        kind = dms.DMS_TYPE_F32 if case["dtype"] == "f32" else dms.DMS_TYPE_BF16
        s["cfg"] = dms.make_sample_config(V, kind, case["temperature"], case["top_k"], case["top_p"], case["min_p"])
        s["ws"] = torch.empty(dms.dms_sample_workspace(s["cfg"], R), dtype=torch.uint8, device=DEV)
    return s


def _run_sample(s):
    case = s["case"]
    R, V = case["rows"], case["vocab"]
    if own:
        _dms().dms_sample(s["cfg"], R, s["logits"], s.get("temperature"), s.get("top_k"), s.get("top_p"), s.get("min_p"),
                          s["u"], s["tokens"], s["logprobs"], s["ws"])
        return {"tokens": s["tokens"], "logprobs": s["logprobs"]}

    def of(name, dtype):
        x = s[name] if name in s else torch.full((R,), case[name], device=DEV)
        return x.to(dtype)[:, None]

    temp, k = of("temperature", torch.float32).double(), of("top_k", torch.long)
    p, least = of("top_p", torch.float32).double(), of("min_p", torch.float32).double()
    k = torch.where(temp > 0, torch.where((k <= 0) | (k > V), V, k), 1)
    temp = torch.where(temp > 0, temp, 1.0)
    x, index = s["logits"].float().sort(dim=-1, descending=True, stable=True)      # ties: lowest index first
    z = (x.double() - x[:, :1].double()) / temp
    weight = (z.exp() * UNIT).round().long()
    rank = torch.arange(V, device=DEV)
    weight = torch.where(rank < k, weight, 0)
    before = weight.cumsum(-1) - weight
    total = before[:, -1:] + weight[:, -1:]
    keep = ((before < p * total) | (rank == 0)) & (weight >= least * UNIT)
    mass = torch.zeros_like(weight).scatter_(1, index, torch.where(keep, weight, 0)).cumsum(-1)
    total = mass[:, -1:]
    token = (mass <= s["u"].double()[:, None] * total).sum(-1, keepdim=True).clamp(max=V - 1)
    picked = torch.zeros_like(z).scatter_(1, index, z).gather(1, token)
    s["tokens"].copy_(token[:, 0])
    s["logprobs"].copy_((picked - (total / UNIT).log())[:, 0])
    return {"tokens": s["tokens"], "logprobs": s["logprobs"]}


def _exact_sample(case, seed):
    """A row at a time: tokens in order of their logits, cut, and walked by index."""
    s = _prepare_sample(case, seed)
    tokens, logprobs = [], []
    V = case["vocab"]
    value = lambda name, i: float(s[name][i]) if name in s else float(np.float32(case[name]))
    for i in range(case["rows"]):
        x = s["logits"][i].double()
        T, k, p, least = (value(n, i) for n in ("temperature", "top_k", "top_p", "min_p"))
        if T <= 0:
            T, k = 1.0, 1
        k = V if k <= 0 else min(V, int(k))
        order = torch.argsort(-x, stable=True)[:k]
        z = (x - x.max()) / T
        w = torch.round(torch.exp(z) * UNIT).long()[order]
        run = torch.cumsum(w, 0)
        c = k if p >= 1 else min(k, 1 + int((run < p * float(run[-1])).sum()))
        c = max(1, min(c, int((w >= least * UNIT).sum())))
        kept, place = torch.sort(order[:c])
        run = torch.cumsum(w[:c][place], 0)
        at = int(torch.searchsorted(run.double(), float(s["u"][i]) * float(run[-1]), right=True))
        tok = int(kept[min(at, c - 1)])
        tokens.append(tok)
        logprobs.append(float(z[tok]) - math.log(float(run[-1]) / UNIT))
    return {"tokens": torch.tensor(tokens, dtype=torch.int32, device=DEV),
            "logprobs": torch.tensor(logprobs, dtype=torch.float64, device=DEV)}


def _work_sample(case):
    n = case["rows"] * case["vocab"]
    return {"bytes": n * (4 if case["dtype"] == "f32" else 2) + 12 * case["rows"], "flops": 4 * n}


# ---------------------------------------------------------------------------

def prepare(case, seed):
    if case["kind"] == "accept":
        return _prepare_accept(case, seed)
    return _prepare_sample(case, seed) if case["kind"] == "sample" else _prepare_cache(case, seed)


def run(s):
    return {"tree": _run_tree, "commit": _run_commit, "accept": _run_accept, "sample": _run_sample}[s["case"]["kind"]](s)


def work(case):
    return {"tree": _work_tree, "commit": _work_commit, "accept": _work_accept, "sample": _work_sample}[case["kind"]](case)


def exact(case, seed):
    """Appended rows and accepted paths have no computed values."""
    if case["kind"] == "tree":
        return _exact_tree(case, seed)
    return _exact_sample(case, seed) if case["kind"] == "sample" else None
