"""Host-side checks of the tree and sampling entry points: bad sizes and arguments
are refused before any HIP call (no GPU needed)."""
import ctypes

import pytest

from paper_2506_05345_amd import dms

B = ctypes.byref
SOME = ctypes.c_void_p(4096)           # an aligned address that no call may read
INV, UNS = dms.DMS_ERR_INVALID, dms.DMS_ERR_UNSUPPORTED


def _cfg(**kw):
    base = dict(num_layers=2, max_seqs=4, num_kv_heads=2, group_size=3, head_dim=64, window=8, page_size=64, num_pages=32,
                max_pages_per_head=4, max_chunk_tokens=0)
    base.update(kw)
    return dms.make_config(**base)


@pytest.fixture
def context(request):
    made = []

    def make(**kw):
        made.append(dms.dms_create(_cfg(**kw), 0x1000, [0x2000, 0x3000], 0x4000))
        return made[-1]

    yield make
    for c in made:
        dms.dms_destroy(c)


SIZES = [((0, 10, 10), INV), ((5, 10, 10), INV), ((1, -1, 0), INV), ((1, 10, -1), INV), ((1, 10, 11), INV),
         ((1, 10, 0), INV), ((2, 21, 10), INV), ((2, 300, 257), UNS), ((4, 2000, 1000), UNS)]


@pytest.mark.parametrize("sizes,code", SIZES)
def test_sizes_refused(context, sizes, code):
    ctx, L = context(), dms.lib()
    n, total, most = sizes
    assert L.dms_tree_workspace(B(_cfg()), n, total, most, B(ctypes.c_size_t())) == code
    assert L.dms_tree_attention(ctx, 0, n, SOME, SOME, total, most, *[SOME] * 7, None) == code
    assert L.dms_tree_commit(ctx, 0, n, SOME, SOME, total, most, *[SOME] * 6, None) == code
    if n < 5:
        assert L.dms_tree_accept(n, SOME, total, most, *[SOME] * 7, None) == code


def test_large_calls_refused():
    """Query rows in int32 and grids of fewer than 2^32 threads."""
    big = _cfg(max_seqs=65536, num_kv_heads=8, group_size=16)
    size = ctypes.c_size_t()
    assert dms.lib().dms_tree_workspace(B(big), 65536, 65536 * 256, 256, B(size)) == UNS
    heads = _cfg(max_seqs=65536, num_kv_heads=60, group_size=1, head_dim=64)
    assert dms.lib().dms_tree_workspace(B(heads), 65536, 65536 * 200, 256, B(size)) == UNS
    assert dms.lib().dms_tree_workspace(B(_cfg(max_seqs=0)), 1, 1, 1, B(size)) == INV
    assert dms.lib().dms_tree_workspace(None, 1, 1, 1, B(size)) == INV
    assert dms.dms_tree_workspace(_cfg(), 4, 1024, 256) > 0
    assert dms.dms_tree_workspace(_cfg(), 4, 0, 0) > 0


@pytest.mark.parametrize("call,count", [("dms_tree_attention", 7), ("dms_tree_commit", 6)])
def test_arguments_refused(context, call, count):
    ctx, fn = context(), getattr(dms.lib(), call)
    go = lambda args, c=ctx, layer=0, ids=SOME, cu=SOME: fn(c, layer, 2, ids, cu, 10, 6, *args, None)
    for i in range(count):
        args = [SOME] * count
        args[i] = None
        assert go(args) == INV, i
    args = [SOME] * count
    assert go(args, c=None) == go(args, layer=2) == go(args, layer=-1) == go(args, ids=None) == go(args, cu=None) == INV
    tensors = (1, 2, 3, 5) if call == "dms_tree_attention" else (2, 3)
    for i in tensors:
        args = [SOME] * count
        args[i] = ctypes.c_void_p(4096 + 8)                    # off its 16-byte alignment
        assert go(args) == INV, i
    args = [SOME] * count
    args[-1] = ctypes.c_void_p(4096 + 128)                     # workspace off its 256-byte alignment
    assert go(args) == INV
    assert fn(ctx, 0, 2, SOME, SOME, 0, 0, *[None] * count, None) == dms.DMS_OK      # no nodes: nothing to do


def test_attention_modes_refused(context):
    L = dms.lib()
    flags = lambda c: L.dms_tree_attention(c, 0, 2, SOME, SOME, 10, 6, *[SOME] * 7, None)
    query = lambda c: L.dms_tree_attention_q(c, 0, 2, SOME, SOME, 10, 6, *[SOME] * 7, None)
    assert query(context()) == INV
    assert flags(context(decision_source=dms.DMS_DECIDE_QUERY)) == INV
    late = context(eviction=dms.DMS_EVICT_IMMEDIATE)
    assert flags(late) == query(late) == UNS
    rows = context(num_kv_heads=1, head_dim=576, group_size=16, kv_format=dms.DMS_KV_MLA)
    assert flags(rows) == query(rows) == UNS


def test_accept_arguments_refused():
    L = dms.lib()
    for i in (0, 1, 2, 4, 5, 6):                               # the first tokens may be missing
        args = [SOME] * 7
        args[i] = None
        assert L.dms_tree_accept(2, SOME, 10, 6, *args, None) == INV, i
    assert L.dms_tree_accept(2, None, 10, 6, *[SOME] * 7, None) == INV
    assert L.dms_tree_accept(65537, SOME, 10, 6, *[SOME] * 7, None) == INV


def _sample(cfg, rows=4, logits=SOME, stride=1000, u=SOME, tokens=SOME, ws=SOME):
    return dms.lib().dms_sample(B(cfg) if cfg else None, rows, logits, stride, None, None, None, None, u, tokens, None, ws,
                                None)


@pytest.mark.parametrize("kw,code", [(dict(vocab=0), INV), (dict(vocab=-1), INV), (dict(vocab=(1 << 20) + 1), UNS),
                                     (dict(vocab=2**31 - 1), UNS), (dict(logits_type=2), INV), (dict(logits_type=-1), INV)])
def test_sample_configurations_refused(kw, code):
    cfg = dms.make_sample_config(**dict(dict(vocab=1000), **kw))
    assert dms.lib().dms_sample_workspace(B(cfg), 4, None) == code
    assert _sample(cfg, stride=1 << 32) == code


def test_sample_arguments_refused():
    cfg = dms.make_sample_config(1000)
    assert _sample(None) == INV and _sample(cfg, rows=-1) == INV and _sample(cfg, rows=1 << 20) == UNS
    assert _sample(cfg, stride=999) == INV and _sample(cfg, stride=-1000) == INV and _sample(cfg, stride=1 << 40) == INV
    for name in ("logits", "u", "tokens", "ws"):
        assert _sample(cfg, **{name: None}) == INV
    assert _sample(cfg, ws=ctypes.c_void_p(4096 + 16)) == INV
    assert _sample(cfg, logits=ctypes.c_void_p(4098)) == INV                # float32 at half an element
    assert _sample(dms.make_sample_config(1000, dms.DMS_TYPE_BF16), logits=ctypes.c_void_p(4097)) == INV
    assert _sample(cfg, rows=0, logits=None, u=None, tokens=None, ws=None) == dms.DMS_OK
    assert dms.dms_sample_workspace(cfg, 0) >= 0
