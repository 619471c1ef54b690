"""Host-side checks of the rotary, windowed-attention, fork and compaction entry
points: bad configurations and arguments are refused before any HIP call (no GPU
needed)."""
import ctypes

import pytest

from paper_2506_05345_amd import dms

B = ctypes.byref
SOME = ctypes.c_void_p(4096)           # an aligned address that no call may read


def _rope(**kw):
    base = dict(num_kv_heads=2, group_size=3, head_dim=64, rotary_dim=64, sections=[32], borrow=1)
    base.update(kw)
    return dms.make_rope_config(**base)


def _rope_fwd(cfg, tokens=4, q=SOME, qs=384, k=SOME, ks=128, pos=SOME, inv=SOME, qo=SOME, ko=SOME, lo=None, de=None):
    return dms.lib().dms_rope_fwd(B(cfg), tokens, q, qs, k, ks, pos, inv, qo, ko, lo, de, None)


@pytest.mark.parametrize("kw,code", [
    (dict(num_kv_heads=0), dms.DMS_ERR_INVALID), (dict(group_size=0), dms.DMS_ERR_INVALID),
    (dict(head_dim=0), dms.DMS_ERR_INVALID), (dict(rotary_dim=63), dms.DMS_ERR_INVALID),
    (dict(rotary_dim=0, sections=[0]), dms.DMS_ERR_INVALID), (dict(rotary_dim=66, sections=[33]), dms.DMS_ERR_INVALID),
    (dict(rotary_offset=1), dms.DMS_ERR_INVALID), (dict(rotary_offset=-2), dms.DMS_ERR_INVALID),
    (dict(head_dim=2048, rotary_dim=1024, sections=[512]), dms.DMS_ERR_UNSUPPORTED),
    (dict(group_size=1 << 20), dms.DMS_ERR_UNSUPPORTED), (dict(num_kv_heads=2**31 - 1), dms.DMS_ERR_UNSUPPORTED),
    (dict(sections=[31]), dms.DMS_ERR_INVALID), (dict(sections=[33, -1]), dms.DMS_ERR_INVALID),
    (dict(sections=[]), dms.DMS_ERR_INVALID), (dict(sections=[8, 8, 8, 8, 0]), dms.DMS_ERR_INVALID),
    (dict(sections=[10, 22], axis_order=dms.DMS_ROPE_INTERLEAVED), dms.DMS_ERR_INVALID),
    (dict(axis_order=2), dms.DMS_ERR_INVALID), (dict(pairing=-1), dms.DMS_ERR_INVALID),
    (dict(in_type=2), dms.DMS_ERR_INVALID), (dict(out_type=-1), dms.DMS_ERR_INVALID),
    (dict(borrow=2), dms.DMS_ERR_INVALID), (dict(decision_bias=float("nan")), dms.DMS_ERR_INVALID),
    (dict(factor=float("inf")), dms.DMS_ERR_INVALID), (dict(factor=float("nan")), dms.DMS_ERR_INVALID),
])
def test_rope_configurations_refused(kw, code):
    cfg = _rope(**kw)
    assert _rope_fwd(cfg, qs=1 << 40, ks=1 << 40) == code
    assert dms.lib().dms_rope_bwd(B(cfg), 4, SOME, SOME, SOME, SOME, None, SOME, 1 << 40, SOME, 1 << 40, None) == code


def test_rope_arguments_refused():
    cfg = _rope()
    for kw in (dict(tokens=-1), dict(qs=383), dict(ks=127), dict(qs=-384), dict(pos=None), dict(inv=None), dict(qo=None),
               dict(ko=None), dict(q=None), dict(k=None), dict(q=None, qo=None, k=None, ko=None),
               dict(q=None, qo=None, lo=SOME), dict(q=None, qo=None, de=SOME)):
        assert _rope_fwd(cfg, **kw) == dms.DMS_ERR_INVALID, kw
    assert _rope_fwd(_rope(borrow=0), lo=SOME) == dms.DMS_ERR_INVALID
    assert dms.lib().dms_rope_fwd(None, 4, SOME, 384, SOME, 128, *[SOME] * 4, None, None, None) == dms.DMS_ERR_INVALID
    big = _rope(num_kv_heads=1 << 10, group_size=16)
    assert _rope_fwd(big, tokens=1 << 20, qs=1 << 40, ks=1 << 40) == dms.DMS_ERR_UNSUPPORTED
    assert _rope_fwd(cfg, tokens=1 << 26) == dms.DMS_ERR_UNSUPPORTED
    assert _rope_fwd(cfg, tokens=0, q=None, k=None, qo=None, ko=None, pos=None, inv=None) == dms.DMS_OK
    bwd = lambda c, dl=None, qo=SOME, qs=384: dms.lib().dms_rope_bwd(B(c), 4, SOME, SOME, SOME, SOME, dl, qo, qs, SOME, 128, None)
    assert bwd(_rope(borrow=0), dl=SOME) == dms.DMS_ERR_INVALID
    assert bwd(cfg, qo=None) == dms.DMS_ERR_INVALID
    assert bwd(cfg, qs=300) == dms.DMS_ERR_INVALID


def _win(**kw):
    base = dict(num_seqs=2, total_tokens=100, max_seqlen=60, num_kv_heads=2, group_size=3, head_dim=128, window=16, sinks=4)
    base.update(kw)
    return dms.make_window_config(**base)


@pytest.mark.parametrize("kw,code", [
    (dict(num_seqs=0), dms.DMS_ERR_INVALID), (dict(num_seqs=65536), dms.DMS_ERR_INVALID),
    (dict(total_tokens=-1), dms.DMS_ERR_INVALID), (dict(max_seqlen=101), dms.DMS_ERR_INVALID),
    (dict(max_seqlen=0), dms.DMS_ERR_INVALID), (dict(max_seqlen=-1), dms.DMS_ERR_INVALID),
    (dict(num_kv_heads=0), dms.DMS_ERR_INVALID), (dict(group_size=0), dms.DMS_ERR_INVALID),
    (dict(group_size=17), dms.DMS_ERR_UNSUPPORTED), (dict(head_dim=96), dms.DMS_ERR_UNSUPPORTED),
    (dict(head_dim=0), dms.DMS_ERR_UNSUPPORTED), (dict(window=0), dms.DMS_ERR_INVALID),
    (dict(sinks=-1), dms.DMS_ERR_INVALID), (dict(softmax_scale=float("nan")), dms.DMS_ERR_INVALID),
    (dict(softmax_scale=float("inf")), dms.DMS_ERR_INVALID), (dict(num_kv_heads=5000), dms.DMS_ERR_UNSUPPORTED),
    (dict(total_tokens=1 << 30, max_seqlen=5), dms.DMS_ERR_UNSUPPORTED),
    # grids of 2^32 threads and more
    (dict(total_tokens=2**31 - 1, num_kv_heads=1, group_size=1), dms.DMS_ERR_UNSUPPORTED),
    (dict(total_tokens=1 << 20, max_seqlen=1 << 20, sinks=1 << 20), dms.DMS_ERR_UNSUPPORTED),
    (dict(total_tokens=2**31 // 6 - 1, max_seqlen=600, sinks=600), dms.DMS_ERR_UNSUPPORTED),
    # the end of a key's window past int32
    (dict(total_tokens=1 << 30, max_seqlen=1 << 30, num_kv_heads=1, group_size=1, window=1 << 30, sinks=0),
     dms.DMS_ERR_UNSUPPORTED),
])
def test_window_configurations_refused(kw, code):
    cfg = _win(**kw)
    assert dms.lib().dms_window_workspace(B(cfg), None) == code
    assert dms.lib().dms_window_attention_fwd(B(cfg), *[SOME] * 7, None) == code
    assert dms.lib().dms_window_attention_bwd(B(cfg), *[SOME] * 11, None) == code


def test_window_arguments_refused():
    cfg = _win()
    # sinks' sums: (T / 512 + 1) 8 (sinks / 32) workgroups of 256 threads, 2049 x 8192 >= 2^24 and 1025 x 8192 < 2^24
    far = lambda T: _win(total_tokens=T, max_seqlen=1 << 15, sinks=2**31 - 1, window=2**31 - 1)
    assert dms.lib().dms_window_workspace(B(far(1 << 20)), None) == dms.DMS_ERR_UNSUPPORTED
    assert dms.dms_window_workspace(far(1 << 19)) > 0
    assert dms.dms_window_workspace(cfg) > 0
    for call, n in ((dms.lib().dms_window_attention_fwd, 7), (dms.lib().dms_window_attention_bwd, 11)):
        for i in range(n):
            args = [SOME] * n
            args[i] = None
            assert call(B(cfg), *args, None) == dms.DMS_ERR_INVALID, i
        args = [SOME] * n
        args[1] = ctypes.c_void_p(4096 + 8)               # q off its 16-byte alignment
        assert call(B(cfg), *args, None) == dms.DMS_ERR_INVALID
        args = [SOME] * n
        args[-1] = ctypes.c_void_p(4096 + 128)            # workspace off its 256-byte alignment
        assert call(B(cfg), *args, None) == dms.DMS_ERR_INVALID
        assert call(None, *[SOME] * n, None) == dms.DMS_ERR_INVALID
        assert call(B(_win(total_tokens=0, max_seqlen=0)), *[None] * n, None) == dms.DMS_OK


def test_fork_and_compact_arguments_refused():
    cfg = dms.make_config(2, 4, 2, 2, 64, 16, 64, 32, 16, 256)
    pools = (ctypes.c_void_p * 2)(SOME, SOME)
    ctx = ctypes.c_void_p()
    assert dms.lib().dms_create(B(cfg), SOME, pools, SOME, B(ctx)) == dms.DMS_OK
    L = dms.lib()
    for layer, n, src, dst in ((-2, 1, SOME, SOME), (2, 1, SOME, SOME), (0, 0, SOME, SOME), (0, 5, SOME, SOME),
                               (-1, 1, None, SOME), (-1, 1, SOME, None)):
        assert L.dms_seq_fork(ctx, layer, n, src, dst, None) == dms.DMS_ERR_INVALID
    assert L.dms_seq_fork(None, 0, 1, SOME, SOME, None) == dms.DMS_ERR_INVALID
    assert L.dms_compact(None, 0, None, None) == dms.DMS_ERR_INVALID
    for layer in (-2, 2):
        assert L.dms_compact(ctx, layer, None, None) == dms.DMS_ERR_INVALID
    assert L.dms_destroy(ctx) == dms.DMS_OK


def test_binding_checks_tensors():
    import torch
    cfg = _rope()
    q, k = torch.zeros((4, 6, 64), dtype=torch.bfloat16), torch.zeros((4, 2, 64), dtype=torch.bfloat16)
    pos, inv = torch.zeros((1, 4), dtype=torch.int32), torch.ones(32, dtype=torch.float64)
    with pytest.raises(dms.DmsError, match="GPU tensor"):
        dms.dms_rope_fwd(cfg, 4, q, k, pos, inv, q, k)
    with pytest.raises(dms.DmsError, match="must be bf16"):
        dms.dms_rope_fwd(cfg, 4, q.float(), k, pos, inv, q, k)
    with pytest.raises(TypeError):
        dms.dms_rope_fwd(cfg, 4, [1], k, pos, inv, q, k)
    w = _win()
    x = torch.zeros((100, 6, 128))
    with pytest.raises(dms.DmsError, match="must be bf16"):
        dms.dms_window_attention_fwd(w, None, x, None, None, None, None, None)
    # rows: a view into wider rows has their stride, other orders are refused
    rows = torch.zeros((4, 10, 64))
    assert dms._rows_stride(rows[:, :6], 6, 64, None) == 640
    assert dms._rows_stride(rows[:1, :6], 6, 64, None) == 384
    assert dms._rows_stride(rows[:, :6].transpose(0, 1), 4, 64, None) is None
    assert dms._rows_stride(rows[:, :6, :32], 6, 32, None) is None
