"""The operators as a program chains them, against float64 from end to end:
training (rotate, windowed attention, its gradient, the rotation's gradient) and
serving (rotate with decisions, prefill, fork, per-chain decode steps, release,
compaction), and a layer trained with a window and sinks served by the cache."""
import math

import numpy as np
import pytest

import dms_synth as sy
import oracle

pytestmark = pytest.mark.gpu


def _bf(x):
    return sy.bf16_bits_to_f32_np(sy.f32_to_bf16_bits_np(np.asarray(x, np.float32))).astype(np.float64)


def _dev(x):
    import torch
    return torch.from_numpy(np.ascontiguousarray(x, np.float32)).cuda().bfloat16()


def test_training_layer_of_rotary_windowed_attention():
    """Gradients of the projection rows: the chain rounds q, k to bf16 after the rotation and the attention's
    gradients to bf16 before they are rotated back, so that an element lies within the attention's slack on the
    rounded inputs, turned (|x1| + |x2| of the slacks of its pair), and half a bf16 step of its own."""
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(0)
    lens, H, g, d, w, sinks, rot = [90, 171], 2, 3, 128, 40, 4, 64
    T, Hq, sec = sum(lens), H * g, [12, 10, 10]
    rows = _bf(rng.normal(size=(T, Hq + 2 * H, d)))
    dout = _bf(rng.normal(size=(T, Hq, d)))
    pos = np.stack([np.concatenate([np.arange(n) for n in lens]) // (a + 1) + 7000 for a in range(3)])
    inv = 1e5 ** (-np.arange(rot // 2) / (rot // 2))
    dev = _dev(rows)
    pd, fd = torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(inv).cuda()
    rc = dms.make_rope_config(H, g, d, rot, sec, axis_order=dms.DMS_ROPE_INTERLEAVED)
    wc = dms.make_window_config(2, T, max(lens), H, g, d, w, sinks)
    cu = torch.tensor([0, 90, T], dtype=torch.int32, device="cuda")
    q, k = torch.empty((T, Hq, d), device="cuda", dtype=torch.bfloat16), torch.empty((T, H, d), device="cuda", dtype=torch.bfloat16)
    v, do = dev[:, Hq + H:].contiguous(), _dev(dout)
    out, lse = torch.empty_like(q), torch.empty((Hq, T), device="cuda")
    dq, dk, dv = torch.empty_like(q), torch.empty_like(k), torch.empty_like(v)
    drows = torch.full_like(dev, 9.0)
    ws = torch.empty(dms.dms_window_workspace(wc), dtype=torch.uint8, device="cuda")
    dms.dms_rope_fwd(rc, T, dev[:, :Hq], dev[:, Hq:Hq + H], pd, fd, q, k)
    dms.dms_window_attention_fwd(wc, cu, q, k, v, out, lse, ws)
    dms.dms_window_attention_bwd(wc, cu, q, k, v, out, lse, do, dq, dk, dv, ws)
    dms.dms_rope_bwd(rc, T, dq, dk, pd, fd, None, drows[:, :Hq], drows[:, Hq:Hq + H])
    torch.cuda.synchronize()
    # the rotated rows, rounded as the library rounds them (checked against the oracle within half a step)
    axes = oracle.rope_axes(sec, True)
    turn = lambda x, back=False: oracle.rope_rotate(x, pos, inv, axes, rot, back=back)
    qr, kr = q.double().cpu().numpy(), k.double().cpu().numpy()
    for got, x in ((qr, rows[:, :Hq]), (kr, rows[:, Hq:Hq + H])):
        y = turn(x)
        assert (np.abs(got - y) <= 2.0 ** -8 * np.abs(y) + 1e-5).all()
    vr = rows[:, Hq + H:]
    half = rot // 2
    a = 0
    for n in lens:
        s = slice(a, a + n)
        grad, slack = oracle.window_attention_grads(qr[s], kr[s], vr[s], dout[s], w, sinks, g)
        for got, name in ((drows[s, :Hq], "dq"), (drows[s, Hq:Hq + H], "dk")):
            y = oracle.rope_rotate(grad[name], pos[:, s], inv, axes, rot, back=True)
            tol = slack[name].copy()
            pair = tol[..., :half] + tol[..., half:rot]
            tol[..., :half], tol[..., half:rot] = pair, pair
            tol = tol + 2.0 ** -8 * (np.abs(y) + tol) + 1e-5
            assert (np.abs(got.double().cpu().numpy() - y) <= tol).all(), name
        assert (np.abs(dv[s].double().cpu().numpy() - grad["dv"]) <= slack["dv"]).all()
        a += n
    assert (drows[:, Hq + H:] == 9.0).all()


def _attend(q, k, v, seen, group, scale):
    out = np.zeros(q.shape)
    for hq in range(q.shape[1]):
        h = hq // group
        out[:, hq] = oracle.masked_attention(q[:, hq], k[:, h], v[:, h], seen[h], scale)
    return out


def test_serving_chains_of_one_prompt():
    """A prompt with image positions is rotated (decisions from its queries), prefilled and forked; the chains
    decode tokens of their own, one is released, the pool compacted, and the others go on.  Every output
    against float64 attention over the sequence's whole history, decisions and rotations taken in float64."""
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(1)
    H, g, d, w, T, bias = 2, 3, 128, 24, 260, -0.8
    Hq, sec, inv = H * g, [24, 20, 20], 1e6 ** (-np.arange(64) / 64)
    axes = oracle.rope_axes(sec, False)
    fd = torch.from_numpy(inv).cuda()
    rc = dms.make_rope_config(H, g, d, d, sec, borrow=1, decision_bias=bias)
    cfg = dms.make_config(1, 6, H, g, d, w, 32, 80, 12, 512)
    c = dms.DmsCache(cfg)
    c.pools[0].fill_(0xFF)
    one = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
    scale = 1 / math.sqrt(d)

    def rotated(rows, pos):
        """The library's rotated q, k with its decisions, checked against the oracle's."""
        n = rows.shape[0]
        dev, pd = _dev(rows), torch.from_numpy(pos.astype(np.int32)).cuda()
        q, k = (torch.empty((n, m, d), device="cuda", dtype=torch.bfloat16) for m in (Hq, H))
        flags = torch.empty((n, H), device="cuda", dtype=torch.uint8)
        dms.dms_rope_fwd(rc, n, dev[:, :Hq], dev[:, Hq:Hq + H], pd, fd, q, k, None, flags)
        logits, rq = oracle.rope_borrow(rows[:, :Hq], g)
        assert np.array_equal(flags.cpu().numpy(), (logits.astype(np.float32) + np.float32(bias) > 0).astype(np.uint8))
        for got, x in ((q, rq), (k, rows[:, Hq:Hq + H])):
            y = oracle.rope_rotate(x, pos, inv, axes, d)
            assert (np.abs(got.double().cpu().numpy() - y) <= 2.0 ** -8 * np.abs(y) + 1e-5).all()
        return q, k, dev[:, Hq + H:].contiguous(), flags

    def host(*xs):
        return [x.double().cpu().numpy() for x in xs]

    rows = _bf(rng.normal(size=(T, Hq + 2 * H, d)))
    pos = np.tile(np.arange(T), (3, 1))
    pos[1, 50:180], pos[2, 50:180] = 50 + np.arange(130) // 13, 50 + np.arange(130) % 13
    pos[0, 50:180] = 50
    q, k, v, flags = rotated(rows, pos)
    out = torch.empty((T, Hq, d), device="cuda")
    dms.dms_prefill_chunk(c.ctx, 0, 1, one([1]), one([0, T]), T, T, q, k, v, flags, out)
    hq, hk, hv, hf = host(q, k, v, flags)
    seen = [oracle.visibility_mask(hf[:, h], w) for h in range(H)]
    assert np.abs(out.double().cpu().numpy() - _attend(hq, hk, hv, seen, g, scale)).max() <= 1e-2
    chains = [4, 0, 3]
    dms.dms_seq_fork(c.ctx, 0, 3, one([1, 1, 1]), one(chains))
    history = {s: [hk, hv, hf] for s in chains + [1]}

    def step(seqs):
        n = len(seqs)
        at = np.tile(np.array([history[s][0].shape[0] for s in seqs]), (3, 1))
        q, k, v, flags = rotated(_bf(rng.normal(size=(n, Hq + 2 * H, d))), at)
        out = torch.empty((n, Hq, d), device="cuda")
        dms.dms_decode_step(c.ctx, 0, n, one(seqs), q, k, v, flags, out)
        nq, nk, nv, nf = host(q, k, v, flags)
        got = out.double().cpu().numpy()
        for i, s in enumerate(seqs):
            history[s] = [np.concatenate([old, new[i:i + 1]]) for old, new in zip(history[s], (nk, nv, nf))]
            K, V, F = history[s]
            last = [oracle.visibility_mask(F[:, h], w)[-1:] for h in range(H)]
            assert np.abs(got[i] - _attend(nq[i:i + 1], K, V, last, g, scale)[0]).max() <= 1e-2, s

    for _ in range(30):
        step(chains)
    step([1, 3])
    dms.dms_seq_reset(c.ctx, 0, 2, one([0, 1]))
    used = one([0])
    dms.dms_compact(c.ctx, 0, used)
    for _ in range(5):
        step([3, 4])
    dms.dms_seq_fork(c.ctx, 0, 1, one([3]), one([5]))
    history[5] = history[3]
    step([5, 4, 3])
    torch.cuda.synchronize()
    assert dms.dms_status(c.ctx) == 0 and 0 < int(used) < 80
    c.close()


def test_cache_serves_a_layer_trained_with_window_and_sinks():
    """Flags 0 for the sinks and 1 for the rest: prefill and decode outputs equal the training forward's."""
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(2)
    for d in (64, 128):
        H, g, w, sinks, T, extra = 2, 4, 32, 5, 300, 12
        n = T + extra
        q, k, v = (_dev(rng.normal(size=(n, m, d))) for m in (H * g, H, H))
        flags = torch.from_numpy((np.arange(n) >= sinks)[:, None].repeat(H, 1).astype(np.uint8)).cuda().contiguous()
        wc = dms.make_window_config(1, n, n, H, g, d, w, sinks)
        want, lse = torch.empty_like(q), torch.empty((H * g, n), device="cuda")
        ws = torch.empty(dms.dms_window_workspace(wc), dtype=torch.uint8, device="cuda")
        one = lambda x: torch.tensor(x, dtype=torch.int32, device="cuda")
        dms.dms_window_attention_fwd(wc, one([0, n]), q, k, v, want, lse, ws)
        c = dms.DmsCache(dms.make_config(1, 2, H, g, d, w, 32, 20, 8, 512))
        out = torch.empty((n, H * g, d), device="cuda")
        dms.dms_prefill_chunk(c.ctx, 0, 1, one([1]), one([0, T]), T, T, q[:T], k[:T], v[:T], flags[:T], out)
        for t in range(T, n):
            row = torch.empty((1, H * g, d), device="cuda")
            dms.dms_decode_step(c.ctx, 0, 1, one([1]), q[t:t + 1], k[t:t + 1], v[t:t + 1], flags[t:t + 1], row)
            out[t] = row[0]
        torch.cuda.synchronize()
        # both round their probabilities to bf16 (2^-8 of sums of p |v|, at most 2^-8 * 4.5 here), one its outputs too
        assert (out - want.float()).abs().max() <= 2 * 2.0 ** -8 * 4.5 + 2.0 ** -8 * 4.5
        assert int(c.export(0).L[1, 0]) == w + sinks
        c.close()
