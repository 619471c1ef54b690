"""Performance cases of the operators around the DMS cache and its attention.

Four kinds of call, each in a plain form (elementary torch operations) and, where
``own`` is true, as a program calls the library:

* ``rope``: rotary positions of one or several axes for queries and keys, with
  the decision neuron of each KV head taken before the rotation
  (``dms_rope_fwd``); ``rope_bwd``: the gradient of that (``dms_rope_bwd``);
* ``window`` / ``window_step``: attention of packed sequences over a sliding
  window and the first tokens of each sequence, forward
  (``dms_window_attention_fwd``) or forward and backward
  (``dms_window_attention_bwd``);
* ``fork``: the chains of the last request are released and every prompt is
  copied to its chains again (``dms_seq_reset``, ``dms_seq_fork``);
* ``compact``: the live pages of a pool with released sequences move to its
  front (``dms_compact``), from a restored snapshot of the page tables.

Layer shapes are those of the benchmark and of the tests: (KV heads, group,
head dim) of the 1.5B, 7B, 8B and 32B attention layers, latent rows, and a tiny
layer of 64 dims.
"""
import math

import numpy as np
import torch

own = False

DEV = "cuda"
SHAPES = {"tiny": (2, 2, 64), "1.5b": (2, 6, 128), "7b": (4, 7, 128), "8b": (8, 4, 128),
          "32b": (8, 5, 128), "mla16": (1, 16, 576)}
BIAS = -5.0          # offset of the borrowed neuron
PAGE = 64            # tokens of a cache page
TILE_BYTES = {"bf16": lambda d: 128 * d, "fp8": lambda d: 64 * d + 256, "mla": lambda d: 64 * d}
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def _rope(shape, tokens, axes=1, order="sections", pairing="halves", types="bf16-bf16", fused=True, borrow=True,
          kind="rope"):
    return {"kind": kind, "shape": shape, "tokens": tokens, "axes": axes, "order": order, "pairing": pairing,
            "types": types, "fused": fused, "borrow": borrow}


def _window(shape, tokens, seqs=1, low=1.0, window=256, sinks=4, kind="window"):
    return {"kind": kind, "shape": shape, "tokens": tokens, "seqs": seqs, "low": low, "window": window,
            "sinks": sinks}


def _fork(shape, context, prompts, copies, layers=1, window=256, evict=0.875, kv="bf16", bounds=False):
    return {"kind": "fork", "shape": shape, "context": context, "prompts": prompts, "copies": copies,
            "layers": layers, "window": window, "evict": evict, "kv": kv, "bounds": bounds}


def _compact(shape, context, seqs, released, layers=1, window=256, evict=0.875, kv="bf16", bounds=False):
    return {"kind": "compact", "shape": shape, "context": context, "seqs": seqs, "released": released,
            "layers": layers, "window": window, "evict": evict, "kv": kv, "bounds": bounds}


def listed():
    return [
        # one decode step of 32 chains: a launch's latency
        dict(_rope("1.5b", 32), name="rope-decode"),
        # a prefill batch with text and images (time, height, width), cut out of the fused projection
        dict(_rope("32b", 16384, axes=3), name="rope-image-prefill"),
        # the gradients of a training batch's queries and keys, from the attention's float32 gradients
        dict(_rope("32b", 16384, types="f32-bf16", kind="rope_bwd"), name="rope-train"),
        # three short sequences of a small layer, one of a single token
        dict(_window("tiny", 278, seqs=3, low=0.004, window=16, sinks=1), name="window-tiny"),
        # forward over a packed batch of the largest layer
        dict(_window("32b", 16384, seqs=2), name="window-32b"),
        # a training step of a short odd micro-batch of a small model
        dict(_window("1.5b", 1777, sinks=16, kind="window_step"), name="window-train-1.5b-odd"),
        # ragged packed sequences, a longer window and many sinks
        dict(_window("7b", 12001, seqs=5, low=0.1, window=512, sinks=64, kind="window_step"),
             name="window-train-7b-ragged"),
        # a training step at the full training context
        dict(_window("32b", 16384, seqs=2, kind="window_step"), name="window-train-32b"),
        # every layer of a short prompt copied to four chains
        dict(_fork("1.5b", 400, 1, 4, layers=28), name="fork-1.5b"),
        # eight prompts of 32K tokens, each copied to 15 further chains: one layer
        dict(_fork("32b", 32768, 8, 15), name="fork-32b"),
        # a small pool after a release
        dict(_compact("1.5b", 700, 12, 4), name="compact-1.5b"),
        # 128 chains at 32K tokens, a third of them released
        dict(_compact("32b", 32768, 128, 43), name="compact-32b"),
    ]


def _log_int(rng, a, b):
    return int(round(math.exp(rng.uniform(math.log(a), math.log(b)))))


def draw(rng):
    kind = rng.choice(["rope", "rope_bwd", "window", "window", "window_step", "window_step", "fork", "compact"])
    if kind in ("rope", "rope_bwd"):
        shape = rng.choice(["tiny", "1.5b", "7b", "8b", "32b", "mla16"])
        tokens = _log_int(rng, 1, 3000 if shape == "mla16" else 16000)
        types = rng.choice(["bf16-bf16", "bf16-bf16", "f32-bf16", "f32-f32", "bf16-f32"])
        return _rope(shape, tokens, rng.choice([1, 1, 2, 3, 3, 4]), rng.choice(["sections", "interleaved"]),
                     rng.choice(["halves", "adjacent"]), types, rng.random() < 0.5,
                     shape != "mla16" and rng.random() < 0.5, kind)
    if kind in ("window", "window_step"):
        shape = rng.choice(["tiny", "1.5b", "7b", "8b", "32b"])
        H, g, _ = SHAPES[shape]
        window = _log_int(rng, 1, 1500)
        tokens = _log_int(rng, 1, 16000)
        while tokens * H * g * (window + 300) > 1.5e8:
            tokens = tokens * 2 // 3 + 1
            window = window * 4 // 5 + 1
        return _window(shape, tokens, min(tokens, _log_int(rng, 1, 8)), rng.uniform(0.02, 1.0), window,
                       rng.choice([0, 1, 4, 16, 33, 64]), kind)
    shape = rng.choice(["tiny", "1.5b", "7b", "8b", "32b", "mla16"])
    kv = "mla" if shape == "mla16" else rng.choice(["bf16", "bf16", "fp8"])
    bounds = kv != "mla" and rng.random() < 0.3
    context = _log_int(rng, 10, 32768)
    window = rng.choice([16, 64, 256])
    evict = rng.choice([0.5, 0.75, 0.875])
    if kind == "fork":
        prompts = rng.choice([1, 1, 2, 5, 8])
        copies = _log_int(rng, 1, 16)
        while prompts * copies * context > 1200000:
            copies = max(1, copies // 2)
            context = context // 2
        layers = rng.choice([1, 2, 7]) if prompts * copies * context < 150000 else 1
        return _fork(shape, context, prompts, copies, layers, window, evict, kv, bounds)
    seqs = _log_int(rng, 2, 100)
    while seqs * context > 1200000:
        context = context // 2
    layers = rng.choice([1, 2, 7]) if seqs * context < 150000 else 1
    return _compact(shape, context, seqs, rng.randint(1, seqs - 1), layers, window, evict, kv, bounds)


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


# ---------------------------------------------------------------------------
# Rotary positions
# ---------------------------------------------------------------------------

def _rope_geometry(case):
    """(Hkv, g, d, rotary_dim, rotary_offset, sections)."""
    H, g, d = SHAPES[case["shape"]]
    rot, off = (64, 512) if case["shape"] == "mla16" else (d, 0)
    half, axes = rot // 2, case["axes"]
    rest = half * 3 // 8 if axes == 3 and case["order"] == "sections" else half // axes
    sections = [half - rest * (axes - 1)] + [rest] * (axes - 1)
    return H, g, d, rot, off, sections


def _axis_of_pair(case):
    """Axis whose position turns pair i."""
    *_, sections = _rope_geometry(case)
    axes = len(sections)
    if case["order"] == "sections":
        return np.repeat(np.arange(axes), sections)
    i = np.arange(sum(sections))
    return np.where(i // axes < np.array(sections)[i % axes], i % axes, 0)


def _positions(case, seed):
    """[axes, tokens]: text, with images whose tokens share a time and run over rows and columns."""
    T, axes = case["tokens"], case["axes"]
    rng = np.random.default_rng(seed)
    pos = np.tile(np.arange(T, dtype=np.int64) + int(rng.integers(0, 100000)), (axes, 1))
    for _ in range(4 if axes > 1 else 0):
        n = int(rng.integers(0, T // 4 + 1))
        a = int(rng.integers(0, max(1, T - n)))
        cols = int(rng.integers(8, 65))
        i = np.arange(n)
        for x in range(axes):
            pos[x, a:a + n] = pos[0, a] + (0, i // cols, i % cols, i // (cols * 8))[x]
    return _i32(pos)


def _prepare_rope(case, seed):
    H, g, d, rot, off, sections = _rope_geometry(case)
    T, Hq = case["tokens"], H * g
    gen = _gen(seed, 1)
    tin, tout = (DTYPES[x] for x in case["types"].split("-"))
    s = {"case": case, "positions": _positions(case, seed),
         "inv_freq": 1e6 ** (-torch.arange(0, rot, 2, dtype=torch.float64, device=DEV) / rot)}
    heads = Hq + 2 * H
    if case["kind"] == "rope":
        if case["fused"]:      # q and k are parts of the rows of one projection
            rows = _normal(gen, (T, heads, d), tin, 2.0)
            s["q"], s["k"] = rows[:, :Hq], rows[:, Hq:Hq + H]
        else:
            s["q"], s["k"] = _normal(gen, (T, Hq, d), tin, 2.0), _normal(gen, (T, H, d), tin, 2.0)
        if case["borrow"]:
            s["q"][:, ::g, 0] += 5.0
        s["q_out"] = torch.empty((T, Hq, d), dtype=tout, device=DEV)
        s["k_out"] = torch.empty((T, H, d), dtype=tout, device=DEV)
        s["logits"] = torch.empty((T, H), device=DEV)
        s["decisions"] = torch.empty((T, H), dtype=torch.uint8, device=DEV)
    else:
        s["dq"], s["dk"] = _normal(gen, (T, Hq, d), tin), _normal(gen, (T, H, d), tin)
        s["dlogits"] = _normal(gen, (T, H), torch.float32)
        if case["fused"]:
            rows = torch.empty((T, heads, d), dtype=tout, device=DEV)
            s["dq_out"], s["dk_out"] = rows[:, :Hq], rows[:, Hq:Hq + H]
        else:
            s["dq_out"] = torch.empty((T, Hq, d), dtype=tout, device=DEV)
            s["dk_out"] = torch.empty((T, H, d), dtype=tout, device=DEV)
    if own:
        dms = _dms()
        types = {"bf16": dms.DMS_TYPE_BF16, "f32": dms.DMS_TYPE_F32}
        a, b = case["types"].split("-")
        s["cfg"] = dms.make_rope_config(
            H, g, d, rot, sections, rotary_offset=off,
            axis_order=dms.DMS_ROPE_SECTIONS if case["order"] == "sections" else dms.DMS_ROPE_INTERLEAVED,
            pairing=dms.DMS_ROPE_HALVES if case["pairing"] == "halves" else dms.DMS_ROPE_ADJACENT,
            in_type=types[a], out_type=types[b], borrow=int(case["borrow"]), decision_bias=BIAS)
    return s


def _rotate(x, cos, sin, case):
    """Rotated copy of float32 rows x [T, heads, d]."""
    _, _, d, rot, off, _ = _rope_geometry(case)
    part = x[..., off:off + rot]
    if case["pairing"] == "halves":
        a, b = part[..., :rot // 2], part[..., rot // 2:]
    else:
        a, b = part[..., 0::2], part[..., 1::2]
    c, s = cos[:, None], sin[:, None]
    ra, rb = a * c - b * s, a * s + b * c
    turned = torch.cat([ra, rb], -1) if case["pairing"] == "halves" else torch.stack([ra, rb], -1).flatten(-2)
    return torch.cat([x[..., :off], turned, x[..., off + rot:]], -1)


def _angles(s):
    axis = torch.as_tensor(_axis_of_pair(s["case"]), device=DEV)
    turn = s["positions"][axis].double().T * s["inv_freq"]
    return turn.cos().float(), turn.sin().float()


def _run_rope(s):
    case = s["case"]
    _, g, *_ = _rope_geometry(case)
    T = case["tokens"]
    if case["kind"] == "rope":
        if own:
            dms = _dms()
            taken = (s["logits"], s["decisions"]) if case["borrow"] else (None, None)
            dms.dms_rope_fwd(s["cfg"], T, s["q"], s["k"], s["positions"], s["inv_freq"], s["q_out"], s["k_out"], *taken)
        else:
            cos, sin = _angles(s)
            q = s["q"].float()
            if case["borrow"]:
                s["logits"] = q[:, ::g, 0].clone()
                s["decisions"] = (s["logits"] + BIAS > 0).to(torch.uint8)
                q = q.clone()
                q[:, ::g, 0] = 0
            s["q_out"] = _rotate(q, cos, sin, case).to(s["q_out"].dtype)
            s["k_out"] = _rotate(s["k"].float(), cos, sin, case).to(s["k_out"].dtype)
        out = {"q": s["q_out"], "k": s["k_out"]}
        return dict(out, logits=s["logits"], decisions=s["decisions"]) if case["borrow"] else out
    if own:
        _dms().dms_rope_bwd(s["cfg"], T, s["dq"], s["dk"], s["positions"], s["inv_freq"],
                            s["dlogits"] if case["borrow"] else None, s["dq_out"], s["dk_out"])
    else:
        cos, sin = _angles(s)
        dq = _rotate(s["dq"].float(), cos, -sin, case)
        if case["borrow"]:
            dq[:, ::g, 0] = s["dlogits"]
        s["dq_out"] = dq.to(s["dq_out"].dtype)
        s["dk_out"] = _rotate(s["dk"].float(), cos, -sin, case).to(s["dk_out"].dtype)
    return {"dq": s["dq_out"], "dk": s["dk_out"]}


def _exact_rope(case, seed):
    s = _prepare_rope(case, seed)
    H, g, d, rot, off, _ = _rope_geometry(case)
    axis = _axis_of_pair(case)
    angle = torch.stack([s["positions"][int(a)].double() * s["inv_freq"][i] for i, a in enumerate(axis)], 1)
    back = case["kind"] == "rope_bwd"
    turn = torch.polar(torch.ones_like(angle), -angle if back else angle)[:, None]

    def spin(x):
        y = x.double().clone()
        lo = torch.arange(rot // 2, device=DEV) + off if case["pairing"] == "halves" else \
            torch.arange(0, rot, 2, device=DEV) + off
        hi = lo + (rot // 2 if case["pairing"] == "halves" else 1)
        z = torch.complex(y[..., lo], y[..., hi]) * turn
        y[..., lo], y[..., hi] = z.real, z.imag
        return y

    if back:
        dq, dk = spin(s["dq"]), spin(s["dk"])
        if case["borrow"]:
            dq[:, torch.arange(H, device=DEV) * g, 0] = s["dlogits"].double()
        return {"dq": dq, "dk": dk}
    q = s["q"].double().clone()
    first = q[:, torch.arange(H, device=DEV) * g, 0].clone()
    if case["borrow"]:
        q[:, torch.arange(H, device=DEV) * g, 0] = 0
    out = {"q": spin(q), "k": spin(s["k"])}
    return dict(out, logits=first, decisions=None) if case["borrow"] else out


def _work_rope(case):
    H, g, d, rot, _, _ = _rope_geometry(case)
    T, heads = case["tokens"], H * g + H
    size = {"bf16": 2, "f32": 4}
    a, b = case["types"].split("-")
    taken = 5 * T * H if case["borrow"] and case["kind"] == "rope" else 4 * T * H if case["borrow"] else 0
    return {"bytes": T * heads * d * (size[a] + size[b]) + 4 * T * case["axes"] + 4 * rot + taken,
            "flops": 3 * T * heads * rot}


# ---------------------------------------------------------------------------
# Windowed attention with sinks
# ---------------------------------------------------------------------------

def _lengths(case):
    """Lengths of the packed sequences: from `low` of the longest to the longest, mixed, adding to `tokens`."""
    n, T = case["seqs"], case["tokens"]
    share = [1.0 if n == 1 else case["low"] + (1 - case["low"]) * i / (n - 1) for i in range(n)]
    step = next(x for x in (7, 5, 3, 1) if math.gcd(x, n) == 1)
    share = [share[(i * step) % n] for i in range(n)]
    cut = [round(T * sum(share[:i]) / sum(share)) for i in range(n + 1)]
    return [b - a for a, b in zip(cut, cut[1:])]


def _prepare_window(case, seed):
    H, g, d = SHAPES[case["shape"]]
    T, Hq = case["tokens"], H * g
    gen = _gen(seed, 2)
    bf = torch.bfloat16
    lens = _lengths(case)
    s = {"case": case, "max_len": max(lens), "cu": _i32(np.concatenate([[0], np.cumsum(lens)])),
         "q": _normal(gen, (T, Hq, d), bf, 2.0), "k": _normal(gen, (T, H, d), bf), "v": _normal(gen, (T, H, d), bf)}
    if case["kind"] == "window_step":
        s["dout"] = _normal(gen, (T, Hq, d), bf)
    if own:
        dms = _dms()
        s["cfg"] = dms.make_window_config(len(lens), T, s["max_len"], H, g, d, case["window"], case["sinks"])
        s["ws"] = torch.empty(max(1, dms.dms_window_workspace(s["cfg"])), dtype=torch.uint8, device=DEV)
        s["out"] = torch.empty_like(s["q"])
        s["lse"] = torch.empty((Hq, T), device=DEV)
        s["dq"], s["dk"], s["dv"] = (torch.empty_like(s[x]) for x in "qkv")
    return s


def _plain_window(s):
    """Blocks of B queries against the block before them and their own, B at least the window, and against
    the sinks of every sequence."""
    case = s["case"]
    H, g, d = SHAPES[case["shape"]]
    T, w, ns, n = case["tokens"], min(case["window"], s["max_len"]), case["sinks"], case["seqs"]
    B = max(w, 64)
    nb = -(-T // B)
    pad = nb * B - T
    cu = s["cu"].long()
    t = torch.arange(-B, nb * B, device=DEV)
    seg = torch.searchsorted(cu[1:], t.clamp(0, T - 1), right=True)
    seg = torch.where((t < 0) | (t >= T), -1, seg)
    qt, kt = t[B:].view(nb, B), t.view(nb + 1, B)
    kt = torch.cat([kt[:-1], kt[1:]], 1)
    qs, ks = seg[B:].view(nb, B), torch.cat([seg.view(nb + 1, B)[:-1], seg.view(nb + 1, B)[1:]], 1)
    see = (qs[:, :, None] == ks[:, None]) & (qs[:, :, None] >= 0) & (kt[:, None] <= qt[:, :, None]) & \
        (kt[:, None] > qt[:, :, None] - w)                                             # [nb, B, 2B]
    first = cu[:-1, None] + torch.arange(ns, device=DEV)
    there = (first < cu[1:, None]).flatten()
    first, owner = first.flatten().clamp(max=T - 1), torch.arange(n, device=DEV).repeat_interleave(ns)
    see0 = (qs[:, :, None] == owner) & there & (first <= qt[:, :, None] - w)           # [nb, B, n sinks]

    def queries(x):     # [T, Hq, d] -> [H, nb, B g, d]
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, 0, pad)).view(nb, B, H, g, d)
        return x.permute(2, 0, 1, 3, 4).reshape(H, nb, B * g, d)

    def keys(x):        # [T, H, d] -> [H, nb, 2B, d]
        x = torch.nn.functional.pad(x.float(), (0, 0, 0, 0, B, pad)).view(nb + 1, B, H, d)
        return torch.cat([x[:-1], x[1:]], 1).permute(2, 0, 1, 3).contiguous()

    def unqueries(x):
        return x.view(H, nb, B, g, d).permute(1, 2, 0, 3, 4).reshape(nb * B, H * g, d)[:T]

    scale = 1 / math.sqrt(d)
    q, k, v = queries(s["q"]), keys(s["k"]), keys(s["v"])
    k0 = s["k"].float()[first].permute(1, 0, 2).contiguous()[:, None]                  # [H, 1, n sinks, d]
    v0 = s["v"].float()[first].permute(1, 0, 2).contiguous()[:, None]
    see, see0 = see.repeat_interleave(g, 1), see0.repeat_interleave(g, 1)
    hide = torch.finfo(torch.float32).min
    p = torch.cat([(q @ k.transpose(-1, -2) * scale).masked_fill_(~see, hide),
                   (q @ k0.transpose(-1, -2) * scale).masked_fill_(~see0, hide)], -1)
    m = p.amax(-1, keepdim=True)
    p = (p - m).exp_() * torch.cat([see, see0], -1)
    l = p.sum(-1, keepdim=True)
    p /= l.clamp(min=1e-30)
    p1, p0 = p[..., :2 * B], p[..., 2 * B:]
    out = unqueries(p1 @ v + p0 @ v0).to(torch.bfloat16)
    lse = (m + l.clamp(min=1e-30).log()).view(H, nb * B, g)[:, :T].permute(0, 2, 1).reshape(H * g, T)
    if case["kind"] == "window":
        return {"out": out, "lse": lse}
    do = queries(s["dout"])
    dp1, dp0 = do @ v.transpose(-1, -2), do @ v0.transpose(-1, -2)
    row = (p1 * dp1).sum(-1, keepdim=True) + (p0 * dp0).sum(-1, keepdim=True)
    ds1, ds0 = p1 * (dp1 - row) * scale, p0 * (dp0 - row) * scale
    dq = unqueries(ds1 @ k + ds0 @ k0)

    def unkeys(x, x0):  # gradients of the blocks' keys and of the sinks -> [T, H, d]
        y = torch.nn.functional.pad(x[:, :, B:], (0, 0, 0, 0, 1, 0)) + torch.nn.functional.pad(x[:, :, :B], (0, 0, 0, 0, 0, 1))
        y = y.permute(1, 2, 0, 3).reshape((nb + 1) * B, H, d)[B:B + T].contiguous()
        return y.index_add_(0, first[there], x0.sum(1).permute(1, 0, 2)[there])

    dk = unkeys(ds1.transpose(-1, -2) @ q, ds0.transpose(-1, -2) @ q)
    dv = unkeys(p1.transpose(-1, -2) @ do, p0.transpose(-1, -2) @ do)
    return {"out": out, "lse": lse, "dq": dq.to(torch.bfloat16), "dk": dk.to(torch.bfloat16), "dv": dv.to(torch.bfloat16)}


def _run_window(s):
    if not own:
        return _plain_window(s)
    dms = _dms()
    dms.dms_window_attention_fwd(s["cfg"], s["cu"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["ws"])
    res = {"out": s["out"], "lse": s["lse"]}
    if s["case"]["kind"] == "window_step":
        dms.dms_window_attention_bwd(s["cfg"], s["cu"], s["q"], s["k"], s["v"], s["out"], s["lse"], s["dout"],
                                     s["dq"], s["dk"], s["dv"], s["ws"])
        res.update(dq=s["dq"], dk=s["dk"], dv=s["dv"])
    return res


def _exact_window(case, seed):
    """Dense attention of one sequence and KV head at a time."""
    s = _prepare_window(case, seed)
    H, g, d = SHAPES[case["shape"]]
    T, step = case["tokens"], case["kind"] == "window_step"
    res = {"out": torch.zeros((T, H * g, d), dtype=torch.float64, device=DEV),
           "lse": torch.zeros((H * g, T), dtype=torch.float64, device=DEV)}
    if step:
        res.update(dq=torch.zeros_like(res["out"]), dk=torch.zeros((T, H, d), dtype=torch.float64, device=DEV),
                   dv=torch.zeros((T, H, d), dtype=torch.float64, device=DEV))
    cu = s["cu"].tolist()
    for a, b in zip(cu, cu[1:]):
        i = torch.arange(b - a, device=DEV)
        gap = i[:, None] - i
        seen = (gap >= 0) & ((gap < case["window"]) | (i < case["sinks"]))
        for hq in range(H * g):
            h = hq // g
            q, k, v = s["q"][a:b, hq].double(), s["k"][a:b, h].double(), s["v"][a:b, h].double()
            x = (q @ k.T / math.sqrt(d)).masked_fill(~seen, -math.inf)
            res["lse"][hq, a:b] = torch.logsumexp(x, 1)
            p = torch.softmax(x, 1)
            res["out"][a:b, hq] = p @ v
            if step:
                do = s["dout"][a:b, hq].double()
                res["dv"][a:b, h] += p.T @ do
                ds = p * (do @ v.T - (do * res["out"][a:b, hq]).sum(1, keepdim=True)) / math.sqrt(d)
                res["dq"][a:b, hq] = ds @ k
                res["dk"][a:b, h] += ds.T @ q
    return res


def _work_window(case):
    H, g, d = SHAPES[case["shape"]]
    T, w, ns = case["tokens"], case["window"], case["sinks"]
    pairs = 0
    for n in _lengths(case):
        t = np.arange(n, dtype=np.int64)
        old = np.maximum(0, t - w + 1)                       # keys before the window
        pairs += int((t + 1 - old + np.minimum(old, ns)).sum())
    rows_q, rows_k = T * H * g, T * H
    fwd = 2 * d * (2 * rows_q + 2 * rows_k) + 4 * rows_q
    if case["kind"] == "window":
        return {"bytes": fwd, "flops": 4 * d * pairs * H * g}
    return {"bytes": fwd + 2 * d * (2 * rows_q + 2 * rows_k), "flops": 14 * d * pairs * H * g}


# ---------------------------------------------------------------------------
# Cache pages
# ---------------------------------------------------------------------------

def _cache_size(case):
    """(sequences, tile bytes, pages of a head's table, pages of the pool)."""
    H, _, d = SHAPES[case["shape"]]
    live = case["prompts"] * (1 + case["copies"]) if case["kind"] == "fork" else case["seqs"]
    most = min(case["context"], case["window"] + int(max(0, case["context"] - case["window"]) * min(1.0, 1.4 * (1 - case["evict"]))) + 1)
    maxp = -(-most // PAGE)
    return live + 1, TILE_BYTES[case["kv"]](d), maxp, live * H * maxp + 8


def _prepare_cache(case, seed):
    """The state arrays of every layer and its pool, as the library documents them: each head of each live
    sequence retains its own number of tokens, pages lie scattered over the pool."""
    H, g, d = SHAPES[case["shape"]]
    S, tile, maxp, pages = _cache_size(case)
    Ly, w = case["layers"], case["window"]
    rng = np.random.default_rng(seed)
    fork = case["kind"] == "fork"
    if fork:
        src = np.repeat(np.arange(case["prompts"]), case["copies"])
        dst = case["prompts"] + np.arange(len(src))
        owners = case["prompts"]
    else:
        owners = case["seqs"]
    cfg = _dms().make_config(Ly, S, H, g, d, w, PAGE, pages, maxp,
                             kv_format={"bf16": 0, "fp8": 1, "mla": 2}[case["kv"]],
                             quest_page_budget=1 if case["bounds"] else 0) if own else None
    # retained tokens of every head
    pos = np.zeros((Ly, S), np.int32)
    length = np.zeros((Ly, S, H), np.int32)
    pos[:, :owners] = np.maximum(1, rng.integers(case["context"] * 3 // 4, case["context"] + 1, (1, owners)))
    old = np.maximum(0, pos[:, :owners, None] - w)
    keep = (1 - case["evict"]) * rng.uniform(0.6, 1.4, (Ly, owners, H))
    length[:, :owners] = np.minimum(np.minimum(pos[:, :owners, None], w) + (old * np.minimum(keep, 1)).astype(np.int32), maxp * PAGE)
    if fork:
        pos[:, dst], length[:, dst] = pos[:, src], length[:, src]
    else:
        gone = rng.permutation(case["seqs"])[:case["released"]]
        pos[:, gone], length[:, gone] = 0, 0
    # page tables: live sequences first take pages in a scattered order, the chains of the last fork (fork) from
    # the top of what is left, as one block in stack order
    table = np.full((Ly, S, H, maxp), -1, np.int32)
    stack = np.zeros((Ly, pages), np.int32)
    top = np.zeros((Ly, 1), np.int32)
    count = -(-length // PAGE)
    for y in range(Ly):
        order = rng.permutation(pages).astype(np.int32)
        mine = np.arange(maxp) < count[y, :, :, None]
        if fork:
            held = mine.copy()
            held[dst] = False
            order = order[::-1]
            n_held, n_all = int(held.sum()), int(mine.sum())
            stack[y] = order
            top[y] = pages - n_all
            table[y][held] = order[pages - n_held:]
            chains = mine[dst]
            part = table[y][dst]
            part[chains] = order[pages - n_all:pages - n_held]
            table[y, dst] = part
        else:
            n_all = int(mine.sum())
            table[y][mine] = order[:n_all]
            stack[y, :pages - n_all] = order[n_all:]
            top[y] = pages - n_all
    gen = _gen(seed, 3)
    slots = maxp * PAGE
    t = {"pos": _i32(pos), "len": _i32(length), "page_table": _i32(table), "stack": _i32(stack), "top": _i32(top)}
    dead = t["len"][..., None] <= 0
    t["ring"] = torch.randint(0, 1 << 30, (Ly, S, H, w), generator=gen, device=DEV, dtype=torch.int32) % \
        t["len"].clamp(min=1)[..., None]
    t["ring"] = torch.where(dead, 0, t["ring"] | (torch.rand((Ly, S, H, w), generator=gen, device=DEV) < case["evict"]).int() << 31)
    t["slot_meta"] = torch.randint(0, case["context"], (Ly, S, H, slots), generator=gen, device=DEV, dtype=torch.int32)
    pool = torch.randn((Ly, pages * (PAGE // 32), tile // 2), generator=gen, device=DEV, dtype=torch.bfloat16)
    bounds = torch.randn((Ly, pages, 2 * d), generator=gen, device=DEV, dtype=torch.bfloat16) if case["bounds"] else None
    s = {"case": case, "pool": pool.view(torch.int16)}
    if own:
        dms = _dms()
        meta_bytes, pool_bytes, ws_bytes, _ = dms.dms_layout(cfg)
        o = dms.dms_state_layout(cfg)
        meta = torch.zeros(meta_bytes, dtype=torch.uint8, device=DEV)
        assert pool_bytes == pool[0].numel() * 2
        s["ws"] = torch.zeros(max(1, ws_bytes), dtype=torch.uint8, device=DEV)
        s["meta"] = meta
        s["ctx"] = _Context(dms, dms.dms_create(cfg, meta, [s["pool"][y] for y in range(Ly)], s["ws"]))
        dms.dms_init_state(s["ctx"].handle)
        layers = meta[o.layer0:o.layer0 + Ly * o.layer_stride].view(Ly, o.layer_stride)

        def inside(name, like):
            at = getattr(o, name)
            size = like[0].numel() * like.element_size()
            return layers[:, at:at + size].view(like.dtype).unflatten(1, like.shape[1:])

        for name, x in t.items():
            s[name] = inside(name, x)
            s[name].copy_(x)
        if bounds is not None:
            s["bounds"] = inside("page_bounds", bounds.view(torch.int16))
            s["bounds"].copy_(bounds.view(torch.int16))
    else:
        s.update(t)
        if bounds is not None:
            s["bounds"] = bounds.view(torch.int16)
    if fork:
        s["src"], s["dst"] = _i32(src), _i32(dst)
    else:
        s["saved"] = (t["page_table"].clone(), t["stack"].clone())
        s["used"] = torch.empty(Ly, dtype=torch.int32, device=DEV)
    return s


class _Context:
    """A context handle that is destroyed with the state that holds it."""

    def __init__(self, dms, handle):
        self.dms, self.handle = dms, handle

    def __del__(self):
        self.dms.dms_destroy(self.handle)


def _state(s):
    names = ["pos", "len", "ring", "page_table", "slot_meta", "stack", "top", "pool"]
    return {x: s[x] for x in names + (["bounds"] if "bounds" in s else [])}


def _each(counts):
    """For counts [rows]: (row, number inside the row, number before the row) of every counted item."""
    before = counts.cumsum(0) - counts
    row = torch.repeat_interleave(torch.arange(counts.numel(), device=DEV), counts)
    return row, torch.arange(row.numel(), device=DEV) - before[row], before


def _run_fork(s):
    case = s["case"]
    if own:
        dms = _dms()
        n = s["dst"].numel()
        dms.dms_seq_reset(s["ctx"].handle, -1, n, s["dst"])
        dms.dms_seq_fork(s["ctx"].handle, -1, n, s["src"], s["dst"])
        return _state(s)
    H = SHAPES[case["shape"]][0]
    Ly, tpp = case["layers"], PAGE // 32
    src, dst = s["src"].long(), s["dst"].long()
    n = src.numel()
    layer = torch.arange(Ly, device=DEV)[:, None, None].expand(Ly, n, H).reshape(-1)
    head = torch.arange(H, device=DEV).expand(Ly, n, H).reshape(-1)
    to = dst[None, :, None].expand(Ly, n, H).reshape(-1)
    of = src[None, :, None].expand(Ly, n, H).reshape(-1)
    # release: pages back on the stack, in call order
    count = ((s["len"][:, dst] + PAGE - 1) // PAGE).long()
    row, k, before = _each(count.flatten())
    start = before.view(Ly, -1)[:, :1] - s["top"].long()            # items before the layer, less its stack height
    s["stack"][layer[row], before[row] + k - start.flatten()[layer[row]]] = s["page_table"][layer[row], to[row], head[row], k]
    s["page_table"][layer[row], to[row], head[row], k] = -1
    top = s["top"].long() + count.sum((1, 2))[:, None]
    # fork: one block of pages off the top, its lowest entry first
    count = ((s["len"][:, src] + PAGE - 1) // PAGE).long()
    row, k, before = _each(count.flatten())
    top = top - count.sum((1, 2))[:, None]
    start = before.view(Ly, -1)[:, :1] - top
    s["page_table"][layer[row], to[row], head[row], k] = s["stack"][layer[row], before[row] + k - start.flatten()[layer[row]]]
    s["top"].copy_(top)
    if "bounds" in s:
        s["bounds"][layer[row], s["page_table"][layer[row], to[row], head[row], k].long()] = \
            s["bounds"][layer[row], s["page_table"][layer[row], of[row], head[row], k].long()]
    length = s["len"][:, src]
    s["pos"][:, dst], s["len"][:, dst], s["ring"][:, dst] = s["pos"][:, src], length, s["ring"][:, src]
    live = torch.arange(s["slot_meta"].shape[-1], device=DEV) < length[..., None]
    s["slot_meta"][:, dst] = torch.where(live, s["slot_meta"][:, src], s["slot_meta"][:, dst])
    row, k, _ = _each(((length + 31) // 32).long().flatten())

    def tiles(seq):
        return s["page_table"][layer[row], seq[row], head[row], k // tpp].long() * tpp + k % tpp

    s["pool"][layer[row], tiles(to)] = s["pool"][layer[row], tiles(of)]
    return _state(s)


def _run_compact(s):
    case = s["case"]
    s["page_table"].copy_(s["saved"][0])
    s["stack"].copy_(s["saved"][1])
    if own:
        _dms().dms_compact(s["ctx"].handle, -1, s["used"])
        return dict(_state(s), used=s["used"])
    Ly, pages, tpp = case["layers"], s["stack"].shape[1], PAGE // 32
    top = s["top"].long()
    used = pages - top                                               # [Ly, 1]
    ids = torch.arange(pages, device=DEV).expand(Ly, pages)
    free = torch.zeros((Ly, pages), dtype=torch.bool, device=DEV)
    free.scatter_(1, torch.where(ids < top, s["stack"].long(), s["stack"][:, :1].long()), True)
    free &= top > 0
    hole, high = free & (ids < used), ~free & (ids >= used)          # equally many in a layer
    y0, x0 = hole.nonzero(as_tuple=True)
    y1, x1 = high.nonzero(as_tuple=True)
    to = ids.clone()
    to[y1, x1] = x0
    page = s["pool"].view(Ly, pages, -1)
    page[y0, x0] = page[y1, x1]
    if "bounds" in s:
        s["bounds"][y0, x0] = s["bounds"][y1, x1]
    held = torch.arange(s["page_table"].shape[-1], device=DEV) < ((s["len"] + PAGE - 1) // PAGE)[..., None]
    moved = to[torch.arange(Ly, device=DEV)[:, None, None, None], s["page_table"].long().clamp(min=0)]
    s["page_table"].copy_(torch.where(held, moved.int(), s["page_table"]))
    s["stack"].copy_(torch.where(ids < top, pages - 1 - ids, s["stack"]))
    s["used"].copy_(used.flatten())
    return dict(_state(s), used=s["used"])


def _work_cache(case):
    """Expected bytes: live pages read once and written once per copy, with their tables and positions."""
    H, _, d = SHAPES[case["shape"]]
    S, tile, maxp, pages = _cache_size(case)
    ctx = case["context"] * 7 // 8
    kept = min(ctx, case["window"]) + max(0, ctx - case["window"]) * (1 - case["evict"])
    heads = case["layers"] * H
    if case["kind"] == "fork":
        n, copies = case["prompts"], case["prompts"] * case["copies"]
        row = kept / 32 * tile + 4 * kept + 4 * case["window"] + 4 * kept / PAGE
        return {"bytes": heads * (n + copies) * row, "flops": 0}
    share = case["released"] / case["seqs"]
    live = heads * (case["seqs"] - case["released"]) * kept / PAGE
    scatter = 1 - live / (case["layers"] * pages)                    # chance that a live page lies past the live count
    return {"bytes": 2 * live * max(share, scatter) * (PAGE // 32) * tile + 8 * case["layers"] * pages, "flops": 0}


# ---------------------------------------------------------------------------

def prepare(case, seed):
    kind = case["kind"]
    if kind in ("rope", "rope_bwd"):
        return _prepare_rope(case, seed)
    if kind in ("window", "window_step"):
        return _prepare_window(case, seed)
    return _prepare_cache(case, seed)


def run(s):
    kind = s["case"]["kind"]
    if kind in ("rope", "rope_bwd"):
        return _run_rope(s)
    if kind in ("window", "window_step"):
        return _run_window(s)
    return _run_fork(s) if kind == "fork" else _run_compact(s)


def work(case):
    kind = case["kind"]
    if kind in ("rope", "rope_bwd"):
        return _work_rope(case)
    return _work_window(case) if kind in ("window", "window_step") else _work_cache(case)


def exact(case, seed):
    """Copies have no computed values."""
    if case["kind"] in ("rope", "rope_bwd"):
        return _exact_rope(case, seed)
    return _exact_window(case, seed) if case["kind"] in ("window", "window_step") else None
