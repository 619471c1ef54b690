"""GPU parity of the rotary positions (several axes, decision neurons taken
before the rotation) against the float64 oracle.

Tolerance of a rotated element, for inputs x1, x2 of its pair: the angle's
fraction of a turn is rounded to float32 (at most 2^-26 turns = 9.4e-8), sine
and cosine and their product with the factor are within 2.5e-7, two products and
a sum within 1.8e-7 of |x1| + |x2|: 6e-7 (|x1| + |x2|) factor in all; a bf16
output adds half a step, 2^-8 of its value."""
import numpy as np
import pytest

import dms_synth as sy
import oracle

pytestmark = pytest.mark.gpu


def _case(T, H, g, d, rot, sections, off=0, interleaved=False, adjacent=False, tin="bf16", tout="bf16", borrow=True,
          factor=1.0, fused=True, far=0):
    return dict(T=T, H=H, g=g, d=d, rot=rot, sections=sections, off=off, interleaved=interleaved, adjacent=adjacent,
                tin=tin, tout=tout, borrow=borrow, factor=factor, fused=fused, far=far)


CASES = [
    _case(1, 1, 1, 64, 64, [32]),
    _case(3, 2, 6, 128, 128, [64], far=131000),
    _case(130, 8, 5, 128, 128, [16, 24, 24]),
    _case(65, 4, 7, 128, 128, [22, 21, 21], interleaved=True, adjacent=True, fused=False),
    _case(50, 2, 2, 64, 32, [4, 4, 4, 4], off=16, tout="f32", factor=1.3),
    _case(41, 1, 16, 576, 64, [32], off=512, borrow=False),
    _case(41, 1, 16, 576, 64, [20, 12], off=512, adjacent=True, borrow=True),
    _case(33, 3, 4, 80, 48, [10, 14], tin="f32", tout="f32", far=2 ** 31 - 200),
    _case(29, 2, 3, 96, 96, [24, 24], tin="f32", interleaved=True),
    _case(17, 1, 2, 6, 2, [1], off=3, adjacent=True),            # odd sizes: one element at a time
    _case(19, 2, 2, 36, 20, [3, 7], off=8, tout="f32"),
    _case(700, 2, 6, 128, 128, [64], fused=False, borrow=False),
    _case(33000, 4, 4, 36, 20, [3, 7], off=8),                   # more elements than a grid has threads
    _case(12, 2, 2, 1024, 512, [256], off=256),
    _case(2100, 1, 2, 64, 64, [12, 10, 10], interleaved=True, adjacent=True),
]


def _values(rng, shape, kind):
    x = rng.normal(0, 2, shape).astype(np.float32)
    return sy.bf16_bits_to_f32_np(sy.f32_to_bf16_bits_np(x)) if kind == "bf16" else x


def _setup(c, seed):
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(seed)
    T, A = c["T"], len(c["sections"])
    pos = rng.integers(-50, 5000, (A, T)) + c["far"]
    pos = np.minimum(pos, 2 ** 31 - 1)
    inv = 1e4 ** (-np.arange(c["rot"] // 2) / (c["rot"] // 2))
    types = {"bf16": dms.DMS_TYPE_BF16, "f32": dms.DMS_TYPE_F32}
    cfg = dms.make_rope_config(c["H"], c["g"], c["d"], c["rot"], c["sections"], c["off"], int(c["interleaved"]),
                               int(c["adjacent"]), types[c["tin"]], types[c["tout"]], int(c["borrow"]), -1.5,
                               c["factor"])
    return rng, pos, inv, cfg, torch.from_numpy(pos.astype(np.int32)).cuda(), torch.from_numpy(inv).cuda()


def _turn(c, x, pos, inv, back=False):
    axes = oracle.rope_axes(c["sections"], c["interleaved"])
    a = (pos, inv, axes, c["rot"], c["off"], c["adjacent"])
    y = oracle.rope_rotate(x, *a, c["factor"], back)
    # |x1| + |x2| of each element's pair: rotations by no angle of absolute values
    z = np.abs(np.asarray(x, np.float64))
    half, off = c["rot"] // 2, c["off"]
    i = np.arange(half)
    lo = off + (2 * i if c["adjacent"] else i)
    hi = lo + (1 if c["adjacent"] else half)
    tol = np.zeros_like(z)
    tol[..., lo] = tol[..., hi] = 6e-7 * c["factor"] * (z[..., lo] + z[..., hi])
    if c["tout"] == "bf16":
        tol += 2.0 ** -8 * (np.abs(y) + tol)
    return y, tol


@pytest.mark.parametrize("i", range(len(CASES)))
def test_forward(i):
    import torch
    from paper_2506_05345_amd import dms
    c = CASES[i]
    rng, pos, inv, cfg, pd, fd = _setup(c, i)
    T, H, Hq, d = c["T"], c["H"], c["H"] * c["g"], c["d"]
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}
    rows = _values(rng, (T, Hq + 2 * H, d), c["tin"])
    dev = torch.from_numpy(rows).cuda().to(dt[c["tin"]])
    q, k = dev[:, :Hq], dev[:, Hq:Hq + H]
    if not c["fused"]:
        q, k = q.contiguous(), k.contiguous()
    qo = torch.full((T, Hq, d), float("nan"), device="cuda", dtype=dt[c["tout"]])
    ko = torch.full((T, H, d), float("nan"), device="cuda", dtype=dt[c["tout"]])
    lo = torch.full((T, H), float("nan"), device="cuda")
    de = torch.full((T, H), 7, device="cuda", dtype=torch.uint8)
    dms.dms_rope_fwd(cfg, T, q, k, pd, fd, qo, ko, *((lo, de) if c["borrow"] else (None, None)))
    torch.cuda.synchronize()
    assert torch.equal(dev.float().cpu(), torch.from_numpy(rows))       # inputs untouched
    rq = rows[:, :Hq].astype(np.float64)
    if c["borrow"]:
        logits, rq = oracle.rope_borrow(rq, c["g"])
        assert np.array_equal(lo.double().cpu().numpy(), logits)
        want = (logits.astype(np.float32) + np.float32(-1.5)) > 0
        assert np.array_equal(de.cpu().numpy(), want.astype(np.uint8))
    for got, x in ((qo, rq), (ko, rows[:, Hq:Hq + H])):
        y, tol = _turn(c, x, pos, inv)
        off = np.abs(got.double().cpu().numpy() - y)
        assert (off <= tol).all(), (i, float((off - tol).max()))
    # one of the two alone, the same bits
    q2, k2 = torch.full_like(qo, float("nan")), torch.full_like(ko, float("nan"))
    dms.dms_rope_fwd(cfg, T, q, None, pd, fd, q2, None)
    dms.dms_rope_fwd(cfg, T, None, k, pd, fd, None, k2)
    torch.cuda.synchronize()
    assert torch.equal(q2, qo) and torch.equal(k2, ko)


@pytest.mark.parametrize("i", range(len(CASES)))
def test_backward(i):
    import torch
    from paper_2506_05345_amd import dms
    c = CASES[i]
    rng, pos, inv, cfg, pd, fd = _setup(c, 100 + i)
    T, H, Hq, d = c["T"], c["H"], c["H"] * c["g"], c["d"]
    dt = {"bf16": torch.bfloat16, "f32": torch.float32}
    dq, dk = _values(rng, (T, Hq, d), c["tin"]), _values(rng, (T, H, d), c["tin"])
    dl = rng.normal(size=(T, H)).astype(np.float32)
    rows = torch.full((T, Hq + 2 * H, d), 3.0, device="cuda", dtype=dt[c["tout"]])
    qo, ko = rows[:, :Hq], rows[:, Hq:Hq + H]
    if not c["fused"]:
        qo, ko = torch.full_like(qo, 3.0).contiguous(), torch.full_like(ko, 3.0).contiguous()
    for dlogits in ((dl, None) if c["borrow"] else (None,)):
        dms.dms_rope_bwd(cfg, T, torch.from_numpy(dq).cuda().to(dt[c["tin"]]), torch.from_numpy(dk).cuda().to(dt[c["tin"]]),
                         pd, fd, None if dlogits is None else torch.from_numpy(dl).cuda(), qo, ko)
        torch.cuda.synchronize()
        for got, x, isq in ((qo, dq, True), (ko, dk, False)):
            y, tol = _turn(c, x, pos, inv, back=True)
            if isq and c["borrow"]:
                y[:, ::c["g"], 0] = 0 if dlogits is None else dl
                tol[:, ::c["g"], 0] = 2.0 ** -8 * np.abs(y[:, ::c["g"], 0]) if c["tout"] == "bf16" else 0
            off = np.abs(got.double().cpu().numpy() - y)
            assert (off <= tol).all(), (i, float((off - tol).max()))
    if c["fused"]:                                                       # between the rows nothing is written
        assert (rows[:, Hq + H:] == 3.0).all()


@pytest.mark.parametrize("adjacent", [False, True])
def test_gradient_against_differences(adjacent):
    """The rotation is linear: <R x + R e, y> - <R x, y> = <e, R^T y> in float32 outputs."""
    import torch
    from paper_2506_05345_amd import dms
    c = _case(9, 2, 3, 64, 48, [10, 14], off=16, adjacent=adjacent, tin="f32", tout="f32")
    rng, pos, inv, cfg, pd, fd = _setup(c, 7)
    x, e, y = (torch.from_numpy(rng.normal(size=(9, 6, 64)).astype(np.float32)).cuda() for _ in range(3))

    def turn(v):
        out = torch.empty_like(v)
        logits = torch.empty((9, 2), device="cuda")
        dms.dms_rope_fwd(cfg, 9, v, None, pd, fd, out, None, logits)
        return out.double(), logits.double()

    dl = torch.from_numpy(rng.normal(size=(9, 2)).astype(np.float32)).cuda()
    back = torch.empty_like(y)
    dms.dms_rope_bwd(cfg, 9, y, None, pd, fd, dl, back, None)
    (a, la), (b, lb) = turn(x + e), turn(x)
    left = float(((a - b) * y.double()).sum() + ((la - lb) * dl.double()).sum())
    right = float((e.double() * back.double()).sum())
    # 6e-7 of |x1| + |x2| an output (test module), twice, against 1152 products of unit size: below 5e-3
    assert abs(left - right) < 5e-3, (left, right)


def test_unaligned_rows_in_place_and_empty():
    import torch
    from paper_2506_05345_amd import dms
    c = _case(37, 2, 3, 64, 64, [32])
    rng, pos, inv, cfg, pd, fd = _setup(c, 8)
    x = _values(rng, (37, 8, 64), "bf16")
    base = torch.from_numpy(x).cuda().bfloat16()
    want_q, want_k = torch.empty((37, 6, 64), device="cuda", dtype=torch.bfloat16), torch.empty((37, 2, 64), device="cuda", dtype=torch.bfloat16)
    dms.dms_rope_fwd(cfg, 37, base[:, :6], base[:, 6:], pd, fd, want_q, want_k)
    # rows that start at odd elements: 2-byte alignment
    wide = torch.zeros(37 * 521 + 1, device="cuda", dtype=torch.bfloat16)
    rows = wide[1:].view(37, 521)[:, 3:515].view(37, 8, 64)
    rows.copy_(base)
    q, k = torch.empty_like(want_q), torch.empty_like(want_k)
    dms.dms_rope_fwd(cfg, 37, rows[:, :6], rows[:, 6:], pd, fd, q, k)
    torch.cuda.synchronize()
    assert torch.equal(q, want_q) and torch.equal(k, want_k)
    # in place on dense tensors
    q, k = base[:, :6].contiguous(), base[:, 6:].contiguous()
    dms.dms_rope_fwd(cfg, 37, q, k, pd, fd, q, k)
    torch.cuda.synchronize()
    assert torch.equal(q, want_q) and torch.equal(k, want_k)
    # no tokens: nothing is read or written
    dms.dms_rope_fwd(cfg, 0, q, k, pd, fd, q, k)
    torch.cuda.synchronize()
    assert torch.equal(q, want_q)
    # a captured rotation replays
    src = base[:, :6].contiguous()
    out = torch.empty_like(src)
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g):
        dms.dms_rope_fwd(cfg, 37, src, None, pd, fd, out, None)
    for i in range(3):
        src.copy_(base[:, :6] * (i + 1))
        out.fill_(0)
        g.replay()
        torch.cuda.synchronize()
        want = torch.empty_like(src)
        dms.dms_rope_fwd(cfg, 37, src, None, pd, fd, want, None)
        torch.cuda.synchronize()
        assert torch.equal(out, want), i
