"""Token sampling on the GPU against its definition: tokens equal, log-probabilities
to the last bits of float32."""
import math

import numpy as np
import pytest

import oracle

pytestmark = pytest.mark.gpu


def run(x, dtype="f32", temperature=None, top_k=None, top_p=None, min_p=None, u=None, cfg=None, stride=None, offset=0,
        logprobs=True):
    import torch
    from paper_2506_05345_amd import dms
    rows, vocab = x.shape
    kind = torch.float32 if dtype == "f32" else torch.bfloat16
    wide = torch.full((rows, (stride or vocab) + offset), 50.0, dtype=kind, device="cuda")
    wide[:, offset:offset + vocab] = torch.from_numpy(x).cuda().to(kind)
    logits = wide[:, offset:offset + vocab]
    c = dms.make_sample_config(vocab, dms.DMS_TYPE_F32 if dtype == "f32" else dms.DMS_TYPE_BF16, **(cfg or {}))
    of = lambda v, t: None if v is None else torch.as_tensor(np.asarray(v), dtype=t, device="cuda")
    f32 = torch.float32
    tokens = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
    logp = torch.full((rows,), -7.0, device="cuda") if logprobs else None
    ws = torch.full((dms.dms_sample_workspace(c, rows),), 0xA5, dtype=torch.uint8, device="cuda")
    dms.dms_sample(c, rows, logits, of(temperature, f32), of(top_k, torch.int32), of(top_p, f32), of(min_p, f32),
                   of(u, f32), tokens, logp, ws)
    return logits.float().cpu().numpy(), tokens.cpu().numpy(), logp.cpu().numpy() if logprobs else None


def check(x, u, got, temperature, top_k, top_p, min_p):
    """Log-probabilities: z and the log of the sum are float64 and their difference is rounded once, half a step of 2^-24
    relative; an error of the sum, at most 2^-40 with weights of 2^-43, and of float64's last bits are far below it."""
    _, tokens, logp = got
    for r in range(len(x)):
        tok, lp = oracle.sample_token(x[r], temperature[r], int(top_k[r]), top_p[r], min_p[r], u[r])
        assert tokens[r] == tok, (r, tokens[r], tok, temperature[r], top_k[r], top_p[r], min_p[r], u[r])
        if logp is not None:
            assert math.isnan(lp) == math.isnan(logp[r])
            if not math.isnan(lp):
                assert abs(logp[r] - lp) <= 2.0 ** -24 * abs(lp) + 1e-10, (r, logp[r], lp)


def mixed(rng, rows):
    pick = lambda *v: rng.choice(np.array(v), rows)
    return (pick(0.0, 0.3, 0.7, 1.0, 2.0, -1.0), pick(0, 0, 1, 3, 40, 5000, -3), pick(1.0, 1.0, 0.95, 0.5, 0.1, 0.0, 2.0),
            pick(0.0, 0.0, 0.05, 0.5, 1.0, 3.0))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [1, 2, 63, 64, 65, 1000, 1025, 4099, 32001])
def test_rows_with_settings_of_their_own(vocab, dtype):
    rng = np.random.default_rng(vocab)
    rows = 60 if vocab < 5000 else 24
    x = (rng.normal(size=(rows, vocab)) * rng.choice([0.3, 2.0, 6.0], (rows, 1))).astype(np.float32)
    T, k, p, m = mixed(rng, rows)
    u = rng.random(rows).astype(np.float32)
    got = run(x, dtype, T, k, p, m, u)
    check(got[0], u, got, T, k, p, m)


@pytest.mark.parametrize("what", ["k", "p", "min", "kp", "none"])
def test_settings_of_the_configuration(what):
    rng = np.random.default_rng(1)
    rows, vocab = 20, 5003
    x = (rng.normal(size=(rows, vocab)) * 2).astype(np.float32)
    cfg = dict(temperature=0.8, top_k=37 if "k" in what else 0, top_p=0.9 if "p" in what else 1.0,
               min_p=0.02 if what == "min" else 0.0)
    u = rng.random(rows).astype(np.float32)
    got = run(x, cfg=cfg, u=u)
    full = lambda v: np.full(rows, v)
    check(got[0], u, got, full(0.8), full(cfg["top_k"]), full(cfg["top_p"]), full(cfg["min_p"]))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("stride,offset", [(1003, 0), (1008, 1), (1004, 2), (1000, 3), (4096, 8)])
def test_rows_of_wider_tensors(stride, offset, dtype):
    """Rows that begin anywhere: no alignment but an element's; what lies between rows is not read as logits."""
    rng = np.random.default_rng(stride)
    rows, vocab = 12, 1000
    x = rng.normal(size=(rows, vocab)).astype(np.float32)
    T, k, p, m = mixed(rng, rows)
    u = rng.random(rows).astype(np.float32)
    got = run(x, dtype, T, k, p, m, u, stride=stride, offset=offset)
    check(got[0], u, got, T, k, p, m)


@pytest.mark.parametrize("vocab", [7, 5000, 40000])
def test_equal_logits_are_cut_by_index(vocab):
    rng = np.random.default_rng(3)
    rows = 16
    x = np.zeros((rows, vocab), np.float32)
    x[1::2] = rng.integers(0, 3, (rows // 2, vocab))           # three values, many equal
    x[::2, ::2] = -0.0                                         # equals 0
    T = np.full(rows, 1.0)
    k = rng.choice([0, 3, vocab // 2, vocab - 1], rows)
    p = rng.choice([1.0, 0.5, 0.25, 0.9], rows)
    m = rng.choice([0.0, 0.1, 0.2], rows)
    for u in (np.zeros(rows), rng.random(rows), np.full(rows, 1 - 2.0 ** -24)):
        u = u.astype(np.float32)
        got = run(x, "f32", T, k, p, m, u)
        check(got[0], u, got, T, k, p, m)


def test_special_values():
    """-inf (masked), NaN, +inf, the type's lowest value, rows without a token, and numbers outside [0, 1)."""
    rng = np.random.default_rng(4)
    low = np.finfo(np.float32).min
    x = rng.normal(size=(14, 300)).astype(np.float32)
    x[0] = -np.inf
    x[1] = np.nan
    x[2, :] = -np.inf
    x[2, 177] = 3
    x[3, ::2] = -np.inf
    x[4, ::3] = np.nan
    x[5, 10] = np.inf
    x[6, [20, 30]] = np.inf
    x[7] = low
    x[8, 1:] = low
    x[9, 5:] = -np.inf
    x[10] = np.finfo(np.float32).max
    x[11] = np.float32(1e-45)
    T = np.full(14, 0.9)
    k, p, m = np.zeros(14, int), np.ones(14), np.zeros(14)
    p[[3, 4, 9]] = 0.8
    k[[4, 5, 12]] = 9
    u = rng.random(14).astype(np.float32)
    u[12], u[13] = 5.0, -1.0
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)
    assert got[1][0] == -1 and got[1][1] == -1 and got[1][2] == 177
    nan = np.full(14, np.nan)
    got = run(x, "f32", nan, None, nan, nan, nan)               # greedy, no cuts
    check(x, np.zeros(14), got, nan, k * 0, nan, nan)


def test_extreme_temperatures():
    rng = np.random.default_rng(5)
    x = rng.normal(size=(8, 2000)).astype(np.float32)
    T = np.array([1e-38, 1e-45, 1e-6, 100.0, 1e30, 3e38, 1.0, 0.01])
    u = rng.random(8).astype(np.float32)
    k, p, m = np.array([0, 0, 5, 0, 0, 7, 0, 0]), np.array([1, 1, 1, 0.9, 0.5, 1, 0.3, 1.0]), np.zeros(8)
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)


def test_large_vocabularies_and_numbers_at_the_borders():
    rng = np.random.default_rng(6)
    vocab = 1 << 20
    x = (rng.normal(size=(3, vocab)) * 3).astype(np.float32)
    T, k, p, m = np.array([1.0, 0.7, 2.5]), np.array([0, 3000, 0]), np.array([1.0, 0.99, 0.95]), np.zeros(3)
    u = np.array([0.5, 1 - 2.0 ** -24, 0.0], np.float32)
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)


def test_distribution():
    """4000 draws of one row: frequencies within 5 standard deviations of the definition's probabilities."""
    rng = np.random.default_rng(7)
    x = np.tile((rng.normal(size=(1, 50))).astype(np.float32), (4000, 1))
    u = rng.random(4000).astype(np.float32)
    _, tokens, logp = run(x, cfg=dict(temperature=0.8, top_k=20), u=u)
    z = x[0].astype(np.float64) / np.float32(0.8)
    keep = np.argsort(-z)[:20]
    prob = np.zeros(50)
    prob[keep] = np.exp(z[keep]) / np.exp(z[keep]).sum()
    freq = np.bincount(tokens, minlength=50)
    assert (np.abs(freq - 4000 * prob) <= 5 * np.sqrt(4000 * prob * (1 - prob)) + 1e-9).all()
    assert np.abs(np.exp(logp.astype(np.float64)) - prob[tokens]).max() <= 1e-6


def test_log_probabilities_may_be_left_out_and_streams_differ():
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(8)
    x = rng.normal(size=(5, 3001)).astype(np.float32)
    u = rng.random(5).astype(np.float32)
    a = run(x, u=u, cfg=dict(top_p=0.9))
    b = run(x, u=u, cfg=dict(top_p=0.9), logprobs=False)
    assert np.array_equal(a[1], b[1])
    c = dms.make_sample_config(3001, top_p=0.9)
    stream = torch.cuda.Stream()
    logits, ud = torch.from_numpy(x).cuda(), torch.from_numpy(u).cuda()
    tokens = torch.empty(5, dtype=torch.int32, device="cuda")
    ws = torch.empty(dms.dms_sample_workspace(c, 5), dtype=torch.uint8, device="cuda")
    stream.wait_stream(torch.cuda.current_stream())
    dms.dms_sample(c, 5, logits, None, None, None, None, ud, tokens, None, ws, stream=stream)
    torch.cuda.synchronize()
    assert np.array_equal(tokens.cpu().numpy(), a[1])


@pytest.mark.parametrize("vocab", [257, 4500])
def test_more_rows_than_run_at_once(vocab):
    rng = np.random.default_rng(9)
    rows = 1030
    x = (rng.normal(size=(rows, vocab)) * 2).astype(np.float32)
    T, k, p, m = mixed(rng, rows)
    u = rng.random(rows).astype(np.float32)
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)


@pytest.mark.parametrize("vocab,values", [(4097, 1), (9000, 3), (50001, 7)])
def test_few_distinct_logits(vocab, values):
    """Thousands of equal logits at every border."""
    rng = np.random.default_rng(vocab)
    rows = 24
    x = rng.choice(np.linspace(-1.0, 1.0, values), (rows, vocab)).astype(np.float32)
    T, _, p, m = mixed(rng, rows)
    k = rng.choice([0, 1, vocab // 3, vocab - 1, vocab, 3500], rows)
    u = rng.random(rows).astype(np.float32)
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)


def test_many_kept_tokens_at_low_temperatures():
    rng = np.random.default_rng(10)
    rows, vocab = 12, 30000
    x = (rng.normal(size=(rows, vocab)) * 3).astype(np.float32)
    T = np.array([0.02, 0.05, 0.1, 0.2] * 3)
    k, p = np.array([1000] * 6 + [0] * 3 + [20000] * 3), np.array([0.95, 0.999999, 1.0] * 4)
    m = np.zeros(rows)
    u = (1 - 2.0 ** -rng.integers(1, 25, rows)).astype(np.float32)
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)


def test_numbers_at_the_borders_of_equal_tokens():
    """2^k equal tokens: token j from u = j 2^-k on."""
    rows = 64
    x = np.full((rows, 64), -np.inf, np.float32)
    x[:, ::2] = 1.5
    u = (np.arange(rows) / 64).astype(np.float32)
    _, tokens, logp = run(x, u=u)
    assert np.array_equal(tokens, 2 * (np.arange(rows) // 2))
    assert np.allclose(logp, -np.log(32), atol=1e-6)
    below = np.nextafter(u[2:], np.float32(0))
    _, tokens, _ = run(x[2:], u=below)
    assert np.array_equal(tokens, 2 * (np.ceil(u[2:] * 32).astype(int) - 1))


@pytest.mark.parametrize("vocab", [4100, 20000])
def test_top_k_past_half_the_vocabulary_and_small_nuclei(vocab):
    rng = np.random.default_rng(vocab + 1)
    rows = 40
    x = (rng.normal(size=(rows, vocab)) * 3).astype(np.float32)
    T = rng.choice([0.7, 1.0, 3.0], rows)
    k = rng.choice([500, 1024, 1025, 2050, vocab - 5], rows)
    p = rng.choice([1.0, 1.0, 0.5, 0.99], rows)
    m = rng.choice([0.0, 0.0, 0.01], rows)
    u = rng.random(rows).astype(np.float32)
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)


def test_few_tokens_left_by_a_mask():
    """Rows of -inf and of the type's lowest value but for a few tokens, with cuts at, above and below their number."""
    rng = np.random.default_rng(12)
    rows, vocab = 48, 9001
    x = np.full((rows, vocab), -np.inf, np.float32)
    x[::3] = np.finfo(np.float32).min
    x[2::3] = -1e9
    for r in range(rows):
        at = rng.choice(vocab, 5, replace=False)
        x[r, at] = rng.normal(size=5)
    k, p, m = rng.choice([0, 1, 4, 5, 6, 300, 6000], rows), rng.choice([1.0, 0.4, 0.999], rows), rng.choice([0.0, 0.3], rows)
    T = np.ones(rows)
    u = rng.random(rows).astype(np.float32)
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)


def test_sorted_logits():
    """The largest tokens side by side."""
    rng = np.random.default_rng(13)
    rows, vocab = 12, 33000
    x = -np.sort(-rng.normal(size=(rows, vocab)) * 3, axis=1).astype(np.float32)
    k, p, m = rng.choice([20, 200, 900], rows), np.ones(rows), np.zeros(rows)
    u = rng.random(rows).astype(np.float32)
    got = run(x, "f32", np.ones(rows), k, p, m, u)
    check(x, u, got, np.ones(rows), k, p, m)


def test_rows_far_apart():
    """Rows 2^30 logits apart: offsets past 32 bits."""
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(14)
    vocab = 9000
    x = (rng.normal(size=(3, vocab)) * 3).astype(np.float32)
    wide = torch.empty(2 * (1 << 30) + vocab, dtype=torch.bfloat16, device="cuda")
    logits = wide.as_strided((3, vocab), (1 << 30, 1))
    logits.copy_(torch.from_numpy(x))
    c = dms.make_sample_config(vocab, dms.DMS_TYPE_BF16, top_p=0.9, temperature=0.8)
    u = torch.tensor([0.1, 0.5, 0.9], device="cuda")
    tokens, logp = torch.empty(3, dtype=torch.int32, device="cuda"), torch.empty(3, device="cuda")
    ws = torch.empty(dms.dms_sample_workspace(c, 3), dtype=torch.uint8, device="cuda")
    dms.dms_sample(c, 3, logits, None, None, None, None, u, tokens, logp, ws)
    held = logits.float().cpu().numpy()
    one = lambda v: np.full(3, v)
    check(held, u.cpu().numpy(), (held, tokens.cpu().numpy(), logp.cpu().numpy()), one(np.float32(0.8)), one(0), one(np.float32(0.9)),
          one(0.0))


@pytest.mark.parametrize("spread", [1e-4, 0.02, 0.5, 2.0])
def test_flat_rows(spread):
    """Logits close to each other: many tokens to a share of the weight, with and without masked ones far below."""
    rng = np.random.default_rng(15)
    rows, vocab = 24, 60000
    x = (rng.normal(size=(rows, vocab)) * spread).astype(np.float32)
    x[::4, 1000:50000] = -np.inf
    x[1::4, :100] = -1e6
    T, _, p, m = mixed(rng, rows)
    T = np.where(T <= 0, 1.7, T)
    k = rng.choice([0, 0, 0, 2000, 40000], rows)
    u = rng.random(rows).astype(np.float32)
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)


@pytest.mark.parametrize("vocab", [300, 5003])
def test_signalling_nan(vocab):
    rng = np.random.default_rng(16)
    x = (rng.normal(size=(8, vocab)) * 2).astype(np.float32)
    bits = x.view(np.uint32)
    for r in range(8):
        bits[r, rng.choice(vocab, 200, replace=False)] = [0x7F800001, 0xFF800001, 0x7FC00000, 0xFFFFFFFF][r % 4]
    T, k, p, m = np.ones(8), np.array([0, 5, 0, 1000] * 2), np.array([1.0, 0.9] * 4), np.zeros(8)
    u = rng.random(8).astype(np.float32)
    got = run(x, "f32", T, k, p, m, u)
    check(x, u, got, T, k, p, m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [4099, 5003, 30000])
def test_top_k_that_ends_among_tokens_without_weight(vocab, dtype):
    """2000 tokens with a weight, 1000 that lie 44 to 45 octaves below the largest and weigh nothing, others further
    below; the k-th one before, at, among and past the weightless, without top-p: a border whose bin lists nothing."""
    rng = np.random.default_rng(vocab + 17)
    rows = 16
    z = np.concatenate([[0.0], rng.uniform(0.5, 43.4, 1999), rng.uniform(44.3, 44.7, 1000),
                        rng.uniform(46, 60, vocab - 3000)])
    x = np.stack([rng.permutation(-z) for _ in range(rows)])
    x[::4] = -z[::-1]                                   # the largest last
    x = (x * math.log(2.0)).astype(np.float32)
    k = np.array([1999, 2000, 2001, 2400, 2500, 2999, 3000, 3001] * 2)
    m = np.where(np.arange(rows) < 8, 0.0, 1e-3)
    u = rng.random(rows).astype(np.float32)
    u[[0, 3, 4]] = 0.0
    one = np.ones(rows)
    got = run(x, dtype, one, k, one, m, u)
    check(got[0], u, got, one, k, one, m)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("vocab", [300, 5003, 30000])
def test_min_p_among_weights_of_few_units(vocab, dtype):
    """min-p of 1e-14 to 1e-10: weights are rounded to integers before they are compared.  Tokens in the order of their
    weights, the largest last, and u = 0: the first token kept is the one taken."""
    rng = np.random.default_rng(vocab + 18)
    m = np.array([1e-14, 5e-14, 1e-13, 1.2e-13, 2e-13, 3e-13, 1e-12, 4e-12, 7e-12, 8e-12, 1e-11, 1e-10])
    rows = 3 * len(m)
    z = np.sort(rng.uniform(33.5, 44.6, (rows, vocab)))[:, ::-1].copy()
    z[:, -1] = 0
    x = (-z * math.log(2.0)).astype(np.float32)
    m = np.tile(m, 3)
    k = np.repeat([0, vocab - 9, 7 * vocab // 8], len(m))
    one, u = np.ones(rows), np.zeros(rows, np.float32)
    got = run(x, dtype, one, k, one, m, u)
    check(got[0], u, got, one, k, one, m)


@pytest.mark.parametrize("vocab", [1000, 5003])
def test_tensors_wider_than_the_vocabulary(vocab):
    """Logits of a padded output layer, whole: rows begin where the tensor's own rows do.  Flat tensors are rows of the
    vocabulary; narrower rows are refused."""
    import torch
    from paper_2506_05345_amd import dms
    rng = np.random.default_rng(vocab + 19)
    rows, wide = 12, vocab + 137
    x = (rng.normal(size=(rows, vocab)) * 2).astype(np.float32)
    u = rng.random(rows).astype(np.float32)
    want = [oracle.sample_token(x[r], 0.8, 0, 0.9, 0.0, u[r])[0] for r in range(rows)]
    cfg = dms.make_sample_config(vocab, temperature=0.8, top_p=0.9)
    ws = torch.empty(dms.dms_sample_workspace(cfg, rows), dtype=torch.uint8, device="cuda")
    ud = torch.from_numpy(u).cuda()
    padded = torch.full((rows, wide), 50.0, device="cuda")
    padded[:, :vocab] = torch.from_numpy(x)
    dense = padded[:, :vocab].contiguous()
    wider = torch.full((rows, wide + 5), 50.0, device="cuda")
    wider[:, 2:2 + wide] = padded

    def tokens(logits, count=rows, **kw):
        out = torch.full((rows,), -7, dtype=torch.int32, device="cuda")
        dms.dms_sample(cfg, count, logits, None, None, None, None, ud, out, None, ws, **kw)
        return out[:count].tolist()

    assert tokens(padded) == tokens(padded, row_stride=wide) == want
    assert tokens(padded.view(3, 4, wide)) == tokens(padded.view(rows, 1, wide)) == want
    assert tokens(wider[:, 2:2 + wide]) == tokens(padded[:, :vocab]) == tokens(padded.view(-1), row_stride=wide) == want
    assert tokens(dense) == tokens(dense.view(-1)) == tokens(dense.view(4, 3, vocab)) == want
    assert tokens(padded[:0], 0) == tokens(padded[:0, :7], 0) == tokens(padded[0, :0], 0) == []
    assert tokens(padded[:5], 5) == tokens(padded, 5) == want[:5]
    assert tokens(padded[3], 1) == [oracle.sample_token(x[3], 0.8, 0, 0.9, 0.0, u[0])[0]]
    narrow = torch.zeros((2 * rows, vocab - 1), device="cuda")
    for logits in (narrow, narrow.view(rows, 2 * vocab - 2)[:, ::2], padded.t().contiguous().t(), padded[:rows - 1]):
        with pytest.raises(dms.DmsError):
            tokens(logits)


SETTINGS = {
    "none": dict(), "k": dict(k=9), "many": dict(k=3000), "p": dict(p=0.8), "min": dict(m=0.1),
    "kp": dict(k=3000, p=0.8), "all": dict(k=20, p=0.9, m=0.05),
}


def among_others(rng, special, vocab, **fixed):
    """Special rows with an ordinary one before and after each, and settings for all of them."""
    x = (rng.normal(size=(2 * len(special) + 1, vocab)) * 2).astype(np.float32)
    x[1::2] = special
    rows = len(x)
    return x, np.full(rows, fixed.get("k", 0)), np.full(rows, fixed.get("p", 1.0)), np.full(rows, fixed.get("m", 0.0)), \
        rng.random(rows).astype(np.float32)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", SETTINGS)
@pytest.mark.parametrize("vocab", [5003, 20000])
def test_special_values_of_rows_in_parts(vocab, what, dtype):
    """Masked, NaN, infinite, lowest, largest and smallest logits in the launches of large vocabularies, between ordinary
    rows of the same call."""
    rng = np.random.default_rng(vocab + len(what))
    low, most = (np.finfo(np.float32).min, np.finfo(np.float32).max) if dtype == "f32" else (-3.3895314e38, 3.3895314e38)
    x = rng.normal(size=(16, vocab)).astype(np.float32)
    x[0] = -np.inf
    x[1] = np.nan
    x[2] = -np.inf
    x[2, vocab - 3] = 3
    x[3, ::2] = -np.inf
    x[4, ::3] = np.nan
    x[5, 4100] = np.inf
    x[6, [20, 4500]] = np.inf
    x[7] = low
    x[8, 1:] = low
    x[9, 5:] = -np.inf
    x[10] = most
    x[11] = np.float32(1e-45) if dtype == "f32" else 0
    x[12, ::2] = np.nan
    x[12, 1::2] = -np.inf
    x[12, 4098] = low
    x[13] = np.where(rng.random(vocab) < 0.5, low, most)
    x[14] = rng.normal(size=vocab) * 1e-38              # denormal, most of them
    x[15, :4099] = np.inf
    x, k, p, m, u = among_others(rng, x, vocab, **SETTINGS[what])
    u[3::4], u[1] = 5.0, -1.0
    T = np.full(len(x), 0.9)
    got = run(x, dtype, T, k, p, m, u)
    check(got[0], u, got, T, k, p, m)
    assert got[1][1] == -1 and got[1][3] == -1 and got[1][5] == vocab - 3
    nan = np.full(len(x), np.nan)
    got = run(x, dtype, nan, None, nan, nan, nan)       # greedy, no cuts
    check(got[0], np.zeros(len(x)), got, nan, k * 0, nan, nan)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("what", SETTINGS)
@pytest.mark.parametrize("vocab", [5003, 20000])
def test_extreme_temperatures_of_rows_in_parts(vocab, what, dtype):
    rng = np.random.default_rng(vocab + len(what) + 1)
    T = np.array([1e-38, 1e-45, 1e-6, 0.01, 100.0, 1e30, 3e38, np.inf])
    x, k, p, m, u = among_others(rng, rng.normal(size=(len(T), vocab)), vocab, **SETTINGS[what])
    x[1::2, ::7] = -np.inf
    T = np.concatenate([[1.0], np.stack([T, np.ones(len(T))], 1).ravel()])
    got = run(x, dtype, T, k, p, m, u)
    check(got[0], u, got, T, k, p, m)


@pytest.mark.parametrize("vocab", [30011, 262144])
def test_flat_rows_with_a_few_large_logits(vocab):
    """Eight logits far above the rest of a flat row: thousands of tokens within a bin of the border, which no list holds."""
    rng = np.random.default_rng(vocab + 20)
    T, p = np.array([0.6, 1.0, 1.0, 1.7, 1.7, 1.0]), np.array([0.3, 0.8, 0.95, 0.5, 0.95, 0.9])
    rows = len(T)
    x = (rng.normal(size=(rows, vocab)) * 0.5).astype(np.float32)
    for r in range(rows):
        x[r, rng.choice(vocab, 8, replace=False)] += 6
    k, m = np.array([0, 0, 0, 0, 0, vocab // 3]), np.zeros(rows)
    u = rng.random(rows).astype(np.float32)
    got = run(x, "f32", T, k, p, m, u)
    check(got[0], u, got, T, k, p, m)
