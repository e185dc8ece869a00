"""The 4-bit KV cache on the GPU against its plain form in 64 bits
(tests/_kvq.py): bytes of the rows exactly, rows read back to their one
rounding, attention within a bound derived from the arithmetic there."""
import sys

import numpy as np
import pytest
import torch

import paper_2607_28418_amd as W
from tests import _kvq, _kvq_exact

pytestmark = pytest.mark.gpu
HD = 128


def say(*a):
    print("[case]", *a, file=sys.stderr, flush=True)


def d(a):
    return torch.from_numpy(np.ascontiguousarray(a)).cuda()


def i32(a):
    return None if a is None else d(np.asarray(a, np.int32))


def rows_f64(seed, shape, dtype, spread=1.0):
    """Values of `dtype` as fp64: normal with a bias per channel and an uneven size per row."""
    g = np.random.default_rng(seed)
    x = g.normal(size=shape) + 0.7 * g.normal(size=shape[-1:])
    x = x * np.exp(spread * g.normal(size=shape[:-1] + (1,)))
    return torch.from_numpy(x.astype(np.float32)).to(dtype)


def cache_shape(n_seq, L, n_kv, qg, hm):
    return ((n_seq, n_kv, L) if hm else (n_seq, L, n_kv)) + (_kvq.row_bytes(qg),)


def expect_cache(x, cache, n_seq, T, L, n_kv, qg, hm, pos, kv_len):
    rows = _kvq.quantize(x.double().numpy().reshape(n_seq * T, n_kv, HD), qg)
    cache = cache.copy()
    for r, b, p in _kvq.where_rows(n_seq, T, L, pos, kv_len):
        if hm:
            cache[b, :, p] = rows[r]
        else:
            cache[b, p] = rows[r]
    return cache


# ---- writing -----------------------------------------------------------------------

SHAPES = [  # n_seq, T, L, n_kv, pos, kv_len
    (1, 1, 1, 1, None, None),
    (1, 1, 40, 8, [39], None),                             # the last position
    (5, 1, 33, 8, [0, 32, 33, -1, 7], [1, 33, 34, 0, 7]),  # decode: first, last, past the end, before it, past kv_len
    (3, 37, 64, 2, [-20, 0, 50], None),                    # left padding, whole, running into the capacity
    (2, 129, 200, 3, [5, -128], [77, 1]),
    (2, 3, 9, 32, [2 ** 31 - 2, -2 ** 31], None),          # nothing lands
    (1, 300, 256, 5, None, [250]),
]


@pytest.mark.parametrize("hm", [False, True])
@pytest.mark.parametrize("qg", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_bytes(dtype, qg, hm):
    for n, (n_seq, T, L, n_kv, pos, kv_len) in enumerate(SHAPES):
        say("quantize", dtype, qg, hm, SHAPES[n])
        k, v = (rows_f64(10 * n + s, (n_seq * T, n_kv * HD), dtype) for s in (1, 2))
        g = np.random.default_rng(n)
        kc, vc = (g.integers(0, 256, cache_shape(n_seq, L, n_kv, qg, hm), dtype=np.uint8) for _ in range(2))
        kd, vd = d(kc), d(vc)
        out = W.wide_kv_quantize(k.cuda(), v.cuda(), kd, vd, n_kv, HD, qg, pos=i32(pos), kv_len=i32(kv_len),
                                 head_major=hm)
        torch.cuda.synchronize()
        assert out[0] is kd and out[1] is vd
        for got, x, was in ((kd, k, kc), (vd, v, vc)):
            want = expect_cache(x, was, n_seq, T, L, n_kv, qg, hm, pos, kv_len)
            assert np.array_equal(got.cpu().numpy(), want), SHAPES[n]


def special_rows(dtype):
    """Rows where a quantiser goes wrong: ties, constants, extremes of size, not-finite values."""
    g = np.random.default_rng(5)
    x = g.normal(size=(64, HD)).astype(np.float32)
    x[0] = 0.0
    x[1] = -3.25
    x[2] = np.arange(HD) % 31 * 0.5                  # ties of whole codes (scale 1)
    x[3] = np.arange(HD) % 31 * -0.5
    x[4] = np.float32(2.0 ** -133) * (np.arange(HD) % 7)   # subnormal
    x[5] = np.float32(2.0 ** -126) * (np.arange(HD) % 16)
    x[6] = np.float32(1.5e38) * g.uniform(-1, 1, HD).astype(np.float32)
    x[7, 3] = np.nan
    x[8, 127] = np.inf
    x[9, 64] = -np.inf
    x[10, 0] = -2.0 ** 127
    x[11] = 100.0 + 0.01 * g.normal(size=HD)         # a narrow range far from zero
    x[12] = -100.0 - 0.01 * g.normal(size=HD)
    x[13, ::2] = 1e-30                               # far smaller than the range
    x[14, :] = -x[14, 0]
    x[14, 5] = np.nextafter(x[14, 5], np.float32(9))
    x[15] = np.where(np.arange(HD) % 2, 3.0, -3.0) * 2.0 ** 100
    for r in range(16, 40):                          # few-bit values: ties of codes and of scales
        x[r] = g.integers(-40, 41, HD) * 2.0 ** (r - 28)
    return torch.from_numpy(x).to(dtype)


@pytest.mark.parametrize("qg", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_special_rows(dtype, qg):
    x = special_rows(dtype)
    rows = x.shape[0]
    kc = torch.zeros(1, rows, 1, _kvq.row_bytes(qg), dtype=torch.uint8, device="cuda")
    vc = kc.clone()
    W.wide_kv_quantize(x.cuda(), x.flip(0).contiguous().cuda(), kc, vc, 1, HD, qg)
    torch.cuda.synchronize()
    want = _kvq.quantize(x.double().numpy(), qg)
    got = kc.cpu().numpy()[0, :, 0]
    bad = [r for r in range(rows) if not np.array_equal(got[r], want[r])]
    assert not bad, [(r, got[r].tolist(), want[r].tolist()) for r in bad[:2]]
    assert np.array_equal(vc.cpu().numpy()[0, ::-1, 0], want)
    for dt in (torch.float32, torch.bfloat16):
        y = W.wide_kv_dequantize(kc, vc, rows, 1, HD, qg, dtype=dt)[0].cpu()
        ref = torch.from_numpy(_kvq.values(want, qg).astype(np.float32)).to(dt)
        assert torch.equal(torch.isnan(y), torch.isnan(ref))
        assert torch.equal(y.nan_to_num(7.0), ref.nan_to_num(7.0))


@pytest.mark.parametrize("qg", [32, 64, 128])
@pytest.mark.parametrize("spread", [3, 14, 17, 40])
def test_quantize_borders(qg, spread):
    """Values of three bits with exponents far apart: many lie on the border of
    two codes, or miss it by what an fp32 difference does not hold."""
    g = np.random.default_rng(spread)
    rows = 2000
    x = g.integers(-7, 8, (rows, HD)) * 2.0 ** -g.integers(0, spread + 1, (rows, HD))
    x[:, ::7] = g.integers(-15, 16, (rows, x[:, ::7].shape[1])) * 0.25
    for dtype in (torch.bfloat16, torch.float32):
        t = torch.from_numpy(x.astype(np.float32)).to(dtype)
        assert (t.double().numpy() == x).all()
        kc = torch.zeros(1, rows, 1, _kvq.row_bytes(qg), dtype=torch.uint8, device="cuda")
        vc = kc.clone()
        W.wide_kv_quantize(t.cuda(), -t.cuda(), kc, vc, 1, HD, qg)
        assert np.array_equal(kc.cpu().numpy()[0, :, 0], _kvq.quantize(x, qg))
        assert np.array_equal(vc.cpu().numpy()[0, :, 0], _kvq.quantize(-x, qg))


@pytest.mark.parametrize("qg", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_quantize_far_apart(dtype, qg):
    """Values and ranges off a border by less than an fp64 difference holds, against whole numbers."""
    x = _kvq_exact.border_rows()[dtype == torch.float32]
    t = torch.from_numpy(x).to(dtype)
    kc = torch.zeros(1, len(x), 1, _kvq.row_bytes(qg), dtype=torch.uint8, device="cuda")
    vc = kc.clone()
    W.wide_kv_quantize(t.cuda(), -t.cuda(), kc, vc, 1, HD, qg)
    assert np.array_equal(kc.cpu().numpy()[0, :, 0], _kvq_exact.quantize(x, qg))
    assert np.array_equal(vc.cpu().numpy()[0, :, 0], _kvq_exact.quantize(-x, qg))


# ---- reading back ------------------------------------------------------------------

@pytest.mark.parametrize("hm", [False, True])
@pytest.mark.parametrize("qg", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
def test_dequantize(dtype, qg, hm):
    for n, (n_seq, T, L, n_kv, pos, kv_len) in enumerate(SHAPES):
        say("dequantize", dtype, qg, hm, SHAPES[n])
        x = rows_f64(n, (2, n_seq, L, n_kv, HD), torch.float32).double().numpy()
        caches = _kvq.quantize(x, qg)
        if hm:
            caches = caches.transpose(0, 1, 3, 2, 4)
        kc, vc = (d(c) for c in caches)
        k = torch.full((n_seq * T, n_kv * HD), 9.0, dtype=dtype, device="cuda")
        got = W.wide_kv_dequantize(kc, vc, T, n_kv, HD, qg, pos=i32(pos), kv_len=i32(kv_len), head_major=hm, k=k,
                                   dtype=dtype)
        torch.cuda.synchronize()
        assert got[0] is k and got[1].dtype == dtype
        for y, c in zip(got, _kvq.quantize(x, qg)):
            want = np.zeros((n_seq * T, n_kv, HD), np.float32)
            for r, b, p in _kvq.where_rows(n_seq, T, L, pos, kv_len):
                want[r] = _kvq.values(c[b, p], qg)   # fp64 is exact here: one rounding to fp32
            want = torch.from_numpy(want).to(dtype).view(n_seq * T, n_kv * HD)
            assert torch.equal(y.cpu().view(torch.int16 if dtype == torch.bfloat16 else torch.int32),
                               want.view(torch.int16 if dtype == torch.bfloat16 else torch.int32)), SHAPES[n]


def test_dequantize_an_empty_cache():
    kc = torch.empty(2, 0, 4, 80, dtype=torch.uint8, device="cuda")
    k, v = W.wide_kv_dequantize(kc, kc.clone(), 3, 4, HD, 32)
    assert not k.any() and not v.any() and k.shape == (6, 512)
    assert W.wide_kv_dequantize(kc, kc.clone(), 0, 4, HD, 32)[0].shape == (0, 512)


# ---- attention -----------------------------------------------------------------------

def make_cache(seed, B, L, n_kv, qg, hm):
    x = rows_f64(seed, (2, B, L, n_kv, HD), torch.float32, spread=0.2).double().numpy()
    c = _kvq.quantize(x, qg)
    return [np.ascontiguousarray(a) for a in (c.transpose(0, 1, 3, 2, 4) if hm else c)]


def poison(c, kv_len, mask, n_q, n_kv, group, hm):
    """Cache rows that may not be used: bytes of NaN scales and lows."""
    c = c.copy()
    B, L = c.shape[0], c.shape[2 if hm else 1]
    for b in range(B):
        n = L if kv_len is None else max(0, min(L, int(kv_len[b])))
        for h in range(n_kv):
            qpk, hpg = n_q // n_kv, group // HD
            on = any(mask[b, i // hpg] for i in range(h * qpk, (h + 1) * qpk))
            view = c[b, h] if hm else c[b, :, h]
            view[n if on else 0:] = 0xff
    return c


def run_attention(q, kc, vc, mask, n_q, n_kv, group, qg, kv_len, hm, **kw):
    return W.wide_attention_decode_kvq(q, kc, vc, mask, n_q, n_kv, HD, group, qg, kv_len=kv_len, head_major=hm, **kw)


def check_attention(got, q, kc, vc, mask, n_q, n_kv, group, qg, kv_len, hm, what):
    want, tol = _kvq.attention(q.double().numpy(), kc, vc, mask, n_q, n_kv, group, qg, kv_len, hm)
    g = got.double().cpu().numpy()
    assert np.isfinite(g).all(), what
    over = np.abs(g - want) - tol
    assert (over <= 0).all(), (what, int((over > 0).sum()), float(over.max()))


HEADS = [  # n_q, n_kv, group
    (8, 2, 512), (4, 4, 128), (16, 2, 256), (16, 1, 2048), (12, 2, 384), (5, 1, 128), (18, 2, 384),
]
LENGTHS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 65, 127, 129, 257, 1000]


@pytest.mark.parametrize("hm", [False, True])
@pytest.mark.parametrize("qg", [32, 64, 128])
@pytest.mark.parametrize("heads", HEADS)
def test_attention(heads, qg, hm):
    n_q, n_kv, group = heads
    ng = n_q * HD // group
    for L in LENGTHS:
        B = 3
        say("attention", heads, qg, hm, L)
        g = np.random.default_rng(L)
        q = torch.from_numpy((1.5 * g.normal(size=(B, n_q * HD))).astype(np.float32)).bfloat16()
        mask = (g.random((B, ng)) < 0.7).astype(np.uint8) * 3
        mask[0] = 1
        kv_len = None if L % 2 else [L, L // 2, max(1, L - 1)]
        kc, vc = make_cache(L, B, L, n_kv, qg, hm)
        kd, vd = (d(poison(c, kv_len, mask, n_q, n_kv, group, hm)) for c in (kc, vc))
        o = torch.full((B, n_q * HD), float("nan"), dtype=torch.bfloat16, device="cuda")
        run_attention(q.cuda(), kd, vd, d(mask), n_q, n_kv, group, qg, i32(kv_len), hm, o=o)
        torch.cuda.synchronize()
        check_attention(o, q, kc, vc, mask, n_q, n_kv, group, qg, kv_len, hm, (heads, qg, hm, L))


def test_attention_empty_rows():
    """Lengths of zero, below zero and past the capacity; tokens without an active group."""
    B, L, n_q, n_kv, group, qg = 6, 70, 8, 2, 512, 32
    kv_len = [0, -5, 70, 700, 1, 33]
    mask = np.ones((B, 2), np.uint8)
    mask[2, 0] = 0
    mask[3] = 0
    q = rows_f64(1, (B, n_q * HD), torch.bfloat16)
    for hm in (False, True):
        kc, vc = make_cache(3, B, L, n_kv, qg, hm)
        kd, vd = (d(poison(c, kv_len, mask, n_q, n_kv, group, hm)) for c in (kc, vc))
        o = run_attention(q.cuda(), kd, vd, d(mask), n_q, n_kv, group, qg, i32(kv_len), hm)
        check_attention(o, q, kc, vc, mask, n_q, n_kv, group, qg, kv_len, hm, hm)
        bits = o.view(torch.int16)
        assert not bits[:2].any() and not bits[3].any() and not bits[2, :512].any()


def test_attention_large_scores_and_not_finite_keys():
    """Scores far apart (one key holds all the weight, early and late maxima), and a NaN key in reach."""
    B, L, n_q, n_kv, group, qg, hm = 4, 400, 8, 2, 1024, 32, False
    kc, vc = make_cache(9, B, L, n_kv, qg, hm)
    q = 40 * rows_f64(2, (B, n_q * HD), torch.float32, spread=0.0).bfloat16().float()
    q = q.bfloat16()
    mask = np.ones((B, 1), np.uint8)
    kv_len = [400, 399, 200, 5]
    o = run_attention(q.cuda(), d(kc), d(vc), d(mask), n_q, n_kv, group, qg, i32(kv_len), hm)
    check_attention(o, q, kc, vc, mask, n_q, n_kv, group, qg, kv_len, hm, "large scores")
    kc[1, 7, 0, 64:] = 0xff                                    # one KV head of one sequence
    o2 = run_attention(q.cuda(), d(kc), d(vc), d(mask), n_q, n_kv, group, qg, i32(kv_len), hm)
    assert torch.isnan(o2[1, :512]).all()
    o2[1, :512] = o[1, :512]
    assert torch.equal(o, o2)


@pytest.mark.parametrize("qg", [32, 64, 128])
@pytest.mark.parametrize("n_q", [8, 16, 32])
@pytest.mark.parametrize("eq,ek,ev", [(0, 0, -110), (0, 0, -119), (110, -110, 0), (-110, 97, 0), (-125, -100, 97)])
def test_attention_far_sizes(eq, ek, ev, n_q, qg):
    """q, K and V of about 2^eq, 2^ek and 2^ev."""
    B, L, n_kv, group, hm = 2, 130, 2, 512, True
    say("sizes", eq, ek, ev, n_q, qg)
    q = (rows_f64(1, (B, n_q * HD), torch.float32, spread=0.3) * 2.0 ** eq).bfloat16()
    kc, vc = (_kvq.quantize(rows_f64(s, (B, n_kv, L, HD), torch.float32, spread=0.2).double().numpy() * 2.0 ** e, qg)
              for s, e in ((2, ek), (3, ev)))
    mask = np.ones((B, n_q * HD // group), np.uint8)
    o = run_attention(q.cuda(), d(kc), d(vc), d(mask), n_q, n_kv, group, qg, None, hm)
    check_attention(o, q, kc, vc, mask, n_q, n_kv, group, qg, None, hm, (eq, ek, ev))


@pytest.mark.parametrize("B,L,n_q,n_kv,group,qg,hm,ragged", [
    (1, 9001, 8, 2, 512, 32, True, False),     # one long sequence: the keys are cut
    (2, 5000, 4, 4, 128, 128, False, True),
    (40, 1500, 8, 2, 512, 64, False, True),
    (64, 700, 4, 1, 512, 32, True, True),
    (130, 300, 16, 8, 256, 32, True, True),
    (700, 20, 8, 4, 128, 32, False, False),
])
def test_attention_batches(B, L, n_q, n_kv, group, qg, hm, ragged):
    say("batch", B, L, n_q, n_kv, group, qg, hm, ragged)
    g = np.random.default_rng(B)
    q = rows_f64(B, (B, n_q * HD), torch.bfloat16, spread=0.3)
    mask = (g.random((B, n_q * HD // group)) < 0.6).astype(np.uint8)
    kv_len = g.integers(0, L + 1, B).tolist() if ragged else None
    kc, vc = make_cache(L, B, L, n_kv, qg, hm)
    kd, vd = (d(poison(c, kv_len, mask, n_q, n_kv, group, hm)) for c in (kc, vc))
    args = (q.cuda(), kd, vd, d(mask), n_q, n_kv, group, qg, i32(kv_len), hm)
    o = run_attention(*args)
    check_attention(o, q, kc, vc, mask, n_q, n_kv, group, qg, kv_len, hm, (B, L))
    assert torch.equal(o.view(torch.int16), run_attention(*args).view(torch.int16))  # the same call, the same bits


@pytest.mark.parametrize("qg", [32, 64, 128])
@pytest.mark.parametrize("B,L,n_q,n_kv,group,lens", [
    (32, 2081, 32, 8, 512, "random"),          # whole rows of eight heads
    (5, 7000, 64, 8, 1024, [6999, 0, 3501, 7000, 65]),
    (9, 2100, 16, 16, 128, "random"),          # two sets of eight
    (33, 2081, 12, 4, 384, "random"),
    (64, 2081, 32, 2, 256, "random"),
    (22, 2081, 24, 12, 256, "random"),         # three sets of four
    (26, 2081, 20, 10, 256, "random"),         # five of two
    (40, 2081, 10, 5, 128, "random"),          # one by one
    (1, 33000, 8, 8, 128, None),
    (300, 2049, 8, 8, 128, "random"),          # more groups than workgroups
])
def test_attention_token_major(B, L, n_q, n_kv, group, lens, qg):
    """Long token-major caches, read by the position.  Before each call another has left NaN wherever a
    workgroup keeps rows, so that what lies behind a sequence's end or belongs to a masked head shows."""
    say("token-major", B, L, n_q, n_kv, group, qg)
    g = np.random.default_rng(B + qg)
    q = rows_f64(B, (B, n_q * HD), torch.bfloat16, spread=0.3)
    mask = (g.random((B, n_q * HD // group)) < 0.6).astype(np.uint8)
    mask[0, 0] = 1
    kv_len = np.minimum(g.integers(0, L + 400, B) // 4 * (g.random(B) < 0.5) + 7, L).tolist() if lens == "random" else lens
    if lens == "random":
        kv_len[:2] = [L, 0]
    few = 4                                                      # sequences with values of their own
    kc, vc = make_cache(L, min(B, few), L, n_kv, qg, False)
    kc, vc = (np.concatenate([c] * -(-B // few))[:B] for c in (kc, vc))
    kd, vd = (d(poison(c, kv_len, mask, n_q, n_kv, group, False)) for c in (kc, vc))
    nan = torch.full_like(kd, 0xff)
    args = (q.cuda(), kd, vd, d(mask), n_q, n_kv, group, qg, i32(kv_len), False)
    first = None
    for _ in range(2):
        run_attention(q.cuda(), nan, nan, d(np.ones_like(mask)), n_q, n_kv, group, qg, None, False)
        o = run_attention(*args)
        check_attention(o, q, kc, vc, mask, n_q, n_kv, group, qg, kv_len, False, (B, L, n_kv))
        assert first is None or torch.equal(o.view(torch.int16), first.view(torch.int16))
        first = o


@pytest.mark.parametrize("B,hm", [(1000, True), (1001, True), (512, False), (513, False)])
def test_attention_many_sequences(B, hm):
    """The most (sequence, KV head) pairs that share their waves, and one sequence more."""
    L, n_q, n_kv, group, qg = 2050, 8, 8, 128, 32
    say("many sequences", B, hm)
    g = np.random.default_rng(B)
    q = rows_f64(B, (B, n_q * HD), torch.bfloat16, spread=0.3)
    mask = (g.random((B, n_kv)) < 0.5).astype(np.uint8)
    kv_len = np.where(g.random(B) < 0.1, L, g.integers(-1, 90, B))
    which = g.integers(0, 4, B)                                  # the sequences' caches, of four
    four = make_cache(5, 4, L, n_kv, qg, hm)
    kd, vd = (d(c)[d(which)] for c in four)
    o = run_attention(q.cuda(), kd, vd, d(mask), n_q, n_kv, group, qg, i32(kv_len), hm)
    some = np.unique(np.r_[0, 1, B - 2, B - 1, np.flatnonzero(kv_len == L)[:4], g.integers(0, B, 20)])
    kc, vc = (c[which[some]] for c in four)
    check_attention(o[torch.from_numpy(some).cuda()], q[some], kc, vc, mask[some], n_q, n_kv, group, qg, kv_len[some], hm,
                    (B, hm))
    off = np.repeat(mask == 0, HD, axis=1) | (kv_len <= 0)[:, None]
    assert not o.cpu()[torch.from_numpy(off)].any() and torch.isfinite(o).all()


def kernels_of(call):
    """Launches of a call's attention kernels: (a workgroup per pair, equal runs, whole rows, joins)."""
    W.wide_timing_enable(True)
    W.wide_timing_reset()
    try:
        call()
        every, runs, rows, joins = (W.wide_timing_query("wide_attn_decode_kvq" + x)[1]
                                    for x in ("", "/runs", "/rows", "_merge"))
    finally:
        W.wide_timing_enable(False)
    return every - runs - rows, runs, rows, joins


@pytest.mark.parametrize("qg", [32, 64, 128])
@pytest.mark.parametrize("B,L,n_q,n_kv,group,hm,cut", [
    (3, 2200, 8, 2, 512, True, "runs"),        # 4 query heads per KV head
    (2, 2081, 64, 8, 1024, True, "runs"),      # 8
    (3, 2500, 10, 2, 640, True, "runs"),       # 5
    (3, 2200, 16, 1, 1024, True, "runs"),      # 16
    (3, 2081, 18, 2, 384, True, "runs"),       # 9
    (2, 2300, 22, 2, 256, True, "runs"),       # 11
    (2, 2081, 64, 8, 512, False, "runs"),
    (3, 2200, 20, 4, 640, False, "runs"),
    (3, 2081, 32, 2, 2048, False, "runs"),
    (2, 2200, 39, 3, 384, False, "runs"),
    (32, 2081, 64, 4, 2048, False, "rows"),
    (32, 2081, 32, 4, 1024, False, "rows"),
    (70, 2049, 6, 3, 384, False, "runs"),      # (one head group over two KV heads)
    (180, 2049, 9, 3, 384, False, "pairs"),    # more than 512 pairs
])
def test_attention_long_by_heads(B, L, n_q, n_kv, group, hm, cut, qg):
    """Contexts past 2048 keys for every number of query heads a KV head has columns for, ragged and
    partly masked, with NaN behind the ends, and the kernel that is meant."""
    say("long", B, L, n_q, n_kv, group, hm, cut, qg)
    g = np.random.default_rng(B + n_q + qg)
    q = rows_f64(n_q, (B, n_q * HD), torch.bfloat16, spread=0.3)
    mask = (g.random((B, n_q * HD // group)) < 0.6).astype(np.uint8)
    mask[0] = 1
    kv_len = np.minimum(g.integers(0, L + 400, B) // (1 if B < 8 else 8), L)
    kv_len[:2] = L, L - 35
    few = min(B, 4)                                              # sequences with values of their own
    kc, vc = (np.concatenate([c] * -(-B // few))[:B] for c in make_cache(n_q, few, L, n_kv, qg, hm))
    kd, vd = (d(poison(c, kv_len, mask, n_q, n_kv, group, hm)) for c in (kc, vc))
    args = (q.cuda(), kd, vd, d(mask), n_q, n_kv, group, qg, i32(kv_len), hm)
    ws = torch.full((W.wide_attention_decode_kvq_workspace_size(B, L, n_q, n_kv, HD, group, qg),), 0xff,
                    dtype=torch.uint8, device="cuda")
    got = []
    ran = kernels_of(lambda: got.append(run_attention(*args, ws=ws)))
    assert ran == {"pairs": (1, 0, 0, 0), "runs": (0, 1, 0, 1), "rows": (0, 0, 1, 1)}[cut]
    check_attention(got[0], q, kc, vc, mask, n_q, n_kv, group, qg, kv_len, hm, (B, L, n_q, n_kv, qg))
    assert torch.equal(got[0].view(torch.int16), run_attention(*args).view(torch.int16))


@pytest.mark.parametrize("n_kv,hm", [(8, True), (9, False)])
def test_attention_more_pairs_than_a_launch_holds(n_kv, hm):
    """2^23 and more (sequence, KV head) pairs: more threads than one launch takes.  With one key the
    answer is its value, with none zeros."""
    B, L, qg = (1 << 23) // n_kv + 5, 1, 128
    say("pairs", B * n_kv, hm)
    g = torch.Generator(device="cuda").manual_seed(n_kv)
    kv = torch.randn((B, n_kv * HD), generator=g, device="cuda").bfloat16()
    kc = torch.zeros(cache_shape(B, L, n_kv, qg, hm), dtype=torch.uint8, device="cuda")
    vc = torch.zeros_like(kc)
    W.wide_kv_quantize(kv, kv, kc, vc, n_kv, HD, qg, head_major=hm)
    mask = (torch.rand((B, n_kv), generator=g, device="cuda") < 0.9).to(torch.uint8)
    kv_len = (torch.rand((B,), generator=g, device="cuda") < 0.9).int()
    o = run_attention(kv, kc, vc, mask, n_kv, n_kv, HD, qg, kv_len, hm)
    n = 0
    for at in torch.arange(B, device="cuda").split(1 << 17):
        v = W.wide_kv_dequantize(kc[at[0]:at[-1] + 1], vc[at[0]:at[-1] + 1], 1, n_kv, HD, qg, head_major=hm,
                                 dtype=torch.float32)[1].view(-1, n_kv, HD)
        on = (mask[at] != 0) & (kv_len[at] > 0)[:, None]
        got = o[at].view(-1, n_kv, HD).float()
        # p = 1; p s in two bf16 parts (2^-16) over 16 + c and 16 s off again, fp32, one rounding to bf16: with
        # v from low to low + 15 s and low < 0 < low + 15 s (normal values), 47 s + |low| <= 5 (|low| + |high|)
        size = 5 * (v.amax(-1, keepdim=True).abs() + v.amin(-1, keepdim=True).abs())
        tol = 2.0 ** -8 * v.abs() + size * (2.0 ** -16 + 70 * 2.0 ** -24)
        assert ((got - v).abs() <= tol)[on].all() and not got[~on].any()
        n += int(on.sum())
    assert n > B * n_kv // 2


@pytest.mark.parametrize("L,hm", [(300, False), (3000, True), (33000, False)])
@pytest.mark.parametrize("n_q", [8, 16, 32])
def test_attention_not_finite_queries(n_q, L, hm):
    """An infinity or a NaN in one query head gives that head NaN and no other anything; a masked head, zeros."""
    B, n_kv, qg = 1, 8, 64
    n_kv = n_kv if n_q > 16 else 2
    q = rows_f64(L, (B, n_q * HD), torch.bfloat16, spread=0.3)
    kd, vd = (d(c) for c in make_cache(L, B, L, n_kv, qg, hm))
    mask = np.ones((B, n_q), np.uint8)
    mask[0, 3] = 0
    clean = run_attention(q.cuda(), kd, vd, d(mask), n_q, n_kv, HD, qg, None, hm)
    assert torch.isfinite(clean).all()
    for at, value in ((1, float("inf")), (1, float("-inf")), (1, float("nan")), (3, float("nan")), (n_q - 1, float("inf"))):
        say("queries", n_q, L, hm, at, value)
        x = q.clone()
        x[0, at * HD + 77] = value
        o = run_attention(x.cuda(), kd, vd, d(mask), n_q, n_kv, HD, qg, None, hm)
        head = slice(at * HD, (at + 1) * HD)
        if mask[0, at]:
            assert torch.isnan(o[0, head]).all()
            o[0, head] = clean[0, head]
        assert torch.equal(o.view(torch.int16), clean.view(torch.int16))


def test_cache_beyond_32_bit_offsets():
    """Rows more than 4 GiB into a cache: written, read back and attended to."""
    n_kv, qg, L = 32, 32, 1 << 20
    B = 2
    kc = torch.empty(B, L, n_kv, 80, dtype=torch.uint8, device="cuda")   # 2.5 GiB a sequence
    vc = torch.empty_like(kc)
    kc[1, L - 600:].fill_(0xff)
    vc[1, L - 600:].fill_(0xff)
    T = 500
    k, v = (rows_f64(s, (B * T, n_kv * HD), torch.bfloat16, spread=0.2) for s in (1, 2))
    for first in (0, L - T):
        pos = i32([first, first])
        W.wide_kv_quantize(k.cuda(), v.cuda(), kc, vc, n_kv, HD, qg, pos=pos)
        k2, v2 = W.wide_kv_dequantize(kc, vc, T, n_kv, HD, qg, pos=pos, dtype=torch.float32)
        for x, y in ((k, k2), (v, v2)):
            want = _kvq.values(_kvq.quantize(x.double().numpy().reshape(-1, HD), qg), qg).astype(np.float32)
            assert np.array_equal(y.cpu().numpy().reshape(-1, HD), want)
    # attention over the first T positions of the second sequence (its cache starts 2.5 GiB in, its end lies past 4)
    mask = np.zeros((B, n_kv), np.uint8)
    mask[1, ::5] = 1
    q = rows_f64(3, (B, n_kv * HD), torch.bfloat16, spread=0.2)
    kv_len = [0, T]
    o = run_attention(q.cuda(), kc, vc, d(mask), n_kv, n_kv, HD, qg, i32(kv_len), False)
    want, tol = _kvq.attention(q.double().numpy(), kc[:, :T].cpu().numpy(), vc[:, :T].cpu().numpy(), mask, n_kv, n_kv,
                               HD, qg, kv_len, False)
    assert (np.abs(o.double().cpu().numpy() - want) <= tol).all()
    # and over all of it, one head: the keys between hold zeros except the two written ends
    kc[1, T:L - T].zero_()
    vc[1, T:L - T].zero_()
    mask[:] = 0
    mask[1, 31] = 1
    o = run_attention(q.cuda(), kc, vc, d(mask), n_kv, n_kv, HD, qg, None, False)
    ends = torch.cat([kc[1, :T, 31], kc[1, L - T:, 31]]).cpu().numpy(), torch.cat([vc[1, :T, 31], vc[1, L - T:, 31]]).cpu().numpy()
    qh = q.double().numpy()[1, 31 * HD:]
    sc = _kvq.values(ends[0], qg) @ qh / np.sqrt(HD)
    p = np.exp(np.concatenate([sc, np.zeros(L - 2 * T)]))
    ref = (p[:2 * T] @ _kvq.values(ends[1], qg)) / p.sum()
    got = o.double().cpu().numpy()[1, 31 * HD:]
    s, low, _ = _kvq.parts(ends[1], qg)
    mag = (p[:2 * T] @ (47 * s + np.abs(low))) / p.sum()
    # fp32 sums over 2^20 keys in chunks of at most 65536: (65536 + 128) u of their size, and as much for sum(p)
    assert (np.abs(got - ref) <= 2.0 ** -8 * np.abs(ref) + mag * (2.0 ** -14 + 2 * 65700 * 2.0 ** -24)).all()
    assert not o[0].any()


# ---- as they are used together ---------------------------------------------------------

@pytest.mark.parametrize("hm", [False, True])
@pytest.mark.parametrize("qg", [32, 64, 128])
def test_prompt_then_tokens(qg, hm):
    """Left-padded prompts into the cache, then tokens one by one, each step's
    attention against the plain form; the cached prefix read back serves the
    prefill attention of a next chunk."""
    B, T, L, n_q, n_kv, group = 3, 50, 64, 8, 2, 512
    pad = [0, 13, 49]
    x = rows_f64(qg, (2, B, T + 6, n_kv * HD), torch.bfloat16, spread=0.2)
    kc = torch.full(cache_shape(B, L, n_kv, qg, hm), 0xff, dtype=torch.uint8, device="cuda")
    vc = kc.clone()
    flat = [t[:, :T].reshape(B * T, -1).contiguous().cuda() for t in x]
    lens = np.array([T - p for p in pad])
    W.wide_kv_quantize(*flat, kc, vc, n_kv, HD, qg, pos=i32([-p for p in pad]), head_major=hm)
    for step in range(6):
        tok = [t[:, T + step].contiguous().cuda() for t in x]
        W.wide_kv_quantize(*tok, kc, vc, n_kv, HD, qg, pos=i32(lens), head_major=hm)
        lens = lens + 1
        q = rows_f64(step, (B, n_q * HD), torch.bfloat16, spread=0.2)
        mask = np.ones((B, n_q * HD // group), np.uint8)
        mask[step % B, step % 2] = 0
        o = run_attention(q.cuda(), kc, vc, d(mask), n_q, n_kv, group, qg, i32(lens), hm)
        check_attention(o, q, kc.cpu().numpy(), vc.cpu().numpy(), mask, n_q, n_kv, group, qg, lens, hm, step)
    # the cache holds exactly the rows that were written
    rows = [_kvq.quantize(t.double().numpy().reshape(B, T + 6, n_kv, HD), qg) for t in x]
    for got, want in zip((kc, vc), rows):
        got = got.cpu().numpy()
        for b in range(B):
            seq = got[b].transpose(1, 0, 2) if hm else got[b]
            assert np.array_equal(seq[:lens[b]], want[b, pad[b]:])
            assert (seq[lens[b]:] == 0xff).all()
    # a chunk of two queries a sequence against the prefix read back, right-aligned
    T_k = int(lens.max())
    k, v = W.wide_kv_dequantize(kc, vc, T_k, n_kv, HD, qg, pos=i32(lens - T_k), kv_len=i32(lens), head_major=hm)
    q2 = rows_f64(77, (B * 2, n_q * HD), torch.bfloat16, spread=0.2)
    m2 = torch.ones(B * 2, n_q * HD // group, dtype=torch.uint8, device="cuda")
    o2 = W.wide_attention_masked(q2.cuda(), k, v, m2, B, n_q, n_kv, HD, group, causal=True, leftpad=i32(T_k - lens))
    kf, vf = (t.double().cpu().numpy().reshape(B, T_k, n_kv, HD) for t in (k, v))
    for b in range(B):
        for i in range(2):
            for h in range(n_q):
                sl = slice(T_k - lens[b], T_k - 1 + i)
                qh = q2.double().numpy()[2 * b + i].reshape(n_q, HD)[h]
                sc = kf[b, sl, h // 4] @ qh / np.sqrt(HD)
                w = np.exp(sc - sc.max())
                w /= w.sum()
                ref, mag = w @ vf[b, sl, h // 4], w @ np.abs(vf[b, sl, h // 4])
                got = o2.double().cpu().numpy()[2 * b + i].reshape(n_q, HD)[h]
                # probabilities in bf16 (2^-8), fp32 elsewhere, one bf16 rounding of o
                assert (np.abs(got - ref) <= (2.0 ** -8 + 2.0 ** -11) * mag + 2.0 ** -8 * np.abs(ref)).all()


def test_graph_of_a_decode_step():
    """A step captured once (write the token, attend) and replayed with new
    positions and rows, eager work of the program between the replays."""
    B, L, n_q, n_kv, group, qg, hm = 4, 600, 8, 2, 512, 32, True
    kc0, vc0 = make_cache(4, B, L, n_kv, qg, hm)
    kc, vc = d(kc0), d(vc0)
    k, v = (torch.zeros(B, n_kv * HD, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(B, n_q * HD, dtype=torch.bfloat16, device="cuda")
    pos, lens = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    mask = torch.ones(B, n_q * HD // group, dtype=torch.uint8, device="cuda")
    o = torch.empty_like(q)
    ws = torch.empty(W.wide_attention_decode_kvq_workspace_size(B, L, n_q, n_kv, HD, group, qg), dtype=torch.uint8,
                     device="cuda")

    def step():
        W.wide_kv_quantize(k, v, kc, vc, n_kv, HD, qg, pos=pos, kv_len=lens, head_major=hm)
        run_attention(q, kc, vc, mask, n_q, n_kv, group, qg, lens, hm, o=o, ws=ws)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    for n in range(4):
        at = np.array([0, 17 + n, 598, 300 - n])
        k.copy_(rows_f64(n, k.shape, torch.bfloat16, spread=0.2).cuda())
        v.copy_(rows_f64(n + 50, k.shape, torch.bfloat16, spread=0.2).cuda())
        qh = rows_f64(n + 90, q.shape, torch.bfloat16, spread=0.2)
        q.copy_(qh.cuda())
        pos.copy_(i32(at))
        lens.copy_(i32(at + 1))
        mask[n % B, 0] = 0
        ws.fill_(0xff)
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        check_attention(got, qh, kc.cpu().numpy(), vc.cpu().numpy(), mask.cpu().numpy(), n_q, n_kv, group, qg, at + 1,
                        hm, n)
        step()                                                 # the same, eagerly
        assert torch.equal(o.view(torch.int16), got.view(torch.int16))
        mask[n % B, 0] = 1


def test_two_streams():
    """Calls on two streams at once, each with its own workspace, on tensors made on a third."""
    B, L, n_q, n_kv, group, qg, hm = 2, 3000, 8, 2, 512, 64, False
    kc, vc = (d(c) for c in make_cache(6, B, L, n_kv, qg, hm))
    mask = torch.ones(B, 2, dtype=torch.uint8, device="cuda")
    qs = [rows_f64(s, (B, n_q * HD), torch.bfloat16, spread=0.2).cuda() for s in range(2)]
    want = [run_attention(q, kc, vc, mask, n_q, n_kv, group, qg, None, hm) for q in qs]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    out = [torch.zeros_like(q) for q in qs]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, q, o in zip(streams, qs, out):
            with torch.cuda.stream(st):
                run_attention(q, kc, vc, mask, n_q, n_kv, group, qg, None, hm, o=o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


@pytest.mark.parametrize("B,L,n_q,n_kv,group,qg,hm,cut", [
    (4, 2300, 8, 2, 512, 32, True, (0, 1, 0, 1)),
    (18, 4097, 16, 4, 512, 64, False, (0, 0, 1, 1)),
])
def test_graph_of_a_long_decode_step(B, L, n_q, n_kv, group, qg, hm, cut):
    """The same over contexts whose work is cut and joined: two launches, and a workspace of NaN bytes
    before each replay.  Sequences, KV heads and, once, the whole batch have nothing to attend to."""
    say("graph", B, L, n_q, n_kv, group, qg, hm)
    few = min(B, 4)
    kc, vc = (d(np.concatenate([c] * -(-B // few))[:B]) for c in make_cache(4, few, L, n_kv, qg, hm))
    k, v = (torch.zeros(B, n_kv * HD, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    q = torch.zeros(B, n_q * HD, dtype=torch.bfloat16, device="cuda")
    pos, lens = (torch.zeros(B, dtype=torch.int32, device="cuda") for _ in range(2))
    mask = torch.ones(B, n_q * HD // group, dtype=torch.uint8, device="cuda")
    o = torch.empty_like(q)
    ws = torch.empty(W.wide_attention_decode_kvq_workspace_size(B, L, n_q, n_kv, HD, group, qg), dtype=torch.uint8,
                     device="cuda")

    def step():
        W.wide_kv_quantize(k, v, kc, vc, n_kv, HD, qg, pos=pos, kv_len=lens, head_major=hm)
        run_attention(q, kc, vc, mask, n_q, n_kv, group, qg, lens, hm, o=o, ws=ws)

    assert kernels_of(step) == cut
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    g = np.random.default_rng(B)
    for n in range(5):
        at = g.integers(0, L, B)
        at[n % B], at[(n + 1) % B], at[(n + 2) % B] = L - 1, -1, 0       # the last place, nothing, one key
        m = (g.random(mask.shape) < 0.6).astype(np.uint8)
        m[(n + 3) % B] = 0
        if n == 2:
            at[:] = -1
        if n == 3:
            m[:] = 0
        k.copy_(rows_f64(n, k.shape, torch.bfloat16, spread=0.2).cuda())
        v.copy_(rows_f64(n + 50, k.shape, torch.bfloat16, spread=0.2).cuda())
        qh = rows_f64(n + 90, q.shape, torch.bfloat16, spread=0.2)
        q.copy_(qh.cuda())
        pos.copy_(i32(at))
        lens.copy_(i32(at + 1))
        mask.copy_(d(m))
        ws.fill_(0xff)
        o.fill_(float("nan"))
        graph.replay()
        torch.cuda.synchronize()
        got = o.clone()
        check_attention(got, qh, kc.cpu().numpy(), vc.cpu().numpy(), m, n_q, n_kv, group, qg, at + 1, hm, n)
        ws.fill_(0xff)
        step()                                                 # the same, eagerly
        assert torch.equal(o.view(torch.int16), got.view(torch.int16))


def test_two_streams_over_whole_rows():
    """As test_two_streams, by the kernel that reads a position's rows whole."""
    B, L, n_q, n_kv, group, qg = 18, 4097, 16, 4, 512, 32
    kc, vc = (d(np.concatenate([c] * 9)) for c in make_cache(6, 2, L, n_kv, qg, False))
    mask = torch.ones(B, n_q * HD // group, dtype=torch.uint8, device="cuda")
    lens = [i32(np.random.default_rng(s).integers(0, L + 1, B)) for s in range(2)]
    qs = [rows_f64(s, (B, n_q * HD), torch.bfloat16, spread=0.2).cuda() for s in range(2)]
    args = [(q, kc, vc, mask, n_q, n_kv, group, qg, n, False) for q, n in zip(qs, lens)]
    want = []
    assert kernels_of(lambda: want.extend(run_attention(*a) for a in args)) == (0, 0, 2, 2)
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in qs]
    out = [torch.zeros_like(q) for q in qs]
    torch.cuda.synchronize()
    for _ in range(5):
        for st, a, o in zip(streams, args, out):
            with torch.cuda.stream(st):
                run_attention(*a, o=o)
    torch.cuda.synchronize()
    assert all(torch.equal(a, b) for a, b in zip(out, want))


def test_binding_refusals():
    def z(*s, dt=torch.bfloat16):
        return torch.zeros(*s, dtype=dt, device="cuda")
    u8, i32_ = torch.uint8, torch.int32
    kc, k = z(2, 16, 8, 80, dt=u8), z(6, 1024)
    ok = dict(k=k, v=k, k_cache=kc, v_cache=kc, n_kv=8, head_dim=128, quant_group=32)
    for bad in (dict(k_cache=z(2, 16, 8, 72, dt=u8)), dict(k_cache=z(2, 16, 8, 80, dt=torch.int8)),
                dict(v_cache=z(2, 17, 8, 80, dt=u8)), dict(n_kv=4), dict(quant_group=64), dict(k=z(6, 512)),
                dict(k=z(5, 1024), v=z(5, 1024)), dict(v=z(6, 1024, dt=torch.float32)), dict(pos=z(3, dt=i32_)),
                dict(kv_len=z(2, dt=torch.int64)), dict(k=z(1024, 6).T), dict(v=z(6, 1024).cpu()),
                dict(head_major=True)):
        with pytest.raises(ValueError):
            W.wide_kv_quantize(**{**ok, **bad})
    with pytest.raises(TypeError):
        W.wide_kv_quantize(**{**ok, "k": k.half(), "v": k.half()})
    ok = dict(k_cache=kc, v_cache=kc, T=3, n_kv=8, head_dim=128, quant_group=32)
    for bad in (dict(k=z(5, 1024)), dict(k=z(6, 1024), v=z(6, 1024, dt=torch.float32)), dict(T=-1),
                dict(head_dim=64), dict(pos=z(2, 1, dt=i32_))):
        with pytest.raises(ValueError):
            W.wide_kv_dequantize(**{**ok, **bad})
    ok = dict(q=z(2, 4096), k_cache=kc, v_cache=kc, mask=z(2, 8, dt=u8), n_q=32, n_kv=8, head_dim=128, group_size=512,
              quant_group=32)
    for bad in (dict(q=z(3, 4096)), dict(q=z(2, 1024)), dict(mask=z(2, 4, dt=u8)), dict(o=z(2, 1024)),
                dict(kv_len=z(3, dt=i32_)), dict(group_size=0), dict(k_cache=z(2, 16, 8, 68, dt=u8))):
        with pytest.raises(ValueError):
            W.wide_attention_decode_kvq(**{**ok, **bad})
    with pytest.raises(W.WideError):
        W.wide_attention_decode_kvq(**{**ok, "ws": torch.empty(16, dtype=u8, device="cuda")})
