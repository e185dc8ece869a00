"""The 4-bit KV cache without a GPU: the plain rows used by the GPU tests, and
what the entry points refuse (fake pointers are never dereferenced)."""
import ctypes

import numpy as np
import pytest
import torch

import paper_2607_28418_amd as W
from tests import _kvq, _kvq_exact

A = ctypes.c_void_p(0x10000)
MIS = ctypes.c_void_p(0x10008)


def err():
    return W.lib().wide_last_error().decode()


# ---- the plain rows ----------------------------------------------------------------

@pytest.mark.parametrize("qg", [32, 64, 128])
def test_plain_rows_by_hand(qg):
    x = np.zeros((1, 128))
    x[0] = np.arange(128) % 16          # every group holds 0..15: low 0, scale 1, codes are the values
    rows = _kvq.quantize(x, qg)
    assert rows.shape == (1, W.wide_kv_quant_row_bytes(128, qg))
    assert np.array_equal(_kvq.values(rows, qg), x)
    # word l: nibble n holds dimension 32 (n % 4) + 2 l + n // 4
    words = rows[0, :64].copy().view("<u4")
    for l in range(16):
        for n in range(8):
            assert (words[l] >> (4 * n)) & 15 == (32 * (n % 4) + 2 * l + n // 4) % 16
    ng = 128 // qg
    assert rows[0, 64:].copy().view("<u2").tolist() == [0x3f80] * ng + [0] * ng


def test_plain_rows_ties_and_rounding():
    x = np.zeros((1, 128))
    x[0, :32] = np.arange(32) * 0.5     # 0 .. 15.5: scale 15.5/15 -> 1.03125 (bf16)
    x[0, 32:64] = np.minimum(np.arange(32) * 0.5, 15)  # scale 1: k + 0.5 goes to the even code
    v = _kvq.values(_kvq.quantize(x, 32), 32)[0]
    assert v[:32].max() == 15 * 1.03125
    assert v[32:64].tolist() == [float(np.rint(t)) for t in x[0, 32:64]]
    # the values are within half a scale plus what low's and scale's own rounding leaves
    g = np.random.default_rng(1)
    y = g.normal(size=(500, 128)) * np.exp(g.normal(size=(500, 1)) * 4)
    for qg in (32, 64, 128):
        s, low, c = _kvq.parts(_kvq.quantize(y, qg), qg)
        assert (np.abs(low + s * c - y) <= 0.5 * s * (1 + 2.0 ** -3)).all()
        assert (low <= y).all() and c.max() == 15


def test_plain_rows_not_finite():
    x = np.ones((4, 128))
    x[0, 5], x[1, 77], x[2, 100] = np.nan, -np.inf, 2.0 ** 127
    v = _kvq.values(_kvq.quantize(x, 32), 32)
    assert np.isnan(v[:3]).all() and (v[3] == 1).all()


def test_positions():
    assert _kvq.where_rows(2, 3, 4, [-1, 2], [2, 9]) == [(1, 0, 0), (2, 0, 1), (3, 1, 2), (4, 1, 3)]
    assert _kvq.where_rows(1, 2, 4, None, None) == [(0, 0, 0), (1, 0, 1)]


def test_exact_rows():
    x = np.full((2, 128), 2.0 ** -60)
    x[:, 0], x[:, 1] = -1.0, 29.0           # low -1, scale 2: 2^-60 lies just above the border of codes 0 and 1
    x[1] = -x[1]                            # low -29: -2^-60 just below the border of 14 and 15
    s, low, c = _kvq.parts(_kvq_exact.quantize(x, 32), 32)
    assert (s[:, :32] == 2).all() and low[0, 0] == -1 and low[1, 0] == -29
    assert c[0, :32].tolist() == [0, 15] + [1] * 30 and c[1, :32].tolist() == [15, 0] + [14] * 30
    assert (s[:, 32:] == 0).all() and (low[0, 32:] == 2.0 ** -60).all() and (low[1, 32:] == -2.0 ** -60).all()
    g = np.random.default_rng(3)            # where 53 bits are enough, the rows of the plain form
    y = g.normal(size=(200, 128)).astype(np.float32).astype(np.float64)
    y[100:] = g.integers(-40, 41, (100, 128)) * 2.0 ** -g.integers(0, 20, (100, 128))
    y[:5, 3] = np.nan, np.inf, 2.0 ** 127, 2.0 ** -140, -2.0 ** -149
    y[6] = 2.0 ** -133 * (np.arange(128) % 7)
    for qg in (32, 64, 128):
        assert np.array_equal(_kvq_exact.quantize(y, qg), _kvq.quantize(y, qg))
    few, all_ = _kvq_exact.border_rows()
    assert (torch.from_numpy(few).bfloat16().double().numpy() == few).all()
    assert (torch.from_numpy(all_).float().double().numpy() == all_).all()


# ---- refusals ------------------------------------------------------------------------

def quantize(dt=W.BF16, n_seq=2, T=3, L=16, n_kv=8, hd=128, qg=32, layout=0, pos=None, kv_len=None, k=A, v=A, kc=A,
             vc=A, read=False):
    if read:
        return W.lib().wide_kv_dequantize(dt, n_seq, T, L, n_kv, hd, qg, layout, pos, kv_len, kc, vc, k, v, None)
    return W.lib().wide_kv_quantize(dt, n_seq, T, L, n_kv, hd, qg, layout, pos, kv_len, k, v, kc, vc, None)


@pytest.mark.parametrize("read", [False, True])
@pytest.mark.parametrize("kw,status,msg", [
    (dict(dt=5), W.ERR_INVALID_ARG, "dtype"),
    (dict(n_seq=-1), W.ERR_INVALID_ARG, ">= 0"),
    (dict(T=-1), W.ERR_INVALID_ARG, ">= 0"),
    (dict(L=-1), W.ERR_INVALID_ARG, ">= 0"),
    (dict(n_kv=0), W.ERR_INVALID_ARG, "n_kv_heads"),
    (dict(n_seq=1 << 20, T=1 << 11), W.ERR_INVALID_ARG, "2^31"),
    (dict(n_seq=1 << 40, T=2147483647), W.ERR_INVALID_ARG, "2^31"),
    (dict(n_seq=1 << 14, T=1 << 14), W.ERR_INVALID_ARG, "2^31"),
    (dict(hd=64), W.ERR_UNSUPPORTED, "head_dim 128"),
    (dict(hd=0), W.ERR_INVALID_ARG, "head_dim"),
    (dict(qg=16), W.ERR_INVALID_ARG, "quant_group"),
    (dict(qg=256), W.ERR_INVALID_ARG, "quant_group"),
    (dict(layout=2), W.ERR_INVALID_ARG, "kv_layout"),
    (dict(k=None), W.ERR_INVALID_ARG, "k is NULL"),
    (dict(v=MIS), W.ERR_INVALID_ARG, "v is not 16-byte aligned"),
    (dict(kc=MIS), W.ERR_INVALID_ARG, "k_cache is not 16-byte aligned"),
    (dict(vc=None), W.ERR_INVALID_ARG, "v_cache is NULL"),
])
def test_rows_validation(read, kw, status, msg):
    assert quantize(read=read, **kw) == status
    assert msg in err()


def test_rows_need_two_buffers():
    assert quantize(vc=A) == W.ERR_INVALID_ARG and "k_cache and v_cache are the same" in err()
    assert quantize(read=True, v=A) == W.ERR_INVALID_ARG and "k and v are the same" in err()


def test_rows_empty_calls():
    for read in (False, True):
        for kw in (dict(n_seq=0), dict(T=0)):
            assert quantize(read=read, k=None, v=None, kc=None, vc=None, **kw) == W.OK
    assert quantize(L=0, k=None, v=None, kc=None, vc=None) == W.OK


def test_row_bytes():
    assert [W.wide_kv_quant_row_bytes(128, g) for g in (32, 64, 128)] == [80, 72, 68]
    for hd, g in ((64, 32), (128, 16), (128, 0), (0, 32)):
        with pytest.raises(ValueError):
            W.wide_kv_quant_row_bytes(hd, g)


def attention(dt=W.BF16, B=32, L=8192, nq=32, nkv=8, hd=128, G=512, qg=32, mask=A, kv_len=None, layout=0, q=A, k=A,
              v=A, o=A, ws=A, ws_bytes=1 << 40):
    return W.lib().wide_attention_decode_kvq(dt, B, L, nq, nkv, hd, G, qg, mask, kv_len, layout, q, k, v, o, ws,
                                             ws_bytes, None)


@pytest.mark.parametrize("kw,status,msg", [
    (dict(dt=W.F32), W.ERR_UNSUPPORTED, "bf16"),
    (dict(dt=9), W.ERR_INVALID_ARG, "dtype"),
    (dict(hd=64, G=256), W.ERR_UNSUPPORTED, "head_dim 128"),
    (dict(nq=34, nkv=2, G=128), W.ERR_UNSUPPORTED, "16 query heads"),
    (dict(nq=30), W.ERR_INVALID_ARG, "multiple of n_kv_heads"),
    (dict(G=192), W.ERR_INVALID_ARG, "multiple of head_dim"),
    (dict(L=0), W.ERR_INVALID_ARG, "length 0"),
    (dict(B=-1), W.ERR_INVALID_ARG, ">= 0"),
    (dict(B=1 << 20, L=1 << 12), W.ERR_INVALID_ARG, "2^31"),
    (dict(B=1 << 20, L=1), W.ERR_UNSUPPORTED, "2^24"),
    (dict(qg=48), W.ERR_INVALID_ARG, "quant_group"),
    (dict(k=MIS), W.ERR_INVALID_ARG, "k_cache is not 16-byte aligned"),
    (dict(v=None), W.ERR_INVALID_ARG, "v_cache is NULL"),
    (dict(o=None), W.ERR_INVALID_ARG, "o is NULL"),
    (dict(q=MIS), W.ERR_INVALID_ARG, "q is not 16-byte aligned"),
    (dict(mask=None), W.ERR_INVALID_ARG, "mask is NULL"),
    (dict(ws_bytes=0), W.ERR_WORKSPACE, "workspace"),
    (dict(ws=None), W.ERR_WORKSPACE, "workspace"),
    (dict(layout=2), W.ERR_INVALID_ARG, "kv_layout"),
])
def test_attention_validation(kw, status, msg):
    assert attention(**kw) == status
    assert msg in err()


def test_attention_empty_and_workspace():
    assert attention(B=0, mask=None, q=None, k=None, v=None, o=None, ws=None, ws_bytes=0) == W.OK
    size = W.wide_attention_decode_kvq_workspace_size
    assert size(0, 8192, 32, 8, 128, 512, 32) == 0
    assert 0 < size(1, 50001, 32, 8, 128, 512, 32) < 1 << 30
    for bad in ((32, 8192, 32, 8, 64, 512, 32), (32, 8192, 32, 8, 128, 512, 33), (1 << 20, 1, 32, 8, 128, 512, 32)):
        assert size(*bad) == W.SIZE_MAX


def test_binding_refuses_host_tensors():
    """(the shape checks of the binding need device tensors: the GPU tests make them)"""
    k = torch.zeros(2, 8 * 128, dtype=torch.bfloat16)
    c = torch.zeros(2, 16, 8, 80, dtype=torch.uint8)
    with pytest.raises(ValueError, match="GPU"):
        W.wide_kv_quantize(k, k, c, c, 8, 128, 32)
    with pytest.raises(ValueError, match="GPU"):
        W.wide_kv_dequantize(c, c, 1, 8, 128, 32)
    with pytest.raises(ValueError, match="GPU"):
        W.wide_attention_decode_kvq(torch.zeros(2, 32 * 128, dtype=torch.bfloat16), c, c,
                                    torch.ones(2, 8, dtype=torch.uint8), 32, 8, 128, 512, 32)
