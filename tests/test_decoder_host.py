"""Refusals of the paged cache's entry points and of the grouped linear, found on
the host before anything is launched."""
import ctypes

import numpy as np
import pytest
import torch

import decoder_plain as plain
from paper_2607_24981_amd import ilw

OK, E_NULL, E_SHAPE, E_PARAM, E_UNSUP, E_WS = 0, -1, -2, -3, -4, -5
FAKE = 0x10000  # aligned, never dereferenced


def cache(**kw):
    f = dict(k=FAKE, v=FAKE, k_scale=FAKE, v_scale=FAKE, page_table=FAKE, n_pages=40, page_size=64,
             max_pages=8, kv_heads=2, head_dim=64)
    f.update(kw)
    return ilw.KVCacheStruct(*[f[n] for n, _ in ilw.KVCacheStruct._fields_])


def append(c=None, **kw):
    c = cache() if c is None else c
    f = dict(qkv=FAKE, ld=512, cu=FAKE, past=FAKE, rope=FAKE, rope_rows=512, rotary=64, inter=0,
             q=FAKE, q_scale=FAKE, tokens=4, seqs=0, max_new=2, heads=4)
    f.update(kw)
    return ilw.lib().ilw_cache_append(ctypes.byref(c) if c else None, *f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(), OK), (dict(seqs=3, tokens=0), OK), (dict(seqs=3, max_new=0), OK),
    (dict(tokens=-1), E_SHAPE), (dict(max_new=-1), E_SHAPE), (dict(seqs=-1), E_SHAPE),
    (dict(seqs=65536), E_SHAPE), (dict(heads=0), E_SHAPE), (dict(heads=5), E_SHAPE),  # ld < a row
    (dict(ld=520), E_SHAPE), (dict(ld=496), E_SHAPE), (dict(rotary=8), E_SHAPE),
    (dict(rotary=80), E_SHAPE), (dict(rotary=-16), E_SHAPE), (dict(inter=2), E_PARAM),
    (dict(rope_rows=511), E_SHAPE), (dict(rope_rows=0, rotary=0), OK),
    (dict(seqs=3, qkv=None), E_NULL), (dict(seqs=3, cu=None), E_NULL),
    (dict(seqs=3, past=None), E_NULL), (dict(seqs=3, rope=None), E_NULL),
    (dict(seqs=3, q=None), E_NULL), (dict(seqs=3, q_scale=None), E_NULL),
    (dict(seqs=3, qkv=FAKE + 8), E_PARAM), (dict(seqs=3, rope=FAKE + 4), E_PARAM),
    (dict(seqs=3, q=FAKE + 8), E_PARAM)])
def test_append_refusals(kw, code):
    assert append(**kw) == code
    assert bool(ilw.last_error()) == (code != OK)


@pytest.mark.parametrize("kw,code", [
    (dict(page_size=8), E_UNSUP), (dict(page_size=48), E_UNSUP), (dict(page_size=512), E_UNSUP),
    (dict(head_dim=96), E_UNSUP), (dict(head_dim=0), E_UNSUP), (dict(kv_heads=0), E_SHAPE),
    (dict(kv_heads=4097), E_SHAPE), (dict(n_pages=0), E_SHAPE), (dict(max_pages=0), E_SHAPE),
    (dict(max_pages=(1 << 14) + 1), E_UNSUP), (dict(n_pages=1 << 30), E_UNSUP),
    (dict(k=None), E_NULL), (dict(v=None), E_NULL), (dict(k_scale=None), E_NULL),
    (dict(v_scale=None), E_NULL), (dict(page_table=None), E_NULL), (dict(k=FAKE + 8), E_PARAM),
    (dict(v=FAKE + 4), E_PARAM)])
def test_cache_refusals(kw, code):
    c = cache(**kw)
    assert append(c, seqs=3, ld=4096, rope_rows=1 << 21, rotary=0) == code
    assert attention(c, seqs=3, max_len=0) == code
    assert ilw.lib().ilw_cache_attention_workspace_bytes(ctypes.byref(c), 3, 1, 0, 4, 0) == 0
    assert ilw.last_error()


def test_null_cache():
    assert append(False) == E_NULL and attention(False) == E_NULL


def attention(c=None, ap=None, **kw):
    c = cache() if c is None else c
    f = dict(q=FAKE, q_scale=FAKE, cu=FAKE, lens=FAKE, out=FAKE, tokens=4, seqs=0, max_q=2,
             max_len=512, heads=4)
    f.update({k: v for k, v in kw.items() if k in f})
    p = dict(score_mult=1 << 26, score_shift=34, out_mult=1 << 30, out_shift=44, causal=1, window=0)
    p.update({k: v for k, v in kw.items() if k in p})
    ws, size = kw.get("workspace", FAKE), kw.get("size", 1 << 40)
    st = ilw.CacheAttnParams(*p.values())
    return ilw.lib().ilw_cache_attention(ctypes.byref(c) if c else None, *f.values(),
                                         None if ap is False else ctypes.byref(st), ws, size, None)


@pytest.mark.parametrize("kw,code", [
    (dict(), OK), (dict(seqs=3, tokens=0), OK), (dict(seqs=3, max_q=0), OK),
    (dict(heads=0), E_SHAPE), (dict(heads=5), E_SHAPE), (dict(heads=1), E_SHAPE),
    (dict(max_q=-1), E_SHAPE), (dict(max_q=1 << 21), E_SHAPE), (dict(max_len=-1), E_SHAPE),
    (dict(max_len=513), E_SHAPE), (dict(tokens=-1), E_SHAPE), (dict(ap=False), E_NULL),
    (dict(score_mult=-1), E_PARAM), (dict(score_shift=16), E_PARAM),
    (dict(score_shift=63), E_PARAM), (dict(score_mult=(1 << 31) - 1, score_shift=30), E_PARAM),
    (dict(score_mult=65025, score_shift=16), E_PARAM),
    (dict(score_mult=130100, score_shift=17), E_PARAM),  # 33026 * 130100 / 2 is past 2^31
    (dict(score_mult=130000, score_shift=17), OK),
    (dict(out_mult=-2 ** 31), E_PARAM), (dict(out_shift=0), E_PARAM), (dict(out_shift=63), E_PARAM),
    (dict(causal=2), E_PARAM), (dict(window=-1), E_PARAM), (dict(window=5, causal=0), E_PARAM),
    (dict(window=5), OK), (dict(seqs=3, q=None), E_NULL), (dict(seqs=3, q_scale=None), E_NULL),
    (dict(seqs=3, cu=None), E_NULL), (dict(seqs=3, lens=None), E_NULL),
    (dict(seqs=3, out=None), E_NULL), (dict(seqs=3, q=FAKE + 8), E_PARAM),
    (dict(seqs=3, out=FAKE + 4), E_PARAM)])
def test_attention_refusals(kw, code):
    assert attention(**kw) == code
    assert bool(ilw.last_error()) == (code != OK)


def test_attention_workspace():
    """Grows with the keys that can be seen, and the call wants as much."""
    def need(max_q, max_len, window, seqs=8):
        return ilw.lib().ilw_cache_attention_workspace_bytes(
            ctypes.byref(cache(max_pages=2048)), seqs, max_q, max_len, 4, window)
    assert need(1, 500, 0) == 0 and need(1, 0, 0) == 0 and need(0, 5000, 0) == 0
    assert 0 < need(1, 20000, 0) < need(1, 100000, 0)
    assert need(1, 100000, 4096) < need(1, 100000, 0)
    assert need(1, 100000, 2 ** 31 - 1) == need(1, 100000, 0)
    assert need(1, 100000, -1) == 0 and ilw.last_error()
    big = cache(max_pages=2048)
    n = need(1, 20000, 0)
    for ws, size in [(None, n), (FAKE, n - 1)]:
        assert attention(big, seqs=8, max_q=1, max_len=20000, workspace=ws, size=size) == E_WS
    assert attention(big, seqs=8, max_q=1, max_len=20000, workspace=FAKE + 8, size=n) == E_PARAM


def test_attention_rows_limit():
    assert attention(cache(kv_heads=1), heads=4096, max_q=1 << 20) == E_UNSUP


def test_launch_limits():
    """More workgroups than a launch holds."""
    assert append(seqs=65535, max_new=1 << 20, tokens=1 << 20) == E_UNSUP
    assert attention(seqs=65535, max_q=8192, heads=8) == E_UNSUP


def grouped(**kw):
    f = dict(x=FAKE, x_rows=10, rows=None, offsets=FAKE, w=FAKE, b=None,
             rq=ilw.Dyadic(FAKE, FAKE, 3 * 32), y=FAKE, M=10, experts=3, N=32, K=64)
    f.update(kw)
    return ilw.lib().ilw_linear_grouped(*f.values(), None)


@pytest.mark.parametrize("kw,code", [
    (dict(M=0), OK), (dict(M=-1), E_SHAPE), (dict(x_rows=-1), E_SHAPE), (dict(x_rows=9), E_SHAPE),
    (dict(x_rows=0, rows=FAKE), E_SHAPE), (dict(N=24), E_SHAPE), (dict(N=0), E_SHAPE),
    (dict(K=40), E_SHAPE), (dict(K=0), E_SHAPE), (dict(K=131088), E_UNSUP),
    (dict(experts=0), E_SHAPE), (dict(experts=1025), E_SHAPE), (dict(M=1 << 31, x_rows=1 << 31), E_UNSUP),
    (dict(N=1 << 30), E_UNSUP), (dict(M=1 << 28, x_rows=1 << 28), E_UNSUP), (dict(x=None), E_NULL), (dict(w=None), E_NULL),
    (dict(y=None), E_NULL), (dict(offsets=None), E_NULL), (dict(x=FAKE + 8), E_PARAM),
    (dict(w=FAKE + 4), E_PARAM), (dict(y=FAKE + 2), E_PARAM),
    (dict(rq=ilw.Dyadic(FAKE, FAKE, 32)), E_SHAPE), (dict(rq=ilw.Dyadic(None, FAKE, 1)), E_NULL),
    (dict(rq=ilw.Dyadic(FAKE, None, 1)), E_NULL)])
def test_grouped_refusals(kw, code):
    assert grouped(**kw) == code
    assert bool(ilw.last_error()) == (code != OK)


def test_binding_refuses_host_tensors_and_shapes():
    z = torch.zeros
    k = z(4, 2, 16, 64, dtype=torch.int8)
    s, t = z(4, 2, dtype=torch.int32), z(2, 2, dtype=torch.int32)
    for bad in [(k, k, s, s, t), (k, k[:3], s, s, t), (k, k, s[:, :1], s, t), (k[0], k[0], s, s, t),
                (k, k, s, s, t[0])]:
        with pytest.raises(ilw.IlwError):
            ilw.KVCache(*bad)
    with pytest.raises(ilw.IlwError):
        ilw.ilw_linear_grouped(z(4, 32, dtype=torch.int8), z(2, 16, 32, dtype=torch.int8),
                               z(3, dtype=torch.int32), None, s, s)
    with pytest.raises(ilw.IlwError):
        ilw.ilw_linear_grouped(z(4, 16, dtype=torch.int8), z(2, 16, 32, dtype=torch.int8),
                               z(3, dtype=torch.int32), None, s, s)


def host_cache(monkeypatch, seqs=2, max_pages=3):
    """A cache of host tensors, which no call is given."""
    monkeypatch.setattr(ilw, "_device", lambda t, name: -1)
    z = torch.zeros
    k, v = (z(4, 2, 16, 64, dtype=torch.int8) for _ in range(2))
    ks, vs = (z(4, 2, dtype=torch.int32) for _ in range(2))
    return ilw.KVCache(k, v, ks, vs, z(seqs, max_pages, dtype=torch.int32))


def test_cache_follows_its_page_table(monkeypatch):
    """A page table set later is the one that calls get, and its sequences."""
    cache = host_cache(monkeypatch)
    fixed = {n: getattr(cache.struct, n) for n, _ in ilw.KVCacheStruct._fields_}
    table = torch.ones(5, 7, dtype=torch.int32)
    cache.page_table = table
    fixed.update(page_table=table.data_ptr(), max_pages=7)
    assert {n: getattr(cache.struct, n) for n, _ in ilw.KVCacheStruct._fields_} == fixed
    assert cache.page_table is table and cache.seqs == 5
    for bad in [table[0], table.long(), torch.ones(5, 8, dtype=torch.int32)[:, :7], table.t()]:
        with pytest.raises(ilw.IlwError):
            cache.page_table = bad
        assert cache.page_table is table and cache.struct.page_table == table.data_ptr()


def test_cache_keeps_what_it_was_made_with(monkeypatch):
    """Nothing else changes beside the addresses that calls go by."""
    cache = host_cache(monkeypatch)
    for name in ["k", "v", "k_scale", "v_scale", "struct", "seqs", "kv_heads", "page_size",
                 "head_dim", "device"]:
        was = getattr(cache, name)
        with pytest.raises(ilw.IlwError, match=name):
            setattr(cache, name, torch.zeros(4, 2, 16, 64, dtype=torch.int8))
        with pytest.raises(ilw.IlwError):
            delattr(cache, name)
        assert getattr(cache, name) is was
    for name in ("k", "v", "k_scale", "v_scale"):
        assert getattr(cache.struct, name) == getattr(cache, name).data_ptr()


# ------------------------------------------- the plain forms that the GPU meets
@pytest.mark.parametrize("P,D", [(16, 32), (32, 64), (64, 128), (128, 256), (256, 32)])
def test_value_order_is_a_permutation(P, D):
    at = plain.value_place(P, D)
    assert sorted(at.reshape(-1)) == list(range(P * D))
    # four tokens of a channel are a word, 16 channels of 64 tokens 1024 bytes
    assert (at[0::4] % 4 == 0).all() and (at[1::4] == at[0::4] + 1).all()
    G = min(P, 64)
    assert (at[:G, :16] < 16 * G).all()


def test_weights_are_the_chord():
    """w between the chord of 2^(16 - a/64) and one below it; at whole octaves exact."""
    for a in range(17 * 64 + 1):
        n = -(-a // 64)
        w = ((64 + 64 * n - a) << 16) >> (n + 6)
        line = 2.0 ** (16 - n) * (1 + (64 * n - a) / 64)
        assert line - 1 < w <= line
        assert 2.0 ** (16 - a / 64) - 1 < w < 1.0615 * 2.0 ** (16 - a / 64) + 1e-9


def test_codes_stay_in_range():
    for A in list(range(0, 600)) + [2 ** 14, 127 * 2 ** 14, 128 * 2 ** 14, 2 ** 22]:
        v = np.array([A, -A, A // 2])
        S = plain.need(v)
        c = plain.codes(v.astype(np.int64), S)
        assert abs(c).max() <= 127 and (abs(2 * (c * S - v)) <= S).all()
