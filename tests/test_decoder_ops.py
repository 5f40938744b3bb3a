"""The paged int8 cache (append, attention) and the grouped linear against plain
64-bit forms.  Every operation is integer: results are equal or wrong."""
import numpy as np
import pytest
import torch

import decoder_plain as plain
from paper_2607_24981_amd import ilw

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]


def say(msg):
    print(f"[gpu] {msg}", flush=True)


def dev(a):
    return ilw.to_device(a)


def same(got, want, what):
    got = got.cpu().numpy() if isinstance(got, torch.Tensor) else got
    bad = np.flatnonzero(got.reshape(-1) != want.reshape(-1))
    assert got.shape == want.shape and not bad.size, (
        what, got.shape, want.shape, bad.size, bad[:5], got.reshape(-1)[bad[:5]],
        want.reshape(-1)[bad[:5]])


def rng(*seed):
    return np.random.Generator(np.random.PCG64(seed))


def make_cache(g, seqs, max_pages, hk, P, D, spare=3, lo=9000, hi=21000):
    n = seqs * max_pages + spare
    c = {"k": g.integers(-127, 128, (n, hk, P, D)).astype(np.int8),
         "v": g.integers(-127, 128, (n, hk, P, D)).astype(np.int8),
         "k_scale": g.integers(lo, hi, (n, hk)).astype(np.int32),
         "v_scale": g.integers(lo // 2, 16500, (n, hk)).astype(np.int32)}
    c["table"] = g.permutation(n)[:seqs * max_pages].reshape(seqs, max_pages).astype(np.int32)
    return c


def on_device(c):
    return ilw.KVCache(*[dev(c[k]) for k in ("k", "v", "k_scale", "v_scale", "table")])


def same_cache(cache, c, what):
    for name in ("k", "v", "k_scale", "v_scale"):
        same(getattr(cache, name), c[name], f"{what}: {name}")


def rope_of(rows, R):
    return ilw.rope_table(rows, R, device="cpu").numpy() if R else None


# -------------------------------------------------------------------- append
def run_append(c, qkv, heads, new, past, max_new, rope, inter, what, first=0, ld=0, pad=0):
    """One call on the GPU and one of the plain form, from the same state."""
    say(f"append {what}")
    hk, P, D = c["k"].shape[1:]
    cu = first + np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = qkv.shape[0]
    cache = on_device(c)
    x = dev(qkv)
    if ld:
        wide = torch.full((T, ld), 99, dtype=torch.int8, device="cuda")
        wide[:, :x.shape[1]] = x
        x = wide[:, :x.shape[1]]
    q = torch.full((T, heads, D), 90, dtype=torch.int8, device="cuda")
    qs = torch.full((T, heads), 91, dtype=torch.int32, device="cuda")
    want_q, want_s = q.cpu().numpy().copy(), qs.cpu().numpy().copy()
    ilw.ilw_cache_append(cache, x, heads, dev(cu), dev(np.asarray(past, np.int32)), max_new,
                         rope=None if rope is None else dev(rope), interleaved=inter, q=q,
                         q_scale=qs)
    plain.append(c, qkv, heads, cu.tolist(), list(past), max_new, rope, inter, want_q, want_s)
    torch.cuda.synchronize()
    same(q, want_q, f"{what}: q")
    same(qs, want_s, f"{what}: q_scale")
    same_cache(cache, c, what)


@pytest.mark.parametrize("P,D,heads,hk,R,inter", [
    (16, 64, 8, 2, 64, False), (64, 128, 4, 1, 128, False), (32, 32, 6, 3, 16, False),
    (128, 256, 3, 3, 128, True), (16, 32, 2, 1, 32, True), (256, 64, 5, 1, 0, False),
    (64, 64, 14, 2, 48, True), (32, 128, 1, 1, 112, False)])
@pytest.mark.parametrize("few", [True, False])
def test_append(P, D, heads, hk, R, inter, few):
    g = rng(P, D, heads, few)
    # sequences that start a page, fill one, cross one, end one, add nothing
    new = [1, 0, 3, 2, 1, 8, 1] if few else [P + 3, 0, 1, 2 * P, 9, P - 1]
    past = [0, 5, P - 1, P - 2, P, 2 * P - 3, 7] if few else [P // 2, 3, P - 1, 1, 0, P + 1]
    c = make_cache(g, len(new), 5, hk, P, D)
    T = sum(new)
    qkv = np.clip(np.rint(g.normal(0, 42, (T, (heads + 2 * hk) * D))), -127, 127).astype(np.int8)
    qkv[T // 2:] //= 3  # smaller rows: pages that keep their scale
    run_append(c, qkv, heads, new, past, max(new), rope_of(5 * P, R), inter,
               f"P={P} D={D} heads={heads}/{hk} R={R} inter={inter} few={few}")


def test_append_extremes():
    """The lowest code, zeros, one value: the largest and the smallest scales."""
    P, D, heads, hk = 16, 64, 2, 1
    c = make_cache(rng(3), 3, 2, hk, P, D)
    qkv = np.zeros((12, 4 * D), np.int8)
    qkv[:4] = -128
    qkv[8, ::7] = 127
    qkv[9:, :] = np.where(np.arange(4 * D) % 2, -128, 127)
    run_append(c, qkv, heads, [4, 4, 4], [0, 3, 0], 4, rope_of(2 * P, D), False, "extremes")
    assert c["k_scale"].max() <= 37154 and c["v_scale"].max() <= 18577


@pytest.mark.parametrize("few", [True, False])
def test_append_limits(few):
    """Rows outside every sequence, more new tokens than max_new, past the
    table's end, pages that are not there, strided rows."""
    P, D, heads, hk = 16, 64, 4, 2
    g = rng(5, few)
    k = 1 if few else 3
    c = make_cache(g, 4, 4, hk, P, D)
    c["table"][0, 1] = -1
    c["table"][1, 0] = c["k"].shape[0]
    c["table"][1, 1] = 2 ** 31 - 1
    new, past = [4 * k, 6 * k, 5 * k, 9 * k], [14, 13, 4 * P - 3, 2 * P + 2]
    T = sum(new) + 9
    qkv = g.integers(-127, 128, (T, (heads + 2 * hk) * D)).astype(np.int8)
    run_append(c, qkv, heads, new, past, 7 * k, rope_of(4 * P, 32), False, f"limits few={few}",
               first=4, ld=(heads + 2 * hk) * D + 48)


def test_append_token_by_token():
    """A page filled one token a call, scales growing on the way."""
    P, D, heads, hk = 32, 64, 2, 1
    g = rng(6)
    c = make_cache(g, 2, 2, hk, P, D)
    rope = rope_of(2 * P, D)
    for i in range(P + 4):
        qkv = np.rint(g.normal(0, 2 + 1.2 * i, (2, (heads + 2 * hk) * D))).clip(-127, 127).astype(np.int8)
        run_append(c, qkv, heads, [1, 1], [i, i], 1, rope, True, f"token {i}")


# ----------------------------------------------------------------- attention
def params(D, octaves=2.0):
    ratio = 64 * octaves / (73.0 * 73.0 * np.sqrt(D)) / 0.84
    shift = 27 - int(np.floor(np.log2(ratio)))
    return {"score_mult": int(ratio * 2 ** shift), "score_shift": shift, "out_mult": 1 << 30,
            "out_shift": 30 + 16 - 2}


def run_attention(c, heads, new, lens, p, causal, window, what, max_q=None, max_len=None, first=0,
                  pad=0, g=None, q=None, q_scale=None):
    say(f"attention {what}")
    hk, P, D = c["k"].shape[1:]
    cu = first + np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    T = int(cu[-1]) + pad
    if q is None:
        q = g.integers(-127, 128, (T, heads, D)).astype(np.int8)
    if q_scale is None:
        q_scale = g.integers(9000, 21000, (T, heads)).astype(np.int32)
    max_q = max(new) if max_q is None else max_q
    max_len = c["table"].shape[1] * P if max_len is None else max_len
    out = torch.full((T, heads * D), 77, dtype=torch.int8, device="cuda")
    want = np.full((T, heads, D), 77, np.int8)
    ilw.ilw_cache_attention(on_device(c), dev(q), dev(q_scale), dev(cu),
                            dev(np.asarray(lens, np.int32)), p, max_q, max_len, causal=causal,
                            window=window, out=out)
    plain.attention(c, q, q_scale, cu.tolist(), list(lens), p, max_q, max_len, causal, window, want)
    torch.cuda.synchronize()
    same(out.view(T, heads, D), want, what)
    return want


@pytest.mark.parametrize("D", [32, 64, 128, 256])
@pytest.mark.parametrize("P", [16, 32, 64, 128])
def test_attention_single_tokens(D, P):
    """One query a sequence, lengths around every boundary, none among them."""
    lens = [0, 1, 2, 15, 16, 17, 63, 64, 65, 127, 128, 129, 200, 300]
    for heads, hk in [(4, 2), (5, 1), (3, 3)]:
        g = rng(D, P, heads)
        c = make_cache(g, len(lens), -(-300 // P), hk, P, D)
        want = run_attention(c, heads, [1] * len(lens), lens, params(D), True, 0,
                             f"decode D={D} P={P} heads={heads}/{hk}", g=g)
        assert not want[0].any() and want[1:].any()


@pytest.mark.parametrize("D", [32, 64, 128, 256])
def test_attention_most_of_one_workgroup(D):
    """16 rows of 1024 keys: the most scores that one workgroup keeps; one more
    key is split.  The rows of one query, and those of sixteen."""
    for heads, new, P in [(16, 1, 16), (1, 16, 64), (5, 3, 32)]:
        for longest in (1024, 1024 + P):
            g = rng(D, heads, longest)
            c = make_cache(g, 3, longest // P, 1, P, D)
            run_attention(c, heads, [new, 1, new], [longest, 3, 1024], params(D), True, 0,
                          f"D={D} heads={heads} new={new} longest={longest}", g=g)


@pytest.mark.parametrize("D,P,heads,hk", [(64, 16, 4, 2), (128, 64, 8, 2), (32, 32, 7, 1),
                                          (256, 128, 2, 2), (128, 16, 12, 1), (64, 256, 3, 3)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 1), (True, 70)])
def test_attention_rows(D, P, heads, hk, causal, window):
    """Several queries a sequence; more of them than keys, so that the first see none."""
    new, lens = [37, 1, 5, 130, 0, 64], [100, 33, 3, 130, 9, 257]
    g = rng(D, P, heads, causal, window)
    c = make_cache(g, len(new), -(-257 // P), hk, P, D)
    run_attention(c, heads, new, lens, params(D), causal, window,
                  f"rows D={D} P={P} heads={heads}/{hk} causal={causal} window={window}", g=g,
                  first=3, pad=5)


@pytest.mark.parametrize("D,P,heads,hk", [(64, 64, 6, 2), (128, 16, 4, 1), (32, 32, 2, 2),
                                          (256, 128, 3, 1), (128, 64, 16, 2), (64, 16, 5, 1)])
@pytest.mark.parametrize("new,window", [(1, 0), (1, 1500), (11, 0), (9, 700)])
def test_attention_long(D, P, heads, hk, new, window):
    """Keys split over workgroups: lengths around the parts' borders, in one
    call with short and empty ones; the parts of a window start anywhere."""
    lens = [2600, 1, 511, 512, 513, 1025, 0, 2048, 1536]
    g = rng(D, P, heads, new, window)
    c = make_cache(g, len(lens), -(-2600 // P), hk, P, D)
    c["table"][2, 3] = -1
    counts = [new] * 4 + [max(1, new // 2)] * 5
    run_attention(c, heads, counts, lens, params(D), True, window,
                  f"long D={D} P={P} heads={heads}/{hk} new={new} window={window}", g=g)


@pytest.mark.parametrize("D,P,heads,hk", [(64, 16, 8, 4), (128, 64, 6, 3), (32, 32, 4, 4),
                                          (256, 128, 4, 4), (128, 16, 3, 3), (32, 16, 8, 4),
                                          (256, 16, 4, 4), (64, 256, 5, 5), (128, 32, 4, 4)])
@pytest.mark.parametrize("causal,window", [(True, 0), (False, 0), (True, 45)])
def test_attention_many_rows(D, P, heads, hk, causal, window):
    """Grids that fill the GPU with the rows of prompts: 192 tiles and more."""
    seqs = 64 if hk > 3 else 80
    g = rng(D, P, heads, causal, window)
    new = [int(x) for x in g.integers(0, 12, seqs)]
    lens = [n + int(x) for n, x in zip(new, g.integers(0, 60, seqs))]
    G = heads // hk
    new[3], lens[3] = 70 // G + 40, 70 // G + 41      # over one tile, the last partly filled
    new[5], lens[5] = 90, 50                          # more queries than keys
    new[7], lens[7] = 66, 0
    new[9], lens[9] = 130 // G, 300
    c = make_cache(g, seqs, -(-300 // P), hk, P, D)
    c["table"][9, ::2] = -1
    run_attention(c, heads, new, lens, params(D), causal, window,
                  f"many rows D={D} P={P} heads={heads}/{hk} causal={causal} window={window}", g=g,
                  first=2, pad=3)


@pytest.mark.parametrize("octaves", [0.0, 0.02, 30.0, 500.0, 4000.0])
def test_attention_score_ranges(octaves):
    """Flat rows, single peaks, scores past 16 bits; a scale that is refused."""
    D, P, heads, hk = 64, 32, 4, 2
    g = rng(int(octaves * 100))
    p = params(D, max(octaves, 0.02))
    if octaves == 0.0:
        p["score_mult"] = 0
    c = make_cache(g, 3, 12, hk, P, D)
    if octaves > 600:  # 33026 * score_mult / 2^(score_shift - 16) past 2^31
        with pytest.raises(ilw.IlwError, match="too large"):
            run_attention(c, heads, [1, 1, 1], [1, 1, 1], p, True, 0, "refused", g=g)
        return
    run_attention(c, heads, [1, 20, 3], [380, 200, 3], p, True, 0, f"octaves={octaves}", g=g)


def test_attention_extreme_codes():
    """Largest codes and scales on both sides, equal rows, opposite rows."""
    D, P, heads, hk = 256, 64, 2, 1
    g = rng(8)
    c = make_cache(g, 2, 4, hk, P, D)
    c["k"][:], c["v"][:] = 127, -127
    c["k"][c["table"][1]] = -128
    c["k_scale"][:], c["v_scale"][:] = 37154, 18577
    q = np.full((6, heads, D), 127, np.int8)
    q[1::2] = -128
    p = {"score_mult": 63000, "score_shift": 16 + 16, "out_mult": (1 << 31) - 1, "out_shift": 46}
    run_attention(c, heads, [3, 3], [256, 255], p, True, 0, "extreme codes", q=q,
                  q_scale=np.full((6, heads), 33026, np.int32))
    p = {"score_mult": (1 << 31) - 1, "score_shift": 62, "out_mult": -(1 << 30), "out_shift": 62}
    run_attention(c, heads, [3, 3], [256, 255], p, False, 0, "smallest scale", q=q,
                  q_scale=np.full((6, heads), 1, np.int32))


def test_attention_limits():
    """Pages that are not there, max_q and max_len below what the arrays say."""
    D, P, heads, hk = 64, 16, 4, 2
    g = rng(9)
    c = make_cache(g, 5, 20, hk, P, D)
    n = c["k"].shape[0]
    c["table"][0, 2:9] = -1
    c["table"][1, :] = n
    c["table"][2, ::3] = 2 ** 31 - 1
    c["table"][3, 19] = -2 ** 31
    new, lens = [3, 2, 30, 40, 9], [320, 100, 200, 320, 313]
    run_attention(c, heads, new, lens, params(D), True, 0, "bad pages", g=g)
    run_attention(c, heads, new, lens, params(D), True, 50, "bad pages, window", g=g)
    run_attention(c, heads, new, lens, params(D), True, 0, "max_q, max_len", g=g, max_q=17,
                  max_len=210)
    run_attention(c, heads, new, lens, params(D), False, 0, "max_len 0", g=g, max_len=0)


# ------------------------------------------------------------------- grouped
def run_grouped(g, counts, N, K, x_rows=0, bias=True, per_tensor=False, first=0, pad=0, rows=None,
                shifts=(38, 42), y_off=0):
    E = len(counts)
    off = first + np.concatenate([[0], np.cumsum(counts)]).astype(np.int32)
    M = int(off[-1]) + pad
    say(f"grouped M={M} E={E} N={N} K={K} rows={x_rows} bias={bias} per_tensor={per_tensor}")
    x = g.integers(-127, 128, (x_rows or M, K)).astype(np.int8)
    if x_rows and rows is None:
        rows = g.integers(0, x_rows, M).astype(np.int32)
    w = g.integers(-127, 128, (E, N, K)).astype(np.int8)
    b = g.integers(-2 ** 15, 2 ** 15, (E, N)).astype(np.int32) if bias else None
    size = (1,) if per_tensor else (E, N)
    mult = g.integers(2 ** 29, 2 ** 30, size).astype(np.int32)
    shift = g.integers(*shifts, size).astype(np.int32)
    buf = torch.full((M * N + 64,), 77, dtype=torch.int8, device="cuda")
    y = buf[16 + y_off:16 + y_off + M * N].view(M, N)
    want = np.full((M, N), 77, np.int8)
    ilw.ilw_linear_grouped(dev(x), dev(w), dev(off), None if b is None else dev(b), dev(mult),
                           dev(shift), rows=None if rows is None else dev(rows), y=y)
    plain.grouped(x, rows, off, w, b, mult, shift, want)
    torch.cuda.synchronize()
    same(y, want, "grouped")
    assert bool((buf[:16 + y_off] == 77).all()) and bool((buf[16 + y_off + M * N:] == 77).all())


@pytest.mark.parametrize("counts", [[1], [0, 0, 5], [16, 1, 0, 33, 7], [130, 0, 300, 2], [1] * 70,
                                    [0] * 100 + [3] + [0] * 40 + [129]])
@pytest.mark.parametrize("N,K", [(16, 16), (48, 208), (272, 128), (528, 1040)])
def test_grouped(counts, N, K):
    g = rng(len(counts), N, K)
    run_grouped(g, counts, N, K)
    run_grouped(g, counts, N, K, x_rows=13, bias=False, per_tensor=True, first=3, pad=4)


def test_grouped_row_index():
    """The same row twice, rows out of range (zeros), an unaligned output."""
    g = rng(4)
    rows = np.array([3, 3, 0, -1, 8, 9, 2 ** 31 - 1, -2 ** 31, 7, 1], np.int32)
    run_grouped(g, [4, 0, 6], 64, 96, x_rows=9, rows=rows, y_off=4)
    run_grouped(g, [4, 0, 6], 64, 96, x_rows=9, rows=rows, bias=False, shifts=(1, 63), y_off=8)


@pytest.mark.parametrize("counts,N,K", [([2000, 3, 900], 320, 256), ([300] * 9, 1024, 144),
                                        ([2500, 2100], 1040, 1024)])
def test_grouped_large(counts, N, K):
    run_grouped(rng(N, K), counts, N, K, x_rows=500)


# Many rows an expert, rows that fill no tile, and many experts of few rows: the
# tiles differ; K in whole steps and not.
@pytest.mark.parametrize("counts,N", [([900, 0, 1189, 0, 3], 4224), ([257] * 2 + [150], 1104),
                                      ([3] * 171 + [70] + [0] * 84, 528), ([65, 63], 48)])
@pytest.mark.parametrize("K", [48, 256])
def test_grouped_tiles(counts, N, K):
    run_grouped(rng(N, K), counts, N, K, x_rows=200, pad=2)


# ------------------------------------------------------------- larger numbers
def scattered(g, seqs, max_pages, hk, P, D, n=40):
    """A small pool that long sequences name again and again."""
    c = make_cache(g, 1, n, hk, P, D, spare=0)
    c["table"] = g.integers(0, n, (seqs, max_pages)).astype(np.int32)
    return c


@pytest.mark.parametrize("D,P", [(32, 64), (64, 16), (128, 64), (256, 32)])
def test_attention_many_rows_steep(D, P):
    """Scores far past 16 bits before they are clamped, by the rows of prompts."""
    hk, heads, seqs = 4, 8, 60
    g = rng(D, P, 5)
    p = params(D, 60.0 * np.sqrt(D))  # a ninth below what is refused
    assert (33026 * p["score_mult"] >> (p["score_shift"] - 16)) * 37154 >> 16 >= 1 << 27
    c = make_cache(g, seqs, -(-200 // P), hk, P, D)
    c["k_scale"][::3] = 37154
    new = [40, 33] + [int(x) for x in g.integers(0, 4, seqs - 2)]
    lens = [200, 20] + [int(x) for x in g.integers(0, 100, seqs - 2)]
    run_attention(c, heads, new, lens, p, True, 0, f"steep D={D} P={P}", g=g)


@pytest.mark.parametrize("max_len", [131072, 131072 + 256])
@pytest.mark.parametrize("flat", [False, True])
def test_attention_long_prompt(max_len, flat):
    """The longest sequence whose sums one kernel takes, and one that is split;
    flat scores give the largest sums there are."""
    D, P, hk, heads, seqs = 32, 256, 4, 4, 48
    g = rng(max_len, flat)
    c = scattered(g, seqs, max_len // P, hk, P, D)
    p = params(D)
    if flat:
        p["score_mult"] = 0
        c["v"][:] = np.where(g.integers(0, 20, c["v"].shape) > 0, -127, 127)
        c["v_scale"][:] = 18577
    new = [3, 66] + [1] * (seqs - 2)
    lens = [max_len, 70] + [int(x) for x in g.integers(0, 90, seqs - 2)]
    run_attention(c, heads, new, lens, p, True, 0, f"long prompt {max_len} flat={flat}", g=g)


def test_pool_past_32_bits():
    """Pages whose bytes lie past 2^32 of the pools."""
    D, P, hk, heads, seqs, max_pages = 64, 256, 1, 2, 3, 13
    n = (1 << 32) // (P * D * hk) + 64
    g = rng(12)
    c = make_cache(g, seqs, max_pages, hk, P, D, spare=0)
    used = c["k"].shape[0]
    say(f"pools of {n * hk * P * D} bytes")
    big = {"k": torch.empty((n, hk, P, D), dtype=torch.int8, device="cuda"),
           "v": torch.empty((n, hk, P, D), dtype=torch.int8, device="cuda"),
           "k_scale": torch.ones((n, hk), dtype=torch.int32, device="cuda"),
           "v_scale": torch.ones((n, hk), dtype=torch.int32, device="cuda")}
    for name, t in big.items():
        t[n - used:] = dev(c[name])
    cache = ilw.KVCache(big["k"], big["v"], big["k_scale"], big["v_scale"],
                        dev(c["table"] + (n - used)))
    rope = rope_of(max_pages * P, D)
    for new, past in [([1, 0, 1], [2500, 0, 255]), ([30, 290, 11], [3000, 200, 0])]:
        T = sum(new)
        cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
        qkv = g.integers(-127, 128, (T, (heads + 2 * hk) * D)).astype(np.int8)
        q, qs = ilw.ilw_cache_append(cache, dev(qkv), heads, dev(cu), dev(np.array(past, np.int32)),
                                     max(new), rope=dev(rope))
        want_q, want_s = np.zeros((T, heads, D), np.int8), np.zeros((T, heads), np.int32)
        plain.append(c, qkv, heads, cu.tolist(), past, max(new), rope, False, want_q, want_s)
        same(q, want_q, "q")
        for name in big:
            same(big[name][n - used:], c[name], name)
        lens = [a + b for a, b in zip(new, past)]
        out = ilw.ilw_cache_attention(cache, q, qs, dev(cu), dev(np.array(lens, np.int32)),
                                      params(D), max(new), max(lens))
        want = np.zeros((T, heads, D), np.int8)
        plain.attention(c, want_q, want_s, cu.tolist(), lens, params(D), max(new), max(lens), True,
                        0, want)
        same(out.view(T, heads, D), want, "attention")


def test_grouped_past_32_bits():
    """An output and weights of more than 2^31 and 2^32 bytes; the last rows."""
    for M, E, N, K in [(70000, 2, 32768, 16), (1200, 1024, 1024, 4112)]:
        say(f"grouped M={M} E={E} N={N} K={K}")
        g = rng(M, N)
        w = torch.randint(-127, 128, (E, N, K), dtype=torch.int8, device="cuda")
        x = g.integers(-127, 128, (M, K)).astype(np.int8)
        cut = M - 9 if E == 2 else M - E
        off = np.array([0, cut, M] if E == 2 else [0] + [cut + 1 + e for e in range(E)], np.int32)
        mult, shift = np.array([1 << 29], np.int32), np.array([38], np.int32)
        y = ilw.ilw_linear_grouped(dev(x), w, dev(off), None, dev(mult), dev(shift))
        rows = [cut - 1, cut, cut + 1, M - 1]
        for r in rows:
            e = int(np.searchsorted(off, r, side="right")) - 1
            want = np.zeros((1, N), np.int8)
            plain.grouped(x[r:r + 1], None, [0, 1], w[e:e + 1].cpu().numpy(), None, mult, shift, want)
            same(y[r:r + 1], want, f"row {r}")
        del w, y


# ---------------------------------------------- as they are used, one after another
class Layer:
    """A decoder layer with experts: linear, append, attention, linear, experts
    up, GELU, experts down; every step's input is the step before."""

    def __init__(self, g, hidden=128, heads=4, hk=2, D=64, E=5, ffn=96):
        def lin(n, k, e=None):
            shape = (n, k) if e is None else (e, n, k)
            w = g.integers(-127, 128, shape).astype(np.int8)
            b = g.integers(-2 ** 12, 2 ** 12, shape[:-1]).astype(np.int32)
            # (73^2 sqrt(k) of an accumulator to about 42 of a code)
            rq = 42 / (73.0 * 73.0 * np.sqrt(k)) * g.uniform(0.9, 1.1, shape[:-1])
            return w, b, np.rint(rq * 2.0 ** 38).astype(np.int32), np.full(shape[:-1], 38, np.int32)
        self.heads, self.hk, self.D = heads, hk, D
        self.host = {"qkv": lin((heads + 2 * hk) * D, hidden), "out": lin(hidden, heads * D),
                     "up": lin(ffn, hidden, E), "down": lin(hidden, ffn, E)}
        self.dev = {k: [dev(a) for a in v] for k, v in self.host.items()}
        self.params = params(D)
        self.rope = rope_of(4096, D)
        self.dev_rope = dev(self.rope)

    def run(self, cache, x, cu, past, lens, max_new, max_len, rows, offsets):
        d = self.dev
        w, b, m, s = d["qkv"]
        t = {"qkv": ilw.ilw_linear(x, w, b, m, s)}
        t["q"], t["qs"] = ilw.ilw_cache_append(cache, t["qkv"], self.heads, cu, past, max_new,
                                               rope=self.dev_rope)
        t["att"] = ilw.ilw_cache_attention(cache, t["q"], t["qs"], cu, lens, self.params, max_new,
                                           max_len)
        w, b, m, s = d["out"]
        t["out"] = ilw.ilw_linear(t["att"], w, b, m, s)
        w, b, m, s = d["up"]
        t["up"] = ilw.ilw_linear_grouped(t["out"], w, offsets, b, m, s, rows=rows)
        t["act"] = ilw.ilw_sdshiftgelu(t["up"], 50, 1 << 30, 37)
        w, b, m, s = d["down"]
        t["down"] = ilw.ilw_linear_grouped(t["act"], w, offsets, b, m, s)
        return t

    def check(self, c, t, x, cu, past, lens, max_new, max_len, rows, offsets):
        """Every step but GELU (tested elsewhere) from the step before."""
        T = len(x)

        def grouped(x, rows, offsets, p):
            w, b, m, s = [a if a.ndim > 1 and len(a) == len(offsets) - 1 else a[None] for a in p]
            y = np.zeros((int(offsets[-1]), w.shape[1]), np.int8)
            plain.grouped(x, rows, offsets, w, b, m, s, y)
            return y
        h = {k: v.cpu().numpy() for k, v in t.items()}
        same(t["qkv"], grouped(x, None, [0, T], self.host["qkv"]), "qkv")
        q, qs = np.zeros((T, self.heads, self.D), np.int8), np.zeros((T, self.heads), np.int32)
        plain.append(c, h["qkv"], self.heads, cu.tolist(), past.tolist(), max_new, self.rope, False,
                     q, qs)
        same(t["q"], q, "q")
        same(t["qs"], qs, "q_scale")
        att = np.zeros_like(q)
        plain.attention(c, q, qs, cu.tolist(), lens.tolist(), self.params, max_new, max_len, True, 0,
                        att)
        same(t["att"], att.reshape(T, -1), "attention")
        same(t["out"], grouped(h["att"], None, [0, T], self.host["out"]), "out")
        same(t["up"], grouped(h["out"], rows, offsets, self.host["up"]), "up")
        same(t["down"], grouped(h["act"], None, offsets, self.host["down"]), "down")
        assert h["down"].any()


def route(g, T, E, each=2):
    """Rows of T tokens sorted by expert, `each` experts a token."""
    e = np.stack([g.permutation(E)[:each] for _ in range(T)])
    order = np.argsort(e.reshape(-1), kind="stable")
    offsets = np.concatenate([[0], np.cumsum(np.bincount(e.reshape(-1), minlength=E))])
    return (order // each).astype(np.int32), offsets.astype(np.int32)


def test_decoder_layer_prompt_then_tokens():
    """A prompt, a second piece of it, then tokens one by one."""
    g = rng(21)
    L = Layer(g)
    c = make_cache(g, 3, 20, L.hk, 16, L.D)
    cache = on_device(c)
    past = np.zeros(3, np.int32)
    for new in [[130, 1, 17], [20, 40, 1]] + [[1, 1, 1]] * 4 + [[0, 2, 1]]:
        say(f"layer {new}")
        T, n = sum(new), np.array(new, np.int32)
        cu = np.concatenate([[0], np.cumsum(n)]).astype(np.int32)
        x = g.integers(-127, 128, (T, 128)).astype(np.int8)
        rows, offsets = route(g, T, 5)
        lens = past + n
        args = (cu, past, lens)
        t = L.run(cache, dev(x), *[dev(a) for a in args], max(new), int(lens.max()), dev(rows),
                  dev(offsets))
        L.check(c, t, x, *args, max(new), int(lens.max()), rows, offsets)
        same_cache(cache, c, "cache")
        past = lens


@pytest.mark.parametrize("max_len", [320, 4000])
def test_decoder_layer_captured(max_len):
    """One token of each sequence as a graph, replayed with other inputs and
    lengths in the same arrays, eager work between the replays; the attention is
    one launch (320) or three over a workspace of the graph's (4000)."""
    g = rng(22, max_len)
    L = Layer(g)
    seqs, P = 3, 16
    c = make_cache(g, seqs, max_len // P, L.hk, P, L.D)
    lens0 = np.array([max_len - 20, 5, max_len // 2], np.int32)
    cache, other = on_device(c), on_device(c)
    x = torch.zeros((seqs, 128), dtype=torch.int8, device="cuda")
    cu = dev(np.arange(seqs + 1, dtype=np.int32))
    past, lens = dev(lens0), dev(lens0 + 1)
    rows, offsets = [dev(a) for a in route(g, seqs, 5)]
    args = (cu, past, lens, 1, max_len, rows, offsets)
    s = torch.cuda.Stream()
    s.wait_stream(torch.cuda.current_stream())
    with torch.cuda.stream(s):
        L.run(cache, x, *args)  # (whatever a first call sets up)
    torch.cuda.current_stream().wait_stream(s)
    for name in ("k", "v", "k_scale", "v_scale"):
        getattr(cache, name).copy_(dev(c[name]))
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        t = L.run(cache, x, *args)
    for i in range(5):
        say(f"replay {i}")
        xi = g.integers(-127, 128, (seqs, 128)).astype(np.int8)
        r, o = route(g, seqs, 5)
        x.copy_(dev(xi))
        past.copy_(dev(lens0 + i))
        lens.copy_(dev(lens0 + i + 1))
        rows.copy_(dev(r))
        offsets.copy_(dev(o))
        graph.replay()
        eager = L.run(other, dev(xi), cu, dev(lens0 + i), dev(lens0 + i + 1), 1, max_len, dev(r), dev(o))
        torch.cuda.synchronize()
        for k in t:
            assert torch.equal(t[k], eager[k]), (i, k)
        for k in ("k", "v", "k_scale", "v_scale"):
            assert torch.equal(getattr(cache, k), getattr(other, k)), (i, k)
        L.check(c, t, xi, np.arange(seqs + 1), lens0 + i, lens0 + i + 1, 1, max_len, r, o)


def test_streams_side_by_side():
    """Two layers on two streams, neither the default one, each its own cache;
    inputs written on the stream that reads them."""
    g = rng(23)
    L = Layer(g)
    runs = []
    for i in range(2):
        c = make_cache(g, 2, 250, L.hk, 16, L.D)
        x = g.integers(-127, 128, (2, 128)).astype(np.int8)
        lens = np.array([3900, 60 + i], np.int32)
        rows, offsets = route(g, 2, 5)
        runs.append(dict(c=c, cache=on_device(c), x=x, lens=lens, rows=rows, offsets=offsets,
                         stream=torch.cuda.Stream()))
    cu = np.arange(3, dtype=np.int32)
    dcu = dev(cu)
    torch.cuda.synchronize()
    for _ in range(3):
        for r in runs:
            with torch.cuda.stream(r["stream"]):
                x = torch.zeros((2, 128), dtype=torch.int8, device="cuda")
                x += dev(r["x"])
                # (the token at lens - 1 is appended again, with what it had)
                r["t"] = L.run(r["cache"], x, dcu, dev(r["lens"] - 1), dev(r["lens"]), 1, 4000,
                               dev(r["rows"]), dev(r["offsets"]))
                r["keep"] = x
    torch.cuda.synchronize()
    for r in runs:
        for _ in range(2):  # the plain cache takes the same three appends
            plain.append(r["c"], r["t"]["qkv"].cpu().numpy(), L.heads, cu.tolist(),
                         (r["lens"] - 1).tolist(), 1, L.rope, False,
                         np.zeros((2, L.heads, L.D), np.int8), np.zeros((2, L.heads), np.int32))
        L.check(r["c"], r["t"], r["x"], cu, r["lens"] - 1, r["lens"], 1, 4000, r["rows"], r["offsets"])


@pytest.mark.parametrize("fill", [0, 0x7f, 0xff])
def test_workspace_of_any_content(fill):
    """A workspace of exactly the size asked for, holding anything."""
    D, P, heads, hk = 128, 64, 6, 2
    g = rng(24)
    c = make_cache(g, 2, 50, hk, P, D)
    c["table"][0, 3] = -1
    lens, new = [3100, 700], [2, 2]
    q = g.integers(-127, 128, (4, heads, D)).astype(np.int8)
    qs = g.integers(9000, 21000, (4, heads)).astype(np.int32)
    cache = on_device(c)
    need = ilw.lib().ilw_cache_attention_workspace_bytes(cache.struct, 2, 2, 3200, heads, 0)
    assert need > 0
    buf = torch.full((need + 512,), fill, dtype=torch.uint8, device="cuda")
    out = ilw.ilw_cache_attention(cache, dev(q), dev(qs), dev(np.array([0, 2, 4], np.int32)),
                                  dev(np.array(lens, np.int32)), params(D), 2, 3200,
                                  workspace=buf[256:256 + need].view(torch.int8))
    want = np.zeros((4, heads, D), np.int8)
    plain.attention(c, q, qs, [0, 2, 4], lens, params(D), 2, 3200, True, 0, want)
    same(out.view(4, heads, D), want, "attention")
    assert bool((buf[:256] == fill).all()) and bool((buf[256 + need:] == fill).all())


def test_decoder_stages_are_timed():
    """One entry a call, whatever it launches."""
    g = rng(25)
    L = Layer(g)
    c = make_cache(g, 1, 250, L.hk, 16, L.D)
    rows, offsets = route(g, 1, 5)
    cache, i32 = on_device(c), lambda *v: dev(np.array(v, np.int32))
    args = (cache, dev(g.integers(-127, 128, (1, 128)).astype(np.int8)), i32(0, 1), i32(3000),
            i32(3001), 1, 4000, dev(rows), dev(offsets))
    L.run(*args)
    ilw.profile_enable(True)
    try:
        for _ in range(3):
            L.run(*args)
        got = ilw.profile_read()
    finally:
        ilw.profile_enable(False)
    for stage, n in [("cache_append", 3), ("cache_attention", 3), ("gemm_grouped", 6)]:
        assert got[stage][1] == n and 0 < got[stage][0] < 100, (stage, got[stage])


@pytest.mark.parametrize("fill", [0, 0x7f, 0xff])
@pytest.mark.parametrize("D,P,heads,max_q", [(128, 64, 8, 2), (64, 16, 24, 1), (32, 128, 8, 40),
                                             (256, 32, 16, 1)])
@pytest.mark.parametrize("max_len,window", [(2000, 0), (2000, 1500), (1999, 1985), (1130, 1100)])
def test_attention_split_in_one_part(D, P, heads, max_q, max_len, window, fill):
    """Sequences enough that nothing is joined: one part writes the output, zeros
    too where a row sees no key (none there, no page, all before the window), over
    a workspace of exactly the size asked for that holds anything."""
    hk, seqs = 8, 65
    g = rng(D, P, max_len, window, fill)
    c = scattered(g, seqs, -(-max_len // P), hk, P, D)
    c["table"][6] = -1
    # within, at and past max_len, and past it by about the window
    lens = [max_len + window + max_q, max_len + window + max_q - 1, max_len + window, max_len + 1,
            max_len, 1, max_len, 0, 4000, max_len + 63] + [int(x) for x in g.integers(0, 300, seqs - 10)]
    new = [int(x) for x in g.integers(1, min(max_q, 3) + 1, seqs)]
    new[0], new[1], new[2] = max_q, max_q, 1
    T = sum(new)
    cu = np.concatenate([[0], np.cumsum(new)]).astype(np.int32)
    q = g.integers(-127, 128, (T, heads, D)).astype(np.int8)
    qs = g.integers(9000, 21000, (T, heads)).astype(np.int32)
    cache = on_device(c)
    need = ilw.lib().ilw_cache_attention_workspace_bytes(cache.struct, seqs, max_q, max_len, heads,
                                                         window)
    rows = max_q * (heads // hk)
    tiles = seqs * hk * -(-rows // 16)
    seen = min(max_len, window + 16) if window else max_len
    steps = -(-seen // 64) + (seen < max_len)
    say(f"one part D={D} P={P} heads={heads} max_len={max_len} window={window} fill={fill}")
    up = lambda n: -(-n // 256) * 256
    assert need == up(tiles * steps * min(rows, 16) * 128) + up(tiles * 64)  # (no parts' sums)
    buf = torch.full((need + 512,), fill, dtype=torch.uint8, device="cuda")
    out = torch.full((T, heads * D), 77, dtype=torch.int8, device="cuda")
    ilw.ilw_cache_attention(cache, dev(q), dev(qs), dev(cu), dev(np.array(lens, np.int32)),
                            params(D), max_q, max_len, window=window, out=out,
                            workspace=buf[256:256 + need].view(torch.int8))
    want = np.full((T, heads, D), 77, np.int8)
    plain.attention(c, q, qs, cu.tolist(), lens, params(D), max_q, max_len, True, window, want)
    assert not window or not want[0].any()
    same(out.view(T, heads, D), want, "attention")
    assert bool((buf[:256] == fill).all()) and bool((buf[256 + need:] == fill).all())


def test_attention_rows_past_max_len_and_window():
    """The same lengths by the kernel of many rows and by one workgroup a tile."""
    D, P, hk, window = 64, 32, 4, 45
    for seqs, max_q, max_len in [(64, 70, 200), (3, 2, 200)]:
        g = rng(max_q, 7)
        c = scattered(g, seqs, -(-max_len // P), hk, P, D)
        lens = [max_len + window + max_q, max_len + window, max_len + 1] + [int(x) for x in g.integers(
            0, 60, seqs - 3)]
        want = run_attention(c, hk, [max_q, 1] + [1] * (seqs - 2), lens, params(D), True, window,
                             f"past max_len and window, {seqs} sequences", g=g, max_len=max_len)
        assert not want[0].any()


def test_another_page_table():
    """The same pools under a table that is set after a first call: other pages, and
    then another number of sequences."""
    D, P, heads, hk = 64, 16, 4, 2
    g = rng(26)
    c = make_cache(g, 3, 6, hk, P, D)
    cache, first = on_device(c), c["table"]
    rope = rope_of(6 * P, D)
    for table in (first, first[::-1].copy(), first[1:, :5].copy(), first):
        seqs = len(table)
        c["table"] = table
        cache.page_table = dev(table)
        past, new = np.array([20, 0, 40], np.int32)[:seqs], np.array([2, 3, 1], np.int32)[:seqs]
        cu, T = np.concatenate([[0], np.cumsum(new)]).astype(np.int32), int(new.sum())
        qkv = g.integers(-127, 128, (T, (heads + 2 * hk) * D)).astype(np.int8)
        say(f"table of {seqs} sequences")
        q, qs = ilw.ilw_cache_append(cache, dev(qkv), heads, dev(cu), dev(past), 3, rope=dev(rope))
        out = ilw.ilw_cache_attention(cache, q, qs, dev(cu), dev(past + new), params(D), 3, 80)
        want_q, want_s = np.zeros((T, heads, D), np.int8), np.zeros((T, heads), np.int32)
        plain.append(c, qkv, heads, cu.tolist(), past.tolist(), 3, rope, False, want_q, want_s)
        want = np.zeros_like(want_q)
        plain.attention(c, want_q, want_s, cu.tolist(), (past + new).tolist(), params(D), 3, 80, True,
                        0, want)
        same(q, want_q, "q")
        same_cache(cache, c, "cache")
        same(out.view(T, heads, D), want, "attention")


@pytest.mark.parametrize("code", [-128, 127])
@pytest.mark.parametrize("D,P", [(32, 256), (128, 16)])
def test_attention_lowest_codes_of_a_long_prompt(D, P, code):
    """131072 keys of one weight, every value -128 (which appending never writes)
    under a scale whose low digit is -128: 2^31, one more than an int32 sum holds;
    and the lowest sum that there is, of 127."""
    max_len, hk, seqs = 131072, 4, 48
    g = rng(D, code + 128)
    c = scattered(g, seqs, max_len // P, hk, P, D)
    c["v"][:] = code
    c["v_scale"][:] = 72 * 256 + 128
    # (below saturation; a wrong sum of low digits moves it by two codes)
    p = {"score_mult": 0, "score_shift": 40, "out_mult": 107 << 24, "out_shift": 47}
    new = [2] + [1] * (seqs - 1)
    lens = [max_len, 40] + [int(x) for x in g.integers(0, 90, seqs - 2)]
    want = run_attention(c, hk, new, lens, p, False, 0, f"lowest codes D={D} code={code}", g=g,
                         max_q=66)
    assert (want[0] == want[0, 0, 0]).all() and 100 < abs(int(want[0, 0, 0])) < 127


@pytest.mark.parametrize("K", [144, 272, 400])
def test_grouped_largest_tile_with_a_tail(K):
    """256 x 256 tiles whose last step is 16 inputs after whole ones: loads straight
    to LDS, then stores, into the same two buffers."""
    counts, N = [1900, 0, 201], 4224
    assert sum(counts) >= 192 * len(counts) and sum(counts) * N > 128 * 65536
    run_grouped(rng(N, K), counts, N, K, x_rows=300, pad=1)


@pytest.mark.parametrize("counts,N", [([70, 130, 65], 6032), ([3, 0, 9, 16] * 33, 1024),
                                      ([40, 7], 144)])
def test_grouped_other_tiles_with_a_tail(counts, N):
    """The same of the other three tiles."""
    for K in (272, 208):
        run_grouped(rng(N, K), counts, N, K, x_rows=90, pad=1)
