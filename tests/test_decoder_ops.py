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
