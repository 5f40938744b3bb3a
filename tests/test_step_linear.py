"""Linears with token and channel scales: every kernel that the launch rule chooses from
with rows picked by index, experts that do not take all rows, outputs on a 4-byte border
and factors of every size, the short form of the factor's product on both sides of its
limit.  Every output is compared."""
import numpy as np
import pytest
import torch

import step_plain as plain
from paper_2607_24981_amd import ilw


def say(msg):
    print(f"[gpu] {msg}", flush=True)


def dev(a):
    return ilw.to_device(a)


def rng(*seed):
    return np.random.Generator(np.random.PCG64([v % (1 << 32) for v in seed]))


def bits_of(v):
    """Bit lengths of whole numbers in [0, 2^53)."""
    return np.frexp(v.astype(np.float64))[1].astype(np.int64)


def whole(c, offsets, rows, bits, y):
    """plain.linear_scaled, an expert's rows at a time in 64-bit integers; changes y."""
    x, w = c["x"], c["w"]
    E, N, K = w.shape
    mult, shift = (np.broadcast_to(c[k].reshape(-1) if c[k].size == 1 else c[k].reshape(E, N),
                                   (E, N)).astype(np.int64) for k in ("mult", "shift"))
    lim = 127 if bits == 8 else 32767
    for e in range(E):
        m = np.arange(offsets[e], offsets[e + 1])
        if not m.size:
            continue
        r = m if rows is None else rows[m].astype(np.int64)
        there = (r >= 0) & (r < x.shape[0])
        r = np.where(there, r, 0)
        acc = (x[r].astype(np.float64) @ w[e].T.astype(np.float64)).astype(np.int64)
        acc[~there] = 0
        S = np.where(there, np.maximum(c["x_scale"][r].astype(np.int64), 0), 0)[:, None]
        Y = np.maximum(mult[e], 0)
        z, u = 32 - bits_of(S), 31 - bits_of(Y)
        F = (((S << z).astype(np.uint64) * (Y << u).astype(np.uint64)) >> np.uint64(32)).astype(np.int64)
        q = shift[e] + z + u - 18
        b = 0 if c["b"] is None else c["b"][e].astype(np.int64).clip(-(1 << 24), 1 << 24)
        v = (((acc * F) >> (q - 4).clip(0, 63)) + b + 8) >> 4
        y[m] = v.clip(-lim, lim)


def case(g, E, N, K, R, bits, bias=True):
    """Ordinary numbers: outputs of a few octaves that mostly fit."""
    shift = 30 + int(round(np.log2(42 * 73 * np.sqrt(K) / (40 if bits == 8 else 192))))
    return {"x": np.clip(np.rint(g.normal(0, 42, (R, K))), -128, 127).astype(np.int8),
            "x_scale": np.exp2(g.uniform(11, 17, R)).astype(np.int32),
            "w": g.integers(-127, 128, (E, N, K)).astype(np.int8),
            "mult": g.integers(1 << 28, 1 << 30, (E, N)).astype(np.int32),
            "shift": g.integers(shift - 1, shift + 2, (E, N)).astype(np.int32),
            "b": g.integers(-900, 900, (E, N)).astype(np.int32) if bias else None}


def run(c, M, offsets, rows, bits, what, lead=0):
    """offsets None: one expert with every row.  lead: values before y in its memory."""
    say(what)
    N = c["w"].shape[1]
    dt = torch.int8 if bits == 8 else torch.int16
    buf = torch.full((M * N + lead + 8,), 77, dtype=dt, device="cuda")
    y = buf[lead:lead + M * N].view(M, N)

    def to(v):
        return None if v is None else dev(v[0] if offsets is None and v.shape != (1,) else v)
    ilw.ilw_linear_scaled(dev(c["x"]), dev(c["x_scale"]), to(c["w"]), to(c["b"]), to(c["mult"]),
                          to(c["shift"]),
                          offsets=None if offsets is None else dev(np.asarray(offsets, np.int32)),
                          rows=None if rows is None else dev(rows), bits=bits, y=y)
    torch.cuda.synchronize()
    want = np.full((M, N), 77, np.int8 if bits == 8 else np.int16)
    whole(c, [0, M] if offsets is None else offsets, rows, bits, want)
    got = y.cpu().numpy()
    bad = np.argwhere(got != want)
    assert not bad.size, (what, len(bad), bad[:4], [(got[m, n], want[m, n]) for m, n in bad[:4]])
    assert (buf[:lead] == 77).all() and (buf[lead + M * N:] == 77).all(), what


def test_whole_is_the_plain_form():
    for seed, bits in ((1, 8), (2, 16)):
        g = rng(seed)
        c = case(g, 3, 32, 48, 20, bits)
        c["x_scale"][:5] = [0, -7, 1, 2 ** 31 - 1, 1 << 30]
        c["mult"][0, :6] = [0, -3, 1, 2 ** 31 - 1, 1 << 30, 77]
        c["shift"][:, ::3] = g.integers(1, 63, (3, 11))
        c["b"][1, :4] = [2 ** 31 - 1, -2 ** 31, 1 << 24, -(1 << 24)]
        rows = g.integers(-2, 22, 30).astype(np.int32)
        got, want = (np.full((30, 32), 77, np.int8 if bits == 8 else np.int16) for _ in range(2))
        whole(c, [2, 9, 9, 27], rows, bits, got)
        plain.linear_scaled(c["x"], c["x_scale"], c["w"], c["b"], c["mult"], c["shift"],
                            [2, 9, 9, 27], rows, bits, want)
        assert np.array_equal(got, want)


# Rows, experts, N and K by the kernel that the launch rule takes for them: channels x
# rows of a workgroup's tile.  Each with whole steps of 128 inputs and with a partial last
# one, from one step to more than the ring holds.
SIZES = {
    "stream 16 x 16": [(30, 1, 496, 2064), (21, 3, 96, 2304)],
    "stream 32 x 16": [(16, 1, 4000, 336), (200, 40, 112, 512), (40, 2, 2000, 640)],
    "stream 64 x 16": [(9, 1, 65552, 128), (900, 300, 272, 144), (3000, 1024, 48, 64)],
    "stream 32 x 32": [(30, 1, 4400, 272), (30, 1, 4400, 512)],
    "stream 64 x 32": [(24, 1, 16400, 384), (180, 9, 3600, 80)],
    "stream 64 x 64, four waves": [(240, 6, 2576, 384), (150, 4, 3600, 144)],
    "stream 64 x 64, two waves": [(1800, 40, 1616, 128), (1800, 40, 1616, 144)],
    "tile 128 x 64": [(1400, 20, 1040, 128), (1400, 20, 1040, 528), (66560, 1024, 16, 64)],
    "tile 128 x 128, three steps ahead": [(1024, 1, 2064, 528), (1100, 4, 2064, 640),
                                          (1100, 4, 2064, 1040), (1024, 1, 2064, 384),
                                          (1100, 4, 2064, 112), (1024, 1, 2064, 128)],
    "tile 128 x 128": [(4096, 5, 1040, 144), (4096, 1, 1040, 256)],
    "tile 256 x 256": [(520, 2, 16784, 80), (300, 1, 30000, 256)],
}
ALL = [(k, *s) for k, sizes in SIZES.items() for s in sizes]
TILES = [(k, *s) for k, sizes in SIZES.items() if k.startswith("tile") for s in sizes]


def cuts(g, M, E, first, last):
    """Offsets of E experts over the rows first .. M - last - 1, some of them without rows."""
    return [first] + [int(v) for v in np.sort(g.integers(first, M - last + 1, E - 1))] + [M - last]


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("kernel,M,E,N,K", ALL)
@pytest.mark.parametrize("bits", [8, 16])
def test_picked_rows(kernel, M, E, N, K, bits):
    """Rows by index, some that point nowhere; rows before the first and behind the last
    expert stay; y on a 4-byte border."""
    g = rng(1, M, E, N, K, bits)
    R = max(3, min(M // 2, 5000))
    c = case(g, E, N, K, R, bits)
    rows = g.integers(0, R, M).astype(np.int32)
    for v in (-1, R, 2 ** 31 - 1, -2 ** 31):
        rows[g.random(M) < 0.04] = v
    first, last = (3, 5) if M > 16 else (1, 2)
    what = f"{kernel}: {M} rows {E} experts {N} x {K} bits={bits}"
    run(c, M, cuts(g, M, E, first, last), rows, bits, what + ", picked", lead=2 if bits == 16 else 4)
    if E == 1:
        run(c, M, None, rows, bits, what + ", picked, dense")


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("kernel,M,E,N,K", ALL)
@pytest.mark.parametrize("bits", [8, 16])
def test_rows_in_place(kernel, M, E, N, K, bits):
    """Without an index, on both output borders."""
    g = rng(2, M, E, N, K, bits)
    c = case(g, E, N, K, M, bits, bias=(M + N) % 32 == 0)
    first, last = (2, 9) if M > 16 else (0, 1)
    what = f"{kernel}: {M} rows {E} experts {N} x {K} bits={bits}, in place"
    run(c, M, cuts(g, M, E, first, last), None, bits, what)
    if E == 1:
        run(c, M, None, None, bits, what + ", dense", lead=2 if bits == 16 else 4)


def every_size(g, c):
    """Scales, multipliers and shifts of every size, none at all, biases past their limit,
    sums of the largest products."""
    R, (E, N, K) = c["x"].shape[0], c["w"].shape
    c["x"][::7], c["w"][:, ::5] = -128, -128
    c["x"][3::7] = 127
    c["x_scale"] = np.exp2(g.uniform(0, 31, R)).astype(np.int64).clip(1, 2 ** 31 - 1).astype(np.int32)
    c["x_scale"][::11], c["x_scale"][1::29], c["x_scale"][2::31] = 0, -5, 2 ** 31 - 1
    c["mult"] = np.exp2(g.uniform(0, 31, (E, N))).astype(np.int64).clip(0, 2 ** 31 - 1).astype(np.int32)
    c["mult"][:, ::13], c["mult"][:, 1::17], c["mult"][:, 2::19] = 0, -3, 2 ** 31 - 1
    c["shift"] = g.integers(1, 63, (E, N)).astype(np.int32)
    c["b"] = g.integers(-(1 << 20), 1 << 20, (E, N)).astype(np.int32)
    c["b"][:, :4] = [2 ** 31 - 1, -2 ** 31, 1 << 24, -(1 << 24)]


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("kernel,M,E,N,K", ALL)
@pytest.mark.parametrize("bits", [8, 16])
def test_factors(kernel, M, E, N, K, bits):
    """First with factors that no workgroup has the short form for, then with such that
    every one has (spare_bits leaves 4 or more at these K): shifts of 40 to 62, scales below
    2^22, multipliers from 2^20 on or none."""
    g = rng(3, M, E, N, K, bits)
    c = case(g, E, N, K, M, bits)
    every_size(g, c)
    offsets = cuts(g, M, E, 0, 0)
    what = f"{kernel}: {M} rows {E} experts {N} x {K} bits={bits}"
    run(c, M, offsets, None, bits, what + ", factors of every size")
    c["shift"] = g.integers(40, 63, (E, N)).astype(np.int32)
    some = c["mult"] > 0
    c["mult"][some] = g.integers(1 << 20, 1 << 31, int(some.sum()))
    some = c["x_scale"] > 0
    c["x_scale"][some] = g.integers(1, 1 << 22, int(some.sum()))
    run(c, M, offsets, None, bits, what + ", long shifts")


@pytest.mark.gpu
@pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")
@pytest.mark.parametrize("kernel,M,E,N,K", TILES)
@pytest.mark.parametrize("bits", [8, 16])
def test_short_form_limit(kernel, M, E, N, K, bits):
    """The short form shifts the high word of (acc 2^e) F right by q - 36 + e, e the bits
    that a sum of K products leaves free: with scales of 1 (z = 17) and multipliers of 2^30
    (u = 0), q - 36 + e = shift - 37 + e.  All factors one below, at and one above 0; then
    one channel, one token or both far below, the others above.  Sums from -9 to 9 and the
    largest ones of both signs."""
    g = rng(4, M, E, N, K, bits)
    e = 17 - K.bit_length()
    c = {"x": np.zeros((M, K), np.int8), "w": g.integers(-1, 2, (E, N, K)).astype(np.int8),
         "x_scale": np.full(M, 1 << 14, np.int32), "mult": np.full((E, N), 1 << 30, np.int32),
         "b": g.integers(-20, 20, (E, N)).astype(np.int32)}
    for i in range(3):
        c["x"][np.arange(M), g.integers(0, K, M)] = g.integers(-3, 4, M)
    c["x"][::50], c["x"][1::50] = 127, -128
    c["w"][:, ::40], c["w"][:, 1::40] = -128, 127
    offsets = cuts(g, M, E, 0, 0)
    what = f"{kernel}: {M} rows {E} experts {N} x {K} bits={bits}"
    for above in (-1, 0, 1):
        c["shift"] = np.full((E, N), 37 - e + above, np.int32)
        run(c, M, offsets, None, bits, what + f", {above} above")
    c["shift"] = np.full((E, N), 37 - e + 3, np.int32)
    few, lows = dict(c), dict(c)
    few["shift"] = c["shift"].copy()
    few["shift"][:, N // 2 + 1] = 20
    run(few, M, offsets, None, bits, what + ", one channel below")
    lows["x_scale"] = c["x_scale"].copy()
    lows["x_scale"][M // 2 + 1] = 1 << 24
    run(lows, M, offsets, None, bits, what + ", one token below")
    few["x_scale"] = lows["x_scale"]
    run(few, M, offsets, None, bits, what + ", one of each below")
