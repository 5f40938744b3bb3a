"""Rows quantized with a scale each, linears with token and channel scales, routing
to experts, their rows combined and log probabilities against plain forms.  Every
operation is integer: results are equal or wrong."""
import numpy as np
import pytest
import torch

import step_plain as plain
from paper_2607_24981_amd import ilw

pytestmark = [pytest.mark.gpu,
              pytest.mark.skipif(not torch.cuda.is_available(), reason="needs a GPU")]
NONE = plain.NONE


def say(msg):
    print(f"[gpu] {msg}", flush=True)


def dev(a):
    return ilw.to_device(a)


def same(got, want, what):
    got = got.cpu().numpy() if isinstance(got, torch.Tensor) else got
    assert got.shape == want.shape and got.dtype == want.dtype, (what, got.shape, want.shape)
    bad = np.flatnonzero(got.reshape(-1) != want.reshape(-1))
    assert not bad.size, (what, got.shape, bad.size, bad[:5], got.reshape(-1)[bad[:5]],
                          want.reshape(-1)[bad[:5]])


def rng(*seed):
    return np.random.Generator(np.random.PCG64(seed))


def strided(a, pad, lead=0):
    """The matrix on the device, its rows `pad` values further apart, `lead` values
    into its memory."""
    wide = torch.full((a.shape[0] * (a.shape[1] + pad) + lead,), 77,
                      dtype=torch.from_numpy(a[:0]).dtype, device="cuda")
    out = wide[lead:].view(a.shape[0], a.shape[1] + pad)[:, :a.shape[1]]
    out.copy_(dev(a))
    return out


# ------------------------------------------------------------------ quantize
@pytest.mark.parametrize("M,K", [(1, 16), (5, 48), (70, 64), (33, 256), (17, 272), (9, 1024),
                                 (1030, 1040), (1100, 4096), (3, 4096), (6, 4112), (2, 16384),
                                 (3, 16400), (2, 40000)])
@pytest.mark.parametrize("pad", [0, 24])
def test_quantize(M, K, pad):
    say(f"quantize M={M} K={K} pad={pad}")
    g = rng(M, K)
    x = np.rint(g.normal(0, 1, (M, K)) * np.exp2(g.uniform(0, 13, (M, 1))))
    x = x.clip(-32768, 32767).astype(np.int16)
    x[0] = 0
    if M > 2:
        x[1], x[2] = 0, -5
        x[1, K - 1] = -32768
    y, scale = ilw.ilw_quantize_rows(strided(x, pad) if pad else dev(x))
    torch.cuda.synchronize()
    want = plain.quantize_rows(x)
    same(scale, want[1], "scale")
    same(y, want[0], "y")


@pytest.mark.parametrize("K", [16, 144, 560, 2336])
def test_quantize_many_rows(K):
    """Where three units a lane are in use: rows of 1, 9, 35 and 146 units."""
    M = (1 << 24) // K + 5
    say(f"quantize M={M} K={K}")
    fewer = (np.arange(M) % 16).astype(np.int16)[:, None]
    x = rng(K).integers(-32768, 32768, (M, K), dtype=np.int16) >> fewer
    y, scale = ilw.ilw_quantize_rows(dev(x))
    torch.cuda.synchronize()
    some = np.r_[0:500, M // 2:M // 2 + 200, M - 500:M]
    want = plain.quantize_rows(x[some])
    same(scale[some], want[1], "scale")
    same(y[some], want[0], "y")
    most = np.abs(x.astype(np.int32)).max(1).astype(np.int64)
    same(scale, np.maximum(1, -(-(most << 14) // 127)).astype(np.int32), "every scale")


@pytest.mark.parametrize("M", [4, 700])
@pytest.mark.parametrize("K", [112, 144, 528, 2032, 2064])
def test_quantize_borders(M, K):
    """Rows around what 4, 16 and 64 lanes hold in two units each."""
    say(f"quantize M={M} K={K}")
    fewer = (np.arange(M) % 16).astype(np.int16)[:, None]
    x = rng(M, K).integers(-32768, 32768, (M, K), dtype=np.int16) >> fewer
    y, scale = ilw.ilw_quantize_rows(dev(x))
    torch.cuda.synchronize()
    want = plain.quantize_rows(x)
    same(scale, want[1], "scale")
    same(y, want[0], "y")


def test_quantize_every_magnitude():
    """Every largest magnitude there is, with the values whose codes are nearest to a
    tie, both signs."""
    A = np.arange(1, 32769, dtype=np.int64)
    S = -(-(A << 14) // 127)
    half = (2 * np.arange(16) + 1) * 8 - 7  # odd multiples of half a code, up to 127
    near = (half[None, :] * S[:, None]) // (2 << 14)
    x = np.concatenate([near, near + 1, -near, -near - 1], 1)
    x = np.clip(x, -A[:, None], np.minimum(A, 32767)[:, None])
    x[:, 0] = -A
    x = x.astype(np.int16)
    say("quantize every magnitude")
    y, scale = ilw.ilw_quantize_rows(dev(x))
    want = plain.quantize_rows(x)
    same(scale, want[1], "scale")
    same(y, want[0], "y")


# -------------------------------------------------------------------- linear
def linear_case(g, M, N, K, E, R, bits, per_tensor, bias, spread=3.0):
    c = {"x": np.clip(np.rint(g.normal(0, 42, (R, K))), -128, 127).astype(np.int8),
         "x_scale": np.exp2(g.uniform(14 - spread, 14 + spread, R)).astype(np.int32),
         "w": g.integers(-127, 128, (E, N, K)).astype(np.int8)}
    shift = 30 + int(round(np.log2(42 * 73 * np.sqrt(K) / (40 if bits == 8 else 192))))
    size = (1,) if per_tensor else (E, N)
    c["mult"] = g.integers(1 << 28, 1 << 30, size).astype(np.int32)
    c["shift"] = g.integers(shift - 1, shift + 2, size).astype(np.int32)
    c["b"] = g.integers(-900, 900, (E, N)).astype(np.int32) if bias else None
    return c


def run_linear(c, M, bits, offsets, rows, what, dense=False, y_lead=0):
    say(f"linear {what}")
    E, N, K = c["w"].shape
    dt = torch.int8 if bits == 8 else torch.int16
    buf = torch.full((M * N + y_lead,), 77, dtype=dt, device="cuda")
    y = buf[y_lead:].view(M, N)
    want = np.full((M, N), 77, np.int8 if bits == 8 else np.int16)

    def lead(v):
        return None if v is None else dev(v[0] if dense and v.shape != (1,) else v)
    ilw.ilw_linear_scaled(dev(c["x"]), dev(c["x_scale"]), lead(c["w"]), lead(c["b"]),
                          lead(c["mult"]), lead(c["shift"]),
                          offsets=None if dense else dev(np.asarray(offsets, np.int32)),
                          rows=None if rows is None else dev(rows), bits=bits, y=y)
    torch.cuda.synchronize()
    plain.linear_scaled(c["x"], c["x_scale"], c["w"], c["b"], c["mult"], c["shift"],
                        [0, M] if dense else offsets, rows, bits, want)
    same(y, want, what)


@pytest.mark.parametrize("M", [1, 2, 15, 16, 17, 33, 70, 130])
@pytest.mark.parametrize("N,K", [(16, 16), (48, 64), (144, 112), (272, 336), (16, 1040)])
@pytest.mark.parametrize("bits", [8, 16])
def test_linear_dense(M, N, K, bits):
    g = rng(M, N, K, bits)
    c = linear_case(g, M, N, K, 1, M, bits, (M + N) % 3 == 0, (M + K) % 2 == 0)
    run_linear(c, M, bits, None, None, f"M={M} N={N} K={K} bits={bits}", dense=True)


@pytest.mark.parametrize("counts", [[3], [0, 5, 0, 1, 0, 17], [16, 15, 33], [64, 65, 1, 0, 130],
                                    [0, 0, 0]])
@pytest.mark.parametrize("N,K", [(16, 64), (80, 144)])
@pytest.mark.parametrize("bits", [8, 16])
def test_linear_grouped(counts, N, K, bits):
    """Rows before the first and behind the last expert stay; an index that points
    nowhere is a row of zeros."""
    g = rng(sum(counts), N, K, bits)
    first, E = 3, len(counts)
    offsets = [first + int(v) for v in np.concatenate([[0], np.cumsum(counts)])]
    M = offsets[-1] + 5
    R = max(4, M // 2)
    c = linear_case(g, M, N, K, E, R, bits, False, True)
    rows = g.integers(0, R, M).astype(np.int32)
    rows[g.random(M) < 0.1] = -1
    rows[g.random(M) < 0.1] = R
    run_linear(c, M, bits, offsets, rows, f"counts={counts} N={N} K={K} bits={bits} rows")
    c = linear_case(g, M, N, K, E, M, bits, True, False)
    run_linear(c, M, bits, offsets, None, f"counts={counts} N={N} K={K} bits={bits}")


# every kernel that the launch rule chooses from, in its order: rows an expert, experts, N, K
TILES = [(20, 1, 272, 2064), (7, 3, 96, 2304), (16, 1, 4000, 336), (5, 40, 112, 512),
         (9, 1, 65552, 128), (3, 300, 272, 144), (30, 1, 4400, 272), (30, 1, 16400, 640),
         (20, 9, 3600, 80), (60, 1, 16400, 144), (40, 6, 2576, 384), (50, 1, 65552, 80),
         (45, 40, 1616, 128), (200, 1, 48000, 64), (260, 2, 16784, 80), (70, 1, 24592, 64),
         (66, 3, 12304, 272), (70, 20, 1040, 128), (90, 17, 976, 48)]


@pytest.mark.parametrize("K", [16, 112, 128, 144, 256, 272, 384, 400, 512, 528, 640, 1040])
@pytest.mark.parametrize("M,N,E", [(1024, 2064, 1), (1100, 2064, 9), (4096, 1040, 1)])
def test_linear_steps(M, N, E, K):
    """1 to 9 steps, whole ones and partial last ones, of tiles that load three steps
    ahead and (the last sizes) one."""
    g = rng(M, N, K)
    c = linear_case(g, M, N, K, E, M, 8, False, True)
    offsets = [0, M] if E == 1 else np.r_[0, np.sort(g.integers(0, M, E - 1)), M]
    run_linear(c, M, 8, offsets, None, f"M={M} N={N} E={E} K={K}", dense=E == 1)


@pytest.mark.parametrize("per,E,N,K", TILES)
@pytest.mark.parametrize("bits", [8, 16])
def test_linear_tiles(per, E, N, K, bits):
    g = rng(per, E, N, K, bits)
    M = per * E
    cuts = np.sort(g.integers(0, M + 1, E - 1)) if E > 1 else np.zeros(0, int)
    offsets = [0] + [int(v) for v in cuts] + [M]
    c = linear_case(g, M, N, K, E, M, bits, False, True)
    say(f"tiles per={per} E={E} N={N} K={K} bits={bits}")
    y = ilw.ilw_linear_scaled(*[dev(c[k]) for k in ("x", "x_scale", "w", "b", "mult", "shift")],
                              offsets=dev(np.asarray(offsets, np.int32)), bits=bits)
    torch.cuda.synchronize()
    # every row of a sample of channels, the first and last ones among them
    cols = np.unique(np.concatenate([g.integers(0, N, 24), [0, 1, 15, 16, N - 17, N - 16, N - 1]]))
    want = np.zeros((M, cols.size), np.int8 if bits == 8 else np.int16)
    plain.linear_scaled(c["x"], c["x_scale"], c["w"][:, cols], c["b"][:, cols], c["mult"][:, cols],
                        c["shift"][:, cols], offsets, None, bits, want)
    same(y[:, dev(cols)], want, "sample")


@pytest.mark.parametrize("bits", [8, 16])
def test_linear_factors(bits):
    """Scales and multipliers of every size, none at all, shifts from 1 to 62, large and
    limited biases, sums of the largest products."""
    g = rng(7, bits)
    M, N, K = 96, 256, 64
    c = linear_case(g, M, N, K, 1, M, bits, False, True)
    c["x"][:8], c["w"][0, :16] = -128, -128
    c["x"][8:16] = 127
    c["x_scale"] = np.exp2(g.uniform(0, 31, M)).astype(np.int64).clip(1, 2 ** 31 - 1).astype(np.int32)
    c["x_scale"][:6] = [1, 2 ** 31 - 1, 0, -5, 1 << 30, 3]
    c["mult"][0] = np.exp2(g.uniform(0, 31, N)).astype(np.int64).clip(0, 2 ** 31 - 1)
    c["mult"][0, :5] = [0, 1, 2 ** 31 - 1, -3, 1 << 30]
    c["shift"][0] = g.integers(1, 63, N)
    c["b"][0] = g.integers(-(1 << 20), 1 << 20, N)
    c["b"][0, :4] = [2 ** 31 - 1, -2 ** 31, 1 << 24, -(1 << 24)]
    run_linear(c, M, bits, None, None, f"factors bits={bits}", dense=True)
    c["shift"][0] = g.integers(40, 63, N)  # every workgroup on the short form
    c["mult"][0] = g.integers(1 << 20, 1 << 31, N)
    c["x_scale"] = g.integers(1, 1 << 22, M).astype(np.int32)
    run_linear(c, M, bits, None, None, f"factors, long shifts, bits={bits}", dense=True)


def test_linear_unaligned_output():
    """y on a 4-byte border."""
    g = rng(9)
    for bits, lead in ((8, 4), (16, 2)):
        c = linear_case(g, 20, 48, 64, 1, 20, bits, False, True)
        run_linear(c, 20, bits, None, None, f"unaligned bits={bits}", dense=True, y_lead=lead)


def test_linear_far_rows():
    """Weights and rows past 2^31 bytes."""
    g = rng(10)
    E, N, K, R = 3, 16384, 65536, 40000
    w = torch.randint(-127, 128, (E, N, K), dtype=torch.int8, device="cuda")
    x = torch.randint(-127, 128, (R, K), dtype=torch.int8, device="cuda")
    x_scale = torch.randint(1 << 13, 1 << 15, (R,), dtype=torch.int32, device="cuda")
    rows = dev(np.array([R - 1, 5, R - 2, 33000], np.int32))
    offsets = [0, 1, 1, 4]
    mult, shift = (torch.full((1,), v, dtype=torch.int32, device="cuda") for v in (1 << 30, 46))
    say("linear far rows")
    y = ilw.ilw_linear_scaled(x, x_scale, w, None, mult, shift, rows=rows,
                              offsets=dev(np.asarray(offsets, np.int32)))
    torch.cuda.synchronize()
    cols = [0, 7, N - 1]
    at = rows.long()
    want = np.zeros((4, 3), np.int16)
    plain.linear_scaled(x[at].cpu().numpy(), x_scale[at].cpu().numpy(), w[:, cols].cpu().numpy(),
                        None, np.array([1 << 30]), np.array([46]), offsets, None, 16, want)
    same(y[:, cols], want, "far rows")


@pytest.mark.parametrize("K", [65536, 65552])
def test_linear_far_channels(K):
    """One matrix past 2^32 bytes."""
    g = rng(11, K)
    N = 66000
    w = torch.randint(-127, 128, (N, K), dtype=torch.int8, device="cuda")
    x = dev(g.integers(-127, 128, (3, K)).astype(np.int8))
    x_scale = dev(np.array([1 << 14, 9000, 30000], np.int32))
    mult, shift = (torch.full((1,), v, dtype=torch.int32, device="cuda") for v in (1 << 30, 46))
    say(f"linear far channels K={K}")
    y = ilw.ilw_linear_scaled(x, x_scale, w, None, mult, shift)
    torch.cuda.synchronize()
    cols = [0, 1, 63, 64, 40000, 65535, 65536, N - 17, N - 1]
    want = np.zeros((3, len(cols)), np.int16)
    plain.linear_scaled(x.cpu().numpy(), x_scale.cpu().numpy(), w[cols].cpu().numpy()[None], None,
                        np.array([1 << 30]), np.array([46]), [0, 3], None, 16, want)
    same(y[:, cols], want, "far channels")


# --------------------------------------------------------------------- route
def run_route(logits, top_k, what, bias=None, sigmoid=False, renormalize=True, groups=1,
              top_groups=1, group_best=2, mult=1 << 30, shift=44, pad=0):
    say(f"route {what}")
    x = strided(logits, pad, 1) if pad else dev(logits)
    r = ilw.ilw_route(x, top_k, bias=None if bias is None else dev(bias), sigmoid=sigmoid,
                      renormalize=renormalize, groups=groups, top_groups=top_groups,
                      group_best=group_best, weight_mult=mult, weight_shift=shift)
    torch.cuda.synchronize()
    want = plain.route(logits, top_k, bias, sigmoid, renormalize, groups, top_groups, group_best,
                       mult, shift)
    for name, got, w in zip(r._fields, r, (want[0], want[1], want[2], want[3], want[4])):
        same(got, w, f"{what}: {name}")
    return want


def scores(g, T, E, sigma=130, ties=False):
    x = np.rint(g.normal(0, sigma, (T, E))).clip(-32767, 32767)
    if ties:
        x = np.rint(x / sigma) * 64
    return x.astype(np.int16)


@pytest.mark.parametrize("T", [1, 2, 63, 64, 65, 130, 257])
@pytest.mark.parametrize("E,top_k", [(1, 1), (3, 2), (64, 4), (65, 8), (100, 32), (256, 8),
                                     (300, 6), (1000, 3), (1024, 16)])
def test_route(T, E, top_k):
    g = rng(T, E)
    sigmoid = (T + E) % 2 == 0
    bias = g.integers(-(1 << 28), 1 << 28, E).astype(np.int32) if T % 2 else None
    run_route(scores(g, T, E, ties=T % 3 == 0), top_k, f"T={T} E={E} top_k={top_k}", bias=bias,
              sigmoid=sigmoid, renormalize=T % 4 != 1, pad=3 * (E % 2))


@pytest.mark.parametrize("E,groups,top_groups,top_k", [
    (64, 8, 4, 6), (256, 8, 4, 8), (64, 64, 10, 10), (96, 3, 1, 32), (512, 16, 2, 5),
    (1024, 64, 64, 32), (6, 2, 2, 6), (15, 5, 3, 3), (1008, 9, 4, 8)])
@pytest.mark.parametrize("best", [1, 2])
def test_route_groups(E, groups, top_groups, top_k, best):
    g = rng(E, groups, best)
    for T, sigmoid in ((70, True), (9, False)):
        x = scores(g, T, E, ties=best == 1)
        x[g.random((T, E)) < 0.2] = NONE
        bias = g.integers(-(1 << 29), 1 << 29, E).astype(np.int32)
        run_route(x, top_k, f"E={E} groups={groups}/{top_groups} best={best} T={T}", bias=bias,
                  sigmoid=sigmoid, groups=groups, top_groups=top_groups, group_best=best)


@pytest.mark.parametrize("sigmoid", [False, True])
def test_route_ends(sigmoid):
    """Tokens without any expert, with fewer than top_k, flat and steep rows, the lowest
    and highest scores, probabilities that are all 0, biases past their limits, weights
    past 32 bits."""
    E, top_k = 40, 5
    g = rng(3, sigmoid)
    x = scores(g, 90, E)
    x[0] = NONE
    x[1] = NONE
    x[1, [7, 30]] = [5, 5]
    x[2], x[3], x[4], x[5] = 0, 32767, -32767, -32767
    x[5, 11] = 32767
    x[6] = np.where(np.arange(E) % 2, 32767, -32767)
    x[7], x[7, 3] = NONE, -32767
    x[8] = -3000
    x[9] = -1984 + np.arange(E)
    x[20:70] = NONE
    bias = np.full(E, -2 ** 31, np.int32)
    bias[::3] = 2 ** 31 - 1
    bias[1::6] = 7
    for b in (None, bias):
        for renorm in (False, True):
            run_route(x, top_k, f"ends {sigmoid} {b is None} {renorm}", bias=b, sigmoid=sigmoid,
                      renormalize=renorm)
    run_route(x, top_k, "weights past 32 bits", sigmoid=sigmoid, mult=2 ** 31 - 1, shift=1)
    run_route(x, top_k, "no weights", sigmoid=sigmoid, mult=0, shift=62)
    run_route(x[20:60], top_k, "no choice at all", sigmoid=sigmoid)


def test_route_no_tokens():
    say("route no tokens")
    r = ilw.ilw_route(torch.zeros(0, 12, dtype=torch.int16, device="cuda"), 3)
    assert r.offsets.tolist() == [0] * 13 and r.rows.numel() == 0 and r.slot.shape == (0, 3)


@pytest.mark.parametrize("T,E,top_k", [(5000, 64, 4), (20000, 128, 8), (70000, 16, 2)])
def test_route_many_tokens(T, E, top_k):
    """The sorting of many workgroups' choices, against a stable sort."""
    g = rng(T)
    x = scores(g, T, E)
    x[g.random(T) < 0.05] = NONE
    say(f"route many T={T}")
    r = ilw.ilw_route(dev(x), top_k)
    torch.cuda.synchronize()
    expert = r.expert.cpu().numpy()
    few = g.integers(0, T, 200)
    same(expert[few], plain.route(x[few], top_k, None, False, True, 1, 1, 2, 1 << 30, 44)[0], "sample")
    flat = expert.reshape(-1)
    order = np.argsort(np.where(flat < 0, E, flat), kind="stable")
    n = int((flat >= 0).sum())
    rows, slot = np.full(flat.size, -1, np.int32), np.full(flat.size, -1, np.int32)
    rows[:n], slot[order[:n]] = order[:n] // top_k, np.arange(n)
    offsets = np.concatenate([[0], np.cumsum(np.bincount(flat[flat >= 0], minlength=E))])
    same(r.offsets, offsets.astype(np.int32), "offsets")
    same(r.rows, rows, "rows")
    same(r.slot, slot.reshape(T, top_k), "slot")


# ------------------------------------------------------------------- combine
@pytest.mark.parametrize("T,top_k,N", [(1, 1, 16), (3, 2, 48), (64, 4, 512), (7, 8, 1040),
                                       (5, 32, 2064), (130, 3, 1024)])
@pytest.mark.parametrize("dtype", [np.int8, np.int16])
@pytest.mark.parametrize("with_skip", [False, True])
def test_combine(T, top_k, N, dtype, with_skip):
    say(f"combine T={T} top_k={top_k} N={N} {dtype.__name__} skip={with_skip}")
    g = rng(T, top_k, N, with_skip)
    lim = np.iinfo(dtype).max
    R = T * top_k
    v = np.rint(g.normal(0, lim / 3, (R, N))).clip(-lim - 1, lim).astype(dtype)
    slot = g.permutation(R).reshape(T, top_k).astype(np.int32)
    slot[g.random((T, top_k)) < 0.1] = -1
    slot[g.random((T, top_k)) < 0.1] = R
    if T > 2:
        slot[1], slot[2, 0] = -1, -2 ** 31
    weight = g.integers(-3000, (1 << 17) // top_k, (T, top_k)).astype(np.int32)
    skip = g.integers(-lim - 1, lim + 1, (T, N)).astype(dtype) if with_skip else None
    for ma, mb, shift in ((1 << 22, 1 << 30, 30), (-123456, -(1 << 27), 28), (1 << 30, 3, 38)):
        want = plain.combine(v, slot, weight, ma, shift, skip, mb)
        y = ilw.ilw_combine(dev(v), dev(slot), dev(weight), ma, shift,
                            skip=None if skip is None else dev(skip), skip_mult=mb)
        torch.cuda.synchronize()
        same(y, want, f"{ma} {mb} {shift}")
    if with_skip:  # in place
        y = dev(skip)
        ilw.ilw_combine(dev(v), dev(slot), dev(weight), 1 << 22, 30, skip=y, skip_mult=1 << 30, y=y)
        torch.cuda.synchronize()
        same(y, plain.combine(v, slot, weight, 1 << 22, 30, skip, 1 << 30), "in place")


@pytest.mark.parametrize("dtype", [np.int8, np.int16])
def test_combine_extremes(dtype):
    """The largest weights and values, sums past 32 bits, shifts of 1 and 62; no rows."""
    say(f"combine extremes {dtype.__name__}")
    lim = np.iinfo(dtype).max
    T, top_k, N = 6, 32, 64
    v = np.full((T * top_k, N), -lim - 1, dtype)
    v[::3] = lim
    slot = np.arange(T * top_k, dtype=np.int32).reshape(T, top_k)
    weight = np.full((T, top_k), 2 ** 31 - 1, np.int32)
    weight[1], weight[2], weight[3, ::2], weight[4], weight[5] = -2 ** 31, 1, -2 ** 31, 0, 1 << 16
    skip = np.full((T, N), -lim - 1, dtype)
    most = 2 ** 31 - 1
    for ma, mb, shift in ((most, most, 62), (-most, most, 62), (most, -most, 1), (1, 1, 1), (0, 0, 40)):
        y = ilw.ilw_combine(dev(v), dev(slot), dev(weight), ma, shift, skip=dev(skip), skip_mult=mb)
        torch.cuda.synchronize()
        same(y, plain.combine(v, slot, weight, ma, shift, skip, mb), f"{ma} {mb} {shift}")
    # around the weights up to which a sum is held in fewer bits
    v[:] = -lim - 1
    weight[:] = np.array([[-(1 << 18)], [-(1 << 18) - 1], [1 << 18], [(1 << 18) - 1], [-(1 << 19)],
                          [1 << 19]])
    for pick in (slice(None), slice(0, 1), slice(1, 2), slice(3, 4), slice(4, 5)):
        y = ilw.ilw_combine(dev(v), dev(slot[pick]), dev(weight[pick]), 1 << 10, 30)
        torch.cuda.synchronize()
        same(y, plain.combine(v, slot[pick], weight[pick], 1 << 10, 30, None, 0), f"{pick}")
    none = torch.empty(0, N, dtype=dev(v).dtype, device="cuda")
    y = ilw.ilw_combine(none, dev(slot), dev(weight), 1, 1, skip=dev(skip), skip_mult=2)
    same(y, plain.combine(v[:0], slot, weight, 1, 1, skip, 2), "no rows")


@pytest.mark.parametrize("N", [16, 48, 1040, 1024, 8192 + 16])
@pytest.mark.parametrize("dtype", [np.int8, np.int16])
def test_combine_widths(dtype, N):
    """Rows that end inside a wave; one, three and five choices; one and many tokens."""
    say(f"combine N={N} {dtype.__name__}")
    g = rng(N)
    lim = np.iinfo(dtype).max
    for T, top_k in ((1, 1), (7, 3), (131, 5)):
        v = g.integers(-lim - 1, lim + 1, (T * top_k, N)).astype(dtype)
        slot = g.integers(-2, T * top_k + 2, (T, top_k)).astype(np.int32)  # (a row twice, and none)
        weight = g.integers(-(1 << 18), 1 << 18, (T, top_k)).astype(np.int32)
        y = torch.full((T + 1, N), 55, dtype=dev(v).dtype, device="cuda")
        ilw.ilw_combine(dev(v), dev(slot), dev(weight), 1 << 20, 30, y=y[:T])
        torch.cuda.synchronize()
        same(y[:T], plain.combine(v, slot, weight, 1 << 20, 30, None, 0), f"{T} {top_k}")
        assert (y[T] == 55).all()


def test_combine_far_rows():
    """Rows past 2^31 bytes."""
    say("combine far rows")
    R, N = 300000, 8192
    v = torch.randint(-128, 128, (R, N), dtype=torch.int8, device="cuda")
    slot = dev(np.array([[R - 1, 0], [R - 7, 299000]], np.int32))
    weight = dev(np.array([[40000, 20000], [7, 65536]], np.int32))
    y = ilw.ilw_combine(v, slot, weight, 1 << 22, 30)
    few = v[slot.long().view(-1)].cpu().numpy()
    same(y, plain.combine(few, np.arange(4).reshape(2, 2), weight.cpu().numpy(), 1 << 22, 30, None, 0),
         "far rows")


# ----------------------------------------------------------------- log probs
def run_log_probs(logits, given, n_top, what, pad=0, lead=0):
    say(f"log probs {what}")
    x = strided(logits, pad, lead) if pad or lead else dev(logits)
    r = ilw.ilw_log_probs(x, None if given is None else dev(given), top=n_top)
    torch.cuda.synchronize()
    if given is None:
        given = np.zeros((logits.shape[0], 0), np.int32)
    want = plain.log_probs(logits, given, n_top)
    for name, got, w in zip(r._fields, r, want):
        same(got, w, f"{what}: {name}")
    return want


VOCABS = [1, 2, 7, 8, 9, 63, 64, 100, 500, 512, 520, 2032, 2048, 2060, 5000, 8176, 8190, 16368, 16384,
          32000, 32752, 32770, 50001, 65520, 65536, 70001, 114672, 114673, 131040, 131072, 200003]


@pytest.mark.parametrize("V", VOCABS)
def test_log_probs(V):
    """Around the borders of what a lane, a wave and a workgroup keep; rows that start
    anywhere; n_top from none to 64, past the vocabulary too."""
    g = rng(V)
    for rows, n_top, n_given, pad, lead in ((1, 0, 1, 0, 0), (3, 1, 0, 1, 0), (2, 20, 3, 5, 3),
                                            (5, 64, 64, 0, 1)):
        x = np.rint(g.normal(0, 192, (rows, V))).astype(np.int16)
        x[g.random((rows, V)) < 0.02] = NONE
        given = g.integers(-1, V + 1, (rows, n_given)).astype(np.int32)
        run_log_probs(x, given, n_top, f"V={V} rows={rows} n_top={n_top} pad={pad} lead={lead}",
                      pad, lead)


@pytest.mark.parametrize("V", [60, 1500, 9000, 30000, 120000, 300000])
@pytest.mark.parametrize("n_top", [1, 7, 64])
def test_log_probs_ties(V, n_top):
    """Flat rows and rows of few values: the best are the first ones; more ties than a
    list holds, in one place and everywhere; rows with none and with one."""
    g = rng(V, n_top)
    x = np.zeros((11, V), np.int16)
    x[1] = -32767
    x[2] = 32767
    x[3] = NONE
    x[4], x[4, V // 2] = NONE, -32767
    x[5] = g.integers(0, 3, V)
    x[6, V - V // 3:] = 900                       # the best ones side by side
    x[7] = np.arange(V) // (V // 50 + 1) * 10     # rising: the last chunk is the best
    x[8] = NONE
    x[8, ::max(1, V // 40)] = -5                  # a few, equal
    x[9] = g.integers(-32767, 32768, V)
    x[10] = -32767
    x[10, ::2] = NONE                             # -32768 next to what can be had
    given = np.stack([np.zeros(11), np.full(11, V - 1), np.full(11, V // 2)], 1).astype(np.int32)
    run_log_probs(x, given, n_top, f"ties V={V} n_top={n_top}")


def test_log_probs_long():
    """The longest vocabulary, a flat row of it: the largest sums."""
    V = 1 << 20
    g = rng(1)
    x = np.rint(g.normal(0, 192, (2, V))).astype(np.int16)
    x[1] = 100
    want = run_log_probs(x, np.array([[5], [V - 1]], np.int32), 64, "V=2^20")
    assert want[1][1] == 20 << 16 and want[0][1, 0] == -(20 << 16)


def test_log_probs_many_rows():
    g = rng(2)
    for rows, V in ((3000, 40), (700, 3000), (1030, 16368), (300, 20000), (257, 32752), (257, 57330)):
        x = np.rint(g.normal(0, 192, (rows, V))).astype(np.int16)
        run_log_probs(x, g.integers(0, V, (rows, 2)).astype(np.int32), 5, f"rows={rows} V={V}")


def test_log_probs_are_log_probabilities():
    """Against the softmax in floating point.  Weights are rounded down by less than
    2^-30 of the largest: 5000 of them change log2 L by less than 1.45 * 5000 * 2^-30 =
    2^-17, and the mean of a/64 < 31 by less than 31 * 5000 * 2^-30 < 2^-12.7.  The
    squarings round down by 2^-30 each and the fraction ends at 2^-16; so does the mean."""
    g = rng(4)
    x = np.rint(g.normal(0, 192, (4, 5000))).astype(np.int16)
    given = g.integers(0, 5000, (4, 8)).astype(np.int32)
    r = ilw.ilw_log_probs(dev(x), dev(given), top=3)
    s = x.astype(np.float64) / 64
    lp = s - np.log2(np.exp2(s - s.max(1, keepdims=True)).sum(1, keepdims=True)) - s.max(1, keepdims=True)
    p = np.exp2(lp)
    assert np.abs(r.given.cpu().numpy() / 65536 - np.take_along_axis(lp, given, 1)).max() < 2 ** -15
    assert np.abs(r.entropy.cpu().numpy() / 65536 + (p * lp).sum(1)).max() < 2 ** -12
