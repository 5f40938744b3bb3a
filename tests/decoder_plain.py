"""Plain 64-bit forms of the paged cache's operators and the grouped linear, in
numpy, one sequence, head and row after another."""
import numpy as np


def value_place(P, D):
    """[P, D]: the byte of (token, channel) in a page and head of the values."""
    j, c = np.arange(P).reshape(-1, 1), np.arange(D).reshape(1, -1)
    G = min(P, 64)
    t = j % G
    return ((j // G) * G * D + (c // 16) * 16 * G + ((t % 16) // 4) * 4 * G + (c % 16) * (G // 4)
            + (t // 16) * 4 + t % 4)


def codes(value, scale):
    return (2 * value + scale) // (2 * scale)


def need(value):
    return max(1, -(-int(np.abs(value).max()) // 127))


def rotate(x, pos, rope, interleaved):
    """x int64 [heads, D] -> Q14 values."""
    out = x << 14
    if rope is None:
        return out
    R = 2 * rope.shape[1]
    c, s = (rope[pos, :, i].astype(np.int64) for i in (0, 1))
    i1 = np.arange(0, R, 2) if interleaved else np.arange(R // 2)
    i2 = i1 + 1 if interleaved else i1 + R // 2
    x1, x2 = x[:, i1], x[:, i2]
    out[:, i1], out[:, i2] = x1 * c - x2 * s, x2 * c + x1 * s
    return out


def append(cache, qkv, heads, cu, past, max_new, rope, interleaved, q, q_scale):
    """cache: dict of arrays k, v, k_scale, v_scale, table; changes it, q and
    q_scale in place."""
    n_pages, hk, P, D = cache["k"].shape
    table = cache["table"]
    place = value_place(P, D)
    for s in range(len(past)):
        n = min(cu[s + 1] - cu[s], max_new)
        pages = {}
        for i in range(n):
            t, pos = cu[s] + i, past[s] + i
            x = qkv[t].astype(np.int64).reshape(heads + 2 * hk, D)
            rot = rotate(x[:heads + hk], min(pos, table.shape[1] * P - 1), rope, interleaved)
            for h in range(heads):
                S = need(rot[h])
                q[t, h], q_scale[t, h] = codes(rot[h], S), S
            if pos < table.shape[1] * P and 0 <= table[s, pos // P] < n_pages:
                pages.setdefault(pos // P, []).append((pos % P, rot[heads:], x[heads + hk:] << 14))
        for block, rows in pages.items():
            page, first = table[s, block], rows[0][0]
            for h in range(hk):
                for part in (1, 2):
                    scales = cache["k_scale" if part == 1 else "v_scale"]
                    flat = cache["k" if part == 1 else "v"][page, h].reshape(-1)
                    at = place if part == 2 else np.arange(P * D).reshape(P, D)
                    S = need(np.stack([r[part][h] for r in rows]))
                    if first > 0:
                        old = int(scales[page, h])
                        S = old if S <= old else max(S, old + old // 8)
                        flat[at[:first]] = codes(flat[at[:first]].astype(np.int64) * old, S)
                    for r in rows:
                        flat[at[r[0]]] = codes(r[part][h], S)
                    scales[page, h] = S


def attention(cache, q, q_scale, cu, lens, p, max_q, max_len, causal, window, out):
    """Writes the rows of out [T, heads, D] that the operator writes."""
    n_pages, hk, P, D = cache["k"].shape
    table = cache["table"]
    heads = q.shape[1]
    place = value_place(P, D)
    far = 17 * 64
    a = np.arange(far + 1)
    n = -(-a // 64)
    chord = np.array([int((64 + 64 * n[i] - a[i]) << 16) >> int(n[i] + 6) for i in a])
    t = p["score_shift"] - 16
    for s in range(len(lens)):
        nq, L = cu[s + 1] - cu[s], min(int(lens[s]), max_len)
        j = np.arange(L)
        page = table[s, j // P]
        there = (page >= 0) & (page < n_pages)
        page = np.where(there, page, 0)
        for h in range(heads):
            g = h // (heads // hk)
            k = cache["k"][page, g, j % P].astype(np.int64)
            v = cache["v"][:, g].reshape(n_pages, -1)[page[:, None], place[j % P]].astype(np.int64)
            sk, sv = (cache[x][page, g].astype(np.int64) for x in ("k_scale", "v_scale"))
            for i in range(min(nq, max_q)):
                row = cu[s] + i
                end = int(lens[s]) - nq + 1 + i if causal else L
                see = there & (j < end)
                if window:
                    see &= j >= end - window
                if not see.any():
                    out[row, h] = 0
                    continue
                A = (int(q_scale[row, h]) * p["score_mult"] + (1 << (t - 1))) >> t
                m = (A * sk + (1 << 15)) >> 16
                x = ((k @ q[row, h].astype(np.int64)) * m + (1 << 27)) >> 28
                x = np.clip(x, -32767, 32767)
                w = np.where(see, chord[np.clip(x[see].max() - x, 0, far)], 0)
                pv = (w * sv + (1 << 15)) >> 16
                total = int(w.sum())
                d = total.bit_length() - 16
                F = (2 ** 31 - 1) // (total >> d)
                for c, T in enumerate((pv @ v).tolist()):
                    r = (T * F) >> (d + 13)
                    y = (r * p["out_mult"] + (1 << (p["out_shift"] - 1))) >> p["out_shift"]
                    out[row, h, c] = min(max(y, -127), 127)


def grouped(x, rows, offsets, w, b, mult, shift, y):
    E, N, K = w.shape
    for e in range(E):
        for m in range(offsets[e], offsets[e + 1]):
            r = m if rows is None else int(rows[m])
            xr = x[r].astype(np.int64) if 0 <= r < len(x) else np.zeros(K, np.int64)
            acc = w[e].astype(np.int64) @ xr + (0 if b is None else b[e].astype(np.int64))
            mu, sh = ((mult[0], shift[0]) if mult.size == 1 else (mult[e], shift[e]))
            half = acc * np.int64(mu) + (np.int64(1) << (np.asarray(sh, np.int64) - 1))
            y[m] = np.clip(half >> np.asarray(sh, np.int64), -127, 127)
