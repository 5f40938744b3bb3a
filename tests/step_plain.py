"""Plain forms of the operators behind a decoder step's attention, in numpy's 64-bit
integers and Python's unlimited ones, one row after another."""
import math

import numpy as np

NONE, LOWEST = -32768, -(1 << 31)
EXP2 = [1 << 30] + [math.floor(2.0 ** (30.0 - f / 64.0) + 0.5) for f in range(1, 64)]


def exp2(a):
    """2^(30 - a/64)."""
    return EXP2[a % 64] >> (a // 64)


def inverse(d):
    return ((1 << 62) - 1) // d


def quantize_rows(x):
    x = x.astype(np.int64)
    y, scale = np.zeros(x.shape, np.int8), np.zeros(x.shape[0], np.int32)
    for m, row in enumerate(x):
        S = max(1, -(-(int(np.abs(row).max()) << 14) // 127))
        y[m], scale[m] = ((row << 15) + S) // (2 * S), S
    return y, scale


def linear_scaled(x, x_scale, w, b, mult, shift, offsets, rows, bits, y):
    """w [E, N, K]; changes y, rows outside [offsets[0], offsets[E]) stay."""
    E, N, K = w.shape
    mult, shift = (np.broadcast_to(v.reshape(-1) if v.size == 1 else v.reshape(E, N), (E, N)).tolist()
                   for v in (mult, shift))
    lim = 127 if bits == 8 else 32767
    for e in range(E):
        for m in range(offsets[e], offsets[e + 1]):
            r = m if rows is None else int(rows[m])
            there = 0 <= r < x.shape[0]
            acc = w[e].astype(np.int64) @ (x[r].astype(np.int64) if there else np.zeros(K, np.int64))
            S = max(0, int(x_scale[r])) if there else 0
            z = 32 - S.bit_length()
            for n, a in enumerate(acc.tolist()):
                Y = max(0, mult[e][n])
                u = 31 - Y.bit_length()
                F = ((S << z) * (Y << u)) >> 32
                q = shift[e][n] + z + u - 18
                c = 0 if b is None else max(-(1 << 24), min(1 << 24, int(b[e][n])))
                v = (((a * F) >> max(q - 4, 0)) + c + 8) >> 4
                y[m, n] = max(-lim, min(lim, v))


def probabilities(s, sigmoid):
    live = [v != NONE for v in s]
    if sigmoid:
        return [((exp2(-v) if v < 0 else 1 << 30) * inverse((1 << 30) + exp2(abs(v)))) >> 32 if ok else 0
                for v, ok in zip(s, live)]
    if not any(live):
        return [0] * len(s)
    top = max(s)
    w = [exp2(top - v) if ok else 0 for v, ok in zip(s, live)]
    L = sum(w)
    d = L.bit_length() - 31
    return [(v * inverse(L >> d)) >> (32 + d) for v in w]


def route(logits, top_k, bias, sigmoid, renormalize, groups, top_groups, group_best, mult, shift):
    T, E = logits.shape
    expert, weight = np.full((T, top_k), -1, np.int32), np.zeros((T, top_k), np.int32)
    per = E // groups
    for t in range(T):
        s = [int(v) for v in logits[t]]
        p = probabilities(s, sigmoid)
        c = [v + (0 if bias is None else max(-(1 << 30), min(1 << 30, int(bias[e]))))
             for e, v in enumerate(p)]
        free = [e for e in range(E) if s[e] != NONE]
        if groups > 1:
            score = {}
            for g in range(groups):
                best = sorted((c[e] for e in free if e // per == g), reverse=True)
                if best:
                    score[g] = sum(best[:group_best])
            kept = sorted(score, key=lambda g: (-score[g], g))[:top_groups]
            free = [e for e in free if e // per in kept]
        chosen = sorted(free, key=lambda e: (-c[e], e))[:top_k]
        W = sum(p[e] for e in chosen)
        for j, e in enumerate(chosen):
            r = p[e]
            if renormalize:
                n = W.bit_length()
                unit = W << (31 - n) if n <= 31 else W >> (n - 31)
                r = (p[e] * inverse(unit)) >> (n + 1) if W else 0
            expert[t, j] = e
            weight[t, j] = min((r * mult + (1 << (shift - 1))) >> shift, (1 << 31) - 1)
    return (expert, weight) + sort(expert, E)


def sort(expert, E):
    """offsets, rows and slot of the choices."""
    T, top_k = expert.shape
    pairs = sorted((int(expert[t, j]), t, j) for t in range(T) for j in range(top_k)
                   if expert[t, j] >= 0)
    rows, slot = np.full(T * top_k, -1, np.int32), np.full((T, top_k), -1, np.int32)
    counts = np.zeros(E + 1, np.int64)
    for i, (e, t, j) in enumerate(pairs):
        rows[i], slot[t, j] = t, i
        counts[e + 1] += 1
    return np.cumsum(counts).astype(np.int32), rows, slot


def combine(v, slot, weight, mult_a, shift, skip, mult_b):
    T, N = slot.shape[0], v.shape[1]
    lim, most = np.iinfo(v.dtype).max, (1 << 31) - 1
    y = np.zeros((T, N), v.dtype)
    for t in range(T):
        total = np.zeros(N, np.int64)
        for j, s in enumerate(slot[t]):
            if 0 <= s < v.shape[0]:
                total += int(weight[t, j]) * v[s].astype(np.int64)
        u = np.clip((total + 128) >> 8, -most, most) * mult_a + (1 << (shift - 1))
        if skip is not None:
            u += skip[t].astype(np.int64) * mult_b
        y[t] = np.clip(u >> shift, -lim, lim)
    return y


def log2_q16(L):
    n = L.bit_length()
    y, out = L >> (n - 31), n - 31
    for _ in range(16):
        y = y * y >> 30
        out = 2 * out + (y >= 1 << 31)
        y >>= y >= 1 << 31
    return out


def log_probs(logits, given, n_top):
    rows, V = logits.shape
    out = (np.full(given.shape, LOWEST, np.int64), np.zeros(rows, np.int64),
           np.full((rows, n_top), -1, np.int64), np.full((rows, n_top), LOWEST, np.int64))
    for r in range(rows):
        s = logits[r].astype(np.int64)
        free = np.flatnonzero(s != NONE)
        if not free.size:
            continue
        top = int(s[free].max())
        a = top - s[free]
        w = np.array(EXP2, np.int64)[a % 64] >> np.minimum(a // 64, 40)
        L, B = int(w.sum()), int((w * a).sum())
        lg = log2_q16(L)
        out[1][r] = lg + 1024 * B // L
        for i, v in enumerate(given[r]):
            if 0 <= v < V and s[v] != NONE:
                out[0][r, i] = 1024 * (int(s[v]) - top) - lg
        best = free[np.argsort(a, kind="stable")[:n_top]]
        out[2][r, :best.size] = best
        out[3][r, :best.size] = 1024 * (s[best] - top) - lg
    return tuple(v.astype(np.int32) for v in out)
