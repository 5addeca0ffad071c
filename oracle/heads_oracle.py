"""Float64 definitions of what lies between a block's Q/K/V projection and its output projection: heads with norm and rotation, the
paged cache, attention of single tokens over it.  Plain loops over tokens, heads and positions; test infrastructure only."""
import numpy as np


def turn_matrix(D, freq, interleaved, rot_scale, position):
    """The rotation of one row as a D x D matrix."""
    M = np.eye(D)
    h = len(freq)
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        t = np.longdouble(position) * np.longdouble(freq[i])   # (the product of far positions needs more than 53 bits)
        c, s = rot_scale * np.cos(t), rot_scale * np.sin(t)
        M[a, a], M[a, b], M[b, a], M[b, b] = c, -s, s, c
    return M


def pair_matrix(D, freq, interleaved, rot_scale):
    """What a row's rounding errors are counted against: |a| + |b| for both values of a pair.  (|M| alone would not do: an angle that is off
    by d moves n_b c + n_a s by d (n_a c - n_b s), which may be large where |n_b c| + |n_a s| is small.)"""
    M = np.eye(D)
    h = len(freq)
    for i in range(h):
        a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + h)
        M[a, a] = M[a, b] = M[b, a] = M[b, b] = abs(rot_scale)
    return M


def head_norm(x, w, eps, freq, interleaved, rot_scale, positions):
    """x [T, n, D] -> results, and the magnitudes that rounding errors go by (sum of |terms|)."""
    T, n, D = x.shape
    v = x if w is None else x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * w
    out = np.empty_like(v)
    for t in range(T):
        out[t] = v[t] @ turn_matrix(D, freq, interleaved, rot_scale, positions[t]).T
    return out, np.abs(v) @ pair_matrix(D, freq, interleaved, rot_scale)


def head_norm_grad(x, w, dy, eps, freq, interleaved, rot_scale, positions):
    """dx, dw and the magnitudes of both."""
    T, n, D = dy.shape
    g, gs = np.empty_like(dy), np.abs(dy) @ pair_matrix(D, freq, interleaved, rot_scale)
    for t in range(T):
        g[t] = dy[t] @ turn_matrix(D, freq, interleaved, rot_scale, positions[t])
    if w is None:
        return g, None, gs, None
    r = 1 / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    dw, dws = (g * x * r).sum((0, 1)), (gs * np.abs(x) * r).sum((0, 1))
    gw, gws = g * w, gs * np.abs(w)
    dx = r * (gw - x * r * r * (gw * x).mean(-1, keepdims=True))
    return dx, dw, r * (gws + np.abs(x) * r * r * (gws * np.abs(x)).mean(-1, keepdims=True)), dws


def slots(table, lengths, offsets, page_size, pages, T):
    """(sequence, position, page or None, slot) of every token; None for tokens outside all sequences or outside the table."""
    out = [None] * T
    for s, n in enumerate(lengths):
        a, b = (s, s + 1) if offsets is None else (offsets[s], offsets[s + 1])
        for t in range(a, b):
            p = n - (b - t)
            if p < 0 or p // page_size >= len(table[s]):
                continue
            page = table[s][p // page_size]
            out[t] = (s, p, int(page) if 0 <= page < pages else None, p % page_size)
    return out


def attention(q, k, v, table, lengths, scale, window=0, softcap=0.0, sinks=None):
    """q [S, Hq, D]; k, v [pages, page_size, heads, D] (values, scales applied).  Returns out, lse, and by row the sum of p |v|
    [S, Hq, D], the largest sum of scale |q| |k| and the largest |z|."""
    S, Hq, D = q.shape
    pages, size, Hk, _ = k.shape
    G = Hq // Hk
    out, lse, mag = np.zeros((S, Hq, D)), np.full((S, Hq), -np.inf), np.zeros((S, Hq, D))
    dot, top = np.zeros((S, Hq)), np.zeros((S, Hq))
    for s in range(S):
        n = max(0, min(int(lengths[s]), len(table[s]) * size))
        first = max(0, n - window) if window else 0
        at = [(table[s][p // size], p % size) for p in range(first, n)]
        at = [(a, b) for a, b in at if 0 <= a < pages]
        rows = np.array(at, dtype=np.int64).reshape(-1, 2)
        for h in range(Hq):
            K, V = k[rows[:, 0], rows[:, 1], h // G], v[rows[:, 0], rows[:, 1], h // G]
            z = scale * (K @ q[s, h])
            if len(z):
                dot[s, h] = (abs(scale) * (np.abs(K) @ np.abs(q[s, h]))).max()
            if softcap:
                z = softcap * np.tanh(z / softcap)
            every = z if sinks is None else np.append(z, sinks[h])
            m = every.max() if len(every) else -np.inf
            if m == -np.inf:
                continue
            total = np.exp(every - m).sum()
            p = np.exp(z - m) / total
            if len(z):
                top[s, h] = np.abs(z[np.isfinite(z)]).max() if np.isfinite(z).any() else 0
            out[s, h], mag[s, h], lse[s, h] = p @ V, p @ np.abs(V), m + np.log(total)
    return out, lse, mag, dot, top
