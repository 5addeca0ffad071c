"""float64 oracle of the operators around the expert layer: block norms with gate and residual, the router's balance loss,
low-rank adapters.  Plain numpy from the formulas; test infrastructure only.

Every function returns its results and, under the same names, magnitudes: the same sums with every term's absolute value, which
is what an evaluation in fewer bits may be off by, times a number of roundings (a sum of terms that cancel keeps the rounding
errors of its terms)."""
import numpy as np


def sigmoid(z):
    return 1.0 / (1.0 + np.exp(-z))


def _rms(v, eps):
    return 1.0 / np.sqrt((v * v).mean(axis=1, keepdims=True) + eps)


def _gate(gate, use_sigmoid):
    if gate is None:
        return None
    a = sigmoid(gate) if use_sigmoid else gate
    return a[:, None] if a.ndim == 1 else a


def block_norm(h, y, gate, w_pre, w_post, eps, rho, beta, use_sigmoid):
    out, mag = {}, {}
    if y is None:
        new, m = h, np.abs(h)
    else:
        u = y if w_post is None else y * _rms(y, eps) * w_post
        a = _gate(gate, use_sigmoid)
        branch = beta * (u if a is None else a * u)
        new, m = rho * h + branch, np.abs(rho * h) + np.abs(branch)
        out["h"], mag["h"] = new, m
    if w_pre is not None:
        r = _rms(new, eps)
        out["x"], mag["x"] = new * r * w_pre, m * r * np.abs(w_pre)
    return out, mag


def block_norm_grad(h, y, gate, dh, dx, w_pre, w_post, eps, rho, beta, use_sigmoid):
    out, mag = {}, {}
    d = np.zeros_like(h) if dh is None else dh
    md = np.abs(d)
    if dx is not None:
        r = _rms(h, eps)
        n, dn = h * r, dx * w_pre
        d = d + r * (dn - n * (dn * n).mean(axis=1, keepdims=True))
        md = md + r * (np.abs(dn) + np.abs(n) * np.abs(dn * n).mean(axis=1, keepdims=True))
        out["dw_pre"], mag["dw_pre"] = (dx * n).sum(axis=0), np.abs(dx * n).sum(axis=0)
    if y is None:
        out["dh"], mag["dh"] = d, md
        return out, mag
    out["dh"], mag["dh"] = rho * d, abs(rho) * md
    e, me = beta * d, abs(beta) * md
    q = _rms(y, eps) if w_post is not None else np.ones((h.shape[0], 1))
    m = y * q
    u = m if w_post is None else m * w_post
    a = _gate(gate, use_sigmoid)
    if a is not None:
        da, mda = e * u, me * np.abs(u)
        if gate.ndim == 1:
            da, mda = da.sum(axis=1, keepdims=True), mda.sum(axis=1, keepdims=True)
        slope = a * _gate(-gate, True) if use_sigmoid else 1.0    # (s(-z) = 1 - s(z), without the difference)
        da, mda = da * slope, mda * slope
        out["dgate"] = da[:, 0] if gate.ndim == 1 else da
        mag["dgate"] = mda[:, 0] if gate.ndim == 1 else mda
        e, me = e * a, me * np.abs(a)
    if w_post is not None:
        out["dw_post"], mag["dw_post"] = (e * m).sum(axis=0), (me * np.abs(m)).sum(axis=0)
        dm, mdm = e * w_post, me * np.abs(w_post)
        e = q * (dm - m * (dm * m).mean(axis=1, keepdims=True))
        me = q * (mdm + np.abs(m) * (mdm * np.abs(m)).mean(axis=1, keepdims=True))
    out["dy"], mag["dy"] = e, me
    return out, mag


def softmax_rows(z):
    """Rows without a value above -inf have no probabilities: zeros."""
    m = z.max(axis=1, keepdims=True)
    dead = np.isneginf(m)
    p = np.exp(z - np.where(dead, 0.0, m))
    s = p.sum(axis=1, keepdims=True)
    return np.where(dead, 0.0, p / np.where(s == 0, 1.0, s))


def members(T, offsets, mask):
    """The tokens of every sequence that count."""
    offsets = [0, T] if offsets is None else [int(o) for o in offsets]
    return [np.array([t for t in range(a, b) if mask is None or mask[t]], dtype=np.int64)
            for a, b in zip(offsets, offsets[1:])]


def balance_loss(z, ids, alpha, offsets=None, mask=None):
    T, E = z.shape
    k = ids.shape[1]
    seqs = members(T, offsets, mask)
    counts = np.zeros((len(seqs), E), dtype=np.int64)
    probs = np.zeros((len(seqs), E))
    total = 0.0
    for s, at in enumerate(seqs):
        if len(at) == 0:
            continue
        probs[s] = softmax_rows(z[at]).mean(axis=0)
        got = ids[at].reshape(-1)
        counts[s] = np.bincount(got[(got >= 0) & (got < E)], minlength=E)
        total += E * (counts[s] / (k * len(at)) * probs[s]).sum()
    used = sum(len(at) > 0 for at in seqs)
    return {"loss": alpha * total / max(1, used), "counts": counts, "probs": probs,
            "tokens": np.array([len(at) for at in seqs] + [used])}


def balance_loss_grad(z, ids, alpha, dloss=1.0, offsets=None, mask=None):
    T, E = z.shape
    k = ids.shape[1]
    fwd = balance_loss(z, ids, alpha, offsets, mask)
    used = max(1, int(fwd["tokens"][-1]))
    out, mag = np.zeros((T, E)), np.zeros((T, E))
    for s, at in enumerate(members(T, offsets, mask)):
        if len(at) == 0:
            continue
        p = softmax_rows(z[at])
        f = fwd["counts"][s] / (k * len(at))
        dot = (p * f).sum(axis=1, keepdims=True)
        w = dloss * alpha * E / (used * len(at))
        out[at] = w * p * (f - dot)
        mag[at] = abs(w) * p * (f + dot)
    return out, mag


def adapter_apply(X, ids, A, B, scale=None, ranks=None, base=None):
    n, R, _ = A.shape
    out = np.zeros((X.shape[0], B.shape[1])) if base is None else base.copy()
    mag_low = np.zeros_like(out)
    for t, a in enumerate(ids):
        if not 0 <= a < n:
            continue
        r = R if ranks is None else int(min(max(ranks[a], 0), R))
        s = 1.0 if scale is None else float(scale[a])
        low = A[a, :r] @ X[t]
        out[t] += s * (B[a, :, :r] @ low)
        mag_low[t] = abs(s) * (np.abs(B[a, :, :r]) @ (np.abs(A[a, :r]) @ np.abs(X[t])))
    return out, mag_low
