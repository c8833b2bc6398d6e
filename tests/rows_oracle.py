"""The sorted-row operators and the 4-bit matrices in plain NumPy, 64 bits: what the tests compare
with. Nothing here uses the library."""
import numpy as np


def sort_tokens(idx, E):
    """(offsets [E + 1], rows [R], pos [R]) of idx [T, k]."""
    pairs = [(int(e) if 0 <= e < E else E, i) for i, e in enumerate(np.asarray(idx).reshape(-1))]
    order = sorted(pairs)
    R = len(pairs)
    rows, pos = np.full(R, -1, np.int32), np.zeros(R, np.int32)
    for r, (e, i) in enumerate(order):
        rows[r] = i if e < E else -1
        pos[i] = r if e < E else -1 - r
    counts = np.bincount([e for e, _ in pairs], minlength=E + 1)
    offsets = np.concatenate([[0], np.cumsum(counts[:E])]).astype(np.int32)
    return offsets, rows, pos


def gather(x, pos, k):
    out = np.zeros((len(pos), x.shape[1]))
    for i, p in enumerate(pos):
        if p >= 0:
            out[p] = x[i // k]
    return out


def combine(ys, pos, gates, add, T):
    """(y, sum of the magnitudes of its terms)."""
    k = len(pos) // T
    y = np.zeros((T, ys.shape[1])) if add is None else add.astype(np.float64).copy()
    mag = np.abs(y)
    for i, p in enumerate(pos):
        if p >= 0:
            w = 1.0 if gates is None else float(gates.reshape(-1)[i])
            y[i // k] += w * ys[p]
            mag[i // k] += np.abs(w * ys[p])
    return y, mag


def combine_backward(dy, ys, pos, gates):
    """(dys, dgates [R], sum of the magnitudes of dgates' terms)."""
    T, R = dy.shape[0], len(pos)
    k = R // T
    dys, dg, mag = np.zeros((R, dy.shape[1])), np.zeros(R), np.zeros(R)
    for i, p in enumerate(pos):
        if p >= 0:
            w = 1.0 if gates is None else float(gates.reshape(-1)[i])
            dys[p] = w * dy[i // k]
            if ys is not None:
                dg[i] = float(np.dot(dy[i // k], ys[p]))
                mag[i] = float(np.dot(np.abs(dy[i // k]), np.abs(ys[p])))
    return dys, dg, mag


def five_bits(a):
    """a >= 0 rounded to five significant bits, ties to even."""
    m, e = np.frexp(a)
    return np.ldexp(np.rint(np.ldexp(m, 5)), e - 5)


def q4_values(w, group):
    """(codes, scales, values) of weights [..., K]."""
    w = np.asarray(w, np.float64)
    v = w.reshape(*w.shape[:-1], w.shape[-1] // group, group)
    top = np.abs(v).max(-1)
    fin = np.isfinite(v).all(-1) & (top < 2.0 ** 120)
    with np.errstate(all="ignore"):
        s = np.where(fin, np.where(top < 2.0 ** -100, 0.0, five_bits(np.where(fin, top, 0) / 7)), np.nan)
        c = np.where((s > 0)[..., None], np.rint(v / s[..., None]), 0.0)
    return c.reshape(w.shape), s, (c * s[..., None]).reshape(w.shape)


def q4_products(x, src, offsets, experts, values):
    """y [R, N] and the sum of the magnitudes of its terms; src [R] rows of x (-1: zeros)."""
    R, N = len(src), values.shape[1]
    y, mag = np.zeros((R, N)), np.zeros((R, N))
    xs = np.where((src >= 0)[:, None], x[np.maximum(src, 0)], 0.0)
    for u, e in enumerate(experts):
        lo, hi = offsets[u], offsets[u + 1]
        if lo < hi:
            y[lo:hi] = xs[lo:hi] @ values[e].T
            mag[lo:hi] = np.abs(xs[lo:hi]) @ np.abs(values[e]).T
    return y, mag
