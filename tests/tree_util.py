"""Speculative decoding in plain float64 (numpy), and batches for its tests."""
import numpy as np

BLOCK = 16


def rotate(x, pos, rot, theta, style, inv_freq=None):
    """x [n][heads][D] float64 turned at positions pos [n] (rot: rotated width)."""
    om = np.asarray(inv_freq) if inv_freq is not None else float(theta) ** (-2.0 * np.arange(rot // 2) / rot)
    ang = np.asarray(pos, np.float64)[:, None] * om
    c, s = np.cos(ang)[:, None, :], np.sin(ang)[:, None, :]
    y = x.copy()
    a, b = (x[..., :rot // 2], x[..., rot // 2:rot]) if style == 0 else (x[..., 0:rot:2], x[..., 1:rot:2])
    u, v = a * c - b * s, b * c + a * s
    if style == 0:
        y[..., :rot // 2], y[..., rot // 2:rot] = u, v
    else:
        y[..., 0:rot:2], y[..., 1:rot:2] = u, v
    return y


def ancestors(parents):
    """Bool [n][n] (row i: i and its ancestors) and depths; a parent outside [0, i) makes a root."""
    n = len(parents)
    see, depth = np.eye(n, dtype=bool), np.zeros(n, np.int32)
    for i, p in enumerate(parents):
        if 0 <= p < i:
            see[i] |= see[p]
            depth[i] = depth[p] + 1
    return see, depth


def pack(see, words):
    """Visibility rows as int64 words."""
    n, m = see.shape
    bits = np.zeros((n, words * 64), np.uint8)
    bits[:, :m] = see
    return np.ascontiguousarray(np.packbits(bits, axis=1, bitorder="little")).view(np.int64).reshape(n, words)


def random_parents(rng, n):
    return np.array([-1] + [int(rng.integers(-1 if rng.random() < 0.1 else 0, i)) for i in range(1, n)], np.int32)[:n]


def attention(q, k, v, see, scale):
    """q [n][Hq][D], k / v [keys][Hkv][D] float64 (turned), see [n][keys]: outputs, and per output the
    mean distance sum_j p_j |v_j - o| that a relative error of the probabilities multiplies."""
    n, hq, d = q.shape
    g = hq // k.shape[1]
    o, spread = np.zeros((n, hq, d)), np.zeros((n, hq, d))
    for h in range(hq):
        with np.errstate(invalid="ignore"):
            s = (q[:, h] @ k[:, h // g].T) * scale
        s = np.where(see, s, -np.inf)
        for t in range(n):
            if not see[t].any():
                continue
            p = np.exp(s[t, see[t]] - s[t, see[t]].max())
            p /= p.sum()
            vv = v[see[t], h // g]
            o[t, h] = p @ vv
            spread[t, h] = p @ np.abs(vv - o[t, h])
    return o, spread
