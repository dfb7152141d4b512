"""The cache held in 8 bits in plain float64 (numpy): codes, scales, the store, norms."""
import numpy as np

BLOCK = 16
E4M3, INT8 = 0, 1
MOST = {E4M3: 448.0, INT8: 127.0}
EXPONENTS = {E4M3: (-126, 119), INT8: (-126, 121)}


def _e4m3_values():
    """The numbers of the codes 0 .. 126 (sign bit clear)."""
    out = []
    for c in range(127):
        e, m = c >> 3, c & 7
        out.append(m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10))
    return np.array(out)


E4M3_VALUES = _e4m3_values()


def encode(x, code):
    """Bytes (uint8) of numbers in units of the scale: to nearest, ties to even, saturating; NaN 0."""
    x = np.where(np.isnan(x), 0.0, np.asarray(x, np.float64))
    x = np.clip(x, -MOST[code], MOST[code])
    if code == INT8:
        return np.rint(x).astype(np.int8).view(np.uint8)
    a = np.abs(x)
    hi = np.searchsorted(E4M3_VALUES, a)                 # first code with a number >= a
    lo = np.maximum(hi - 1, 0)
    up, down = E4M3_VALUES[hi] - a, a - E4M3_VALUES[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    c = np.where(a == E4M3_VALUES[hi], hi, c)
    return (c | np.where(np.signbit(x), 0x80, 0)).astype(np.uint8)


def decode(b, code):
    b = np.asarray(b, np.uint8)
    if code == INT8:
        return b.view(np.int8).astype(np.float64)
    mag = np.append(E4M3_VALUES, np.nan)[b & 0x7f]
    return np.where(b & 0x80, -mag, mag)


def scale_of(most, code):
    lo, hi = EXPONENTS[code]
    e = lo
    while e < hi and most > MOST[code] * 2.0 ** e:
        e += 1
    return 2.0 ** e


def write(codes, scale, new, slots, code):
    """One of keys and values: codes uint8 [blocks][H][16][D], scale float [blocks][H] (both changed), rows new
    [n][H][D], slots [n].  Rows of one block follow one another."""
    nb = codes.shape[0]
    i = 0
    while i < len(slots):
        if not 0 <= slots[i] < nb * BLOCK:
            i += 1
            continue
        b, j = slots[i] // BLOCK, i
        rows = {}
        while j < len(slots) and 0 <= slots[j] < nb * BLOCK and slots[j] // BLOCK == b:
            rows[slots[j] % BLOCK] = j
            j += 1
        for h in range(codes.shape[1]):
            x = {o: np.asarray(new[r, h], np.float64) for o, r in rows.items()}
            size = max([np.abs(v[np.isfinite(v)]).max(initial=0.0) for v in x.values()])
            fresh = 0 in rows
            old = 0.0 if fresh else float(scale[b, h])
            s = max(scale_of(size, code), old)
            for o in range(BLOCK):
                if o in x:
                    codes[b, h, o] = encode(x[o] / s, code)
                elif fresh:
                    codes[b, h, o] = 0
                elif s != old:
                    codes[b, h, o] = encode(decode(codes[b, h, o], code) * (old / s), code)
            scale[b, h] = s
        i = j


def norm(x, w, eps):
    """x [n][heads][D] float64."""
    y = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    return y if w is None else y * w
