"""Plain 64-bit implementations of the calls on 8-bit keys and values, from their definitions (NumPy, on the host)."""
import math

import numpy as np

E_MIN, E_MAX = -64, 64
BLOCK = 64
NAN_CODE = 0x7f


def _decode_table():
    v = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        a = m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7)
        if c & 0x7f == 0x7f:
            a = math.nan
        v[c] = -a if c & 0x80 else a
    return v


VALUES = _decode_table()
GRID = VALUES[:127]


def encode(x):
    """Nearest e4m3 code of x, |x| <= 448, ties to the even code; NaN and infinities to the NaN code."""
    x = np.asarray(x, np.float64)
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    assert a.size == 0 or a.max() <= 448
    i = np.clip(np.searchsorted(GRID, a, side="right") - 1, 0, 125)
    lo, hi = GRID[i], GRID[i + 1]
    up = (a - lo > hi - a) | ((a - lo == hi - a) & (i % 2 == 1))
    code = (i + up).astype(np.uint8) | (np.signbit(x).astype(np.uint8) << 7)
    return np.where(np.isfinite(x), code, np.uint8(NAN_CODE))


def same_codes(a, b):
    """Equal codes, either NaN code for NaN."""
    a, b = np.asarray(a), np.asarray(b)
    return (a == b) | (((a & 0x7f) == 0x7f) & ((b & 0x7f) == 0x7f))


def scale_of(x):
    """The least power of two 2^e, E_MIN <= e <= E_MAX, with |x| <= 448 * 2^e for the finite values of x."""
    a = np.abs(x[np.isfinite(x)])
    top = a.max() if a.size else 0.0
    e = E_MIN
    while e < E_MAX and top > 448 * 2.0 ** e:
        e += 1
    return 2.0 ** e


def norm_rotate(x, weight, eps, cos_sin, position, adjacent):
    """x [..., heads, 128] of tokens at `position` [...]."""
    x = np.asarray(x, np.float64).copy()
    with np.errstate(invalid="ignore", divide="ignore", over="ignore"):
        if weight is not None:
            x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(weight, np.float64)
        if cos_sin is None:
            return x
        half = cos_sin.shape[1]
        cs = np.asarray(cos_sin, np.float64)[np.clip(position, 0, len(cos_sin) - 1)][..., None, :, :]
        i = np.arange(half)
        one, two = (2 * i, 2 * i + 1) if adjacent else (i, i + half)
        a, b, c, s = x[..., one], x[..., two], cs[..., 0], cs[..., 1]
        y = x.copy()
        y[..., one], y[..., two] = a * c - b * s, b * c + a * s
    return y


def quantize(X, perm):
    """X [B, H, L, 128] -> codes [B, H, L, 128], scales [B, H, ceil(L / 64)]."""
    X = np.asarray(X, np.float64)
    B, H, L, d = X.shape
    n = -(-L // BLOCK)
    codes, scales = np.zeros(X.shape, np.uint8), np.zeros((B, H, n))
    for b in range(B):
        for h in range(H):
            x = X[b, h] if perm is None else X[b, h][np.clip(perm[b, h], 0, L - 1)]
            for i in range(n):
                rows = slice(i * BLOCK, (i + 1) * BLOCK)
                scales[b, h, i] = scale_of(x[rows])
                codes[b, h, rows] = encode(x[rows] / scales[b, h, i])
    return codes, scales


def append(codes, scales, table, old, new, first, X):
    """In place: rows first[b] .. first[b] + new[b] - 1 of X [T, H, 128] (64-bit values) behind old[b] tokens of sequence b."""
    n_pages, H, P, _ = codes.shape
    for b in range(len(old)):
        done = 0
        held = min(max(old[b], 0), table.shape[1] * P)
        n = min(new[b], table.shape[1] * P - held)
        while done < n:
            slot = held + done
            o, page = slot % P, table[b, slot // P]
            m = min(P - o, n - done)
            if 0 <= page < n_pages:
                for h in range(H):
                    x = X[first[b] + done:first[b] + done + m, h]
                    sc = scale_of(x)
                    if o:
                        sc = max(sc, scales[page, h])
                        v = VALUES[codes[page, h, :o]] * (scales[page, h] / sc)
                        codes[page, h, :o] = np.where((codes[page, h, :o] & 0x7f) == 0x7f, codes[page, h, :o], encode(v))
                    codes[page, h, o:o + m] = encode(x / sc)
                    scales[page, h] = sc
            done += m


def attend(q, k, v, scale):
    """q [g, 128], k, v [n, 128] -> out [g, 128], lse [g], and how far fp32 accumulation of the scores may move the output."""
    g = len(q)
    if len(k) == 0:
        return np.zeros((g, 128)), np.full(g, -np.inf), np.zeros(g)
    x = q @ k.T * scale
    m = x.max(1, keepdims=True)
    p = np.exp(x - m)
    l = p.sum(1, keepdims=True)
    # a score is a sum of 128 products in fp32, times two factors; the probabilities are sums of two bf16 (2^-17 of themselves),
    # summed in fp32
    dx = (np.abs(q) @ np.abs(k).T * scale).max(1) * 132 * 2.0 ** -24 + np.abs(x).max(1) * 2.0 ** -22
    moved = (2 * dx + 2.0 ** -16 + len(k) * 2.0 ** -24) * np.abs(v).max()
    return (p / l) @ v, (m + np.log(l))[:, 0], np.stack([moved, dx + (len(k) + 64) * 2.0 ** -24], 1)
