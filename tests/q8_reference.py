"""The 8-bit pool's stored form, attention over it and the norm + rotation, in 64 bits and written from
their definitions (include/mtserve.h); nothing here calls the library."""
import numpy as np


def e4m3_values():
    """Value of every code: a sign, four exponent bits (bias 7), three mantissa bits; 0x7f and 0xff are NaN."""
    v = np.empty(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        v[c] = (m * 2.0 ** -9 if e == 0 else (8 + m) * 2.0 ** (e - 10)) * (-1 if c & 0x80 else 1)
    v[[0x7F, 0xFF]] = np.nan
    return v


VALUES = e4m3_values()


def quantise(x):
    """Rows [..., D] -> (codes uint8, exponents int, values float64)."""
    x = np.asarray(x, dtype=np.float64)
    finite = np.isfinite(x)
    amax = np.abs(np.where(finite, x, 0.0)).max(-1)
    e = np.full(amax.shape, -60)
    while True:                                      # the smallest e with amax <= 464 * 2^e
        more = (amax > 464.0 * 2.0 ** e) & (e < 60)
        if not more.any():
            break
        e = e + more
    y = np.clip(np.where(finite, x, 0.0) * 2.0 ** -e[..., None].astype(np.float64), -448.0, 448.0)
    # nearest code, ties to the even one: distances to all magnitudes
    grid = VALUES[:0x7F]
    at = np.searchsorted(grid, np.abs(y))            # grid[at - 1] < |y| <= grid[at]
    lo = np.maximum(at - 1, 0)
    d_lo, d_hi = np.abs(y) - grid[lo], grid[at] - np.abs(y)
    code = np.where(d_lo < d_hi, lo, np.where(d_lo > d_hi, at, np.where(lo % 2 == 0, lo, at)))
    code = np.where(np.signbit(x) & finite, code | 0x80, code)
    code = np.where(finite, code, 0x7F).astype(np.uint8)
    return code, e, VALUES[code] * 2.0 ** e[..., None].astype(np.float64)


def granule(D):
    return min(16, D // 4)


def code_offset(kv, h, slot, d, S, D):
    g, t = granule(D), slot % 16
    k = (d // g * 16 + t) * g + d % g
    v = (((d // (4 * g) * 4 + t // 4) * 16 + d % 16) * (g // 4) + d // 16 % (g // 4)) * 4 + t % 4
    return h * 2 * S * (D + 1) + kv * S * D + slot // 16 * 16 * D + (k if kv == 0 else v)


def exp_offset(kv, h, slot, S, D):
    return h * 2 * S * (D + 1) + 2 * S * D + kv * S + slot


def store(image, pages, S, pos0, rows):
    """Rows [2][n][H][D] of one user at positions pos0 .. into the page images uint8 [num_pages][page_bytes]."""
    _, n, H, D = rows.shape
    codes, e, _ = quantise(rows)
    d = np.arange(D)[None, :]
    h = np.arange(H)
    for i in range(n):
        p, s = pages[(pos0 + i) // S], (pos0 + i) % S
        for kv in (0, 1):
            image[p, code_offset(kv, h[:, None], s, d, S, D)] = codes[kv, i]
            image[p, exp_offset(kv, h, s, S, D)] = e[kv, i] + 127


def load(image, pages, S, n, H, D):
    """Values [2][n][H][D] of a user's first n tokens."""
    out = np.empty((2, n, H, D))
    d, h = np.arange(D)[None, :], np.arange(H)
    for i in range(n):
        p, s = pages[i // S], i % S
        for kv in (0, 1):
            e = image[p, exp_offset(kv, h, s, S, D)].astype(np.float64) - 127
            out[kv, i] = VALUES[image[p, code_offset(kv, h[:, None], s, d, S, D)]] * 2.0 ** e[:, None]
    return out


def attention(q, kv, prefix, scale):
    """q [n][Hq][D], kv [2][prefix + n][H][D] -> (out, sum p |v|, largest logit error's scale sum |q k|) in 64 bits."""
    n, Hq, D = q.shape
    H = kv.shape[2]
    out, mag, lsum = np.empty((n, Hq, D)), np.empty((n, Hq, D)), np.empty((n, Hq))
    q = q.astype(np.float64)
    for i in range(n):
        k, v = kv[0, :prefix + i + 1], kv[1, :prefix + i + 1]
        for h in range(Hq):
            kk, vv = k[:, h // (Hq // H)], v[:, h // (Hq // H)]
            s = kk @ q[i, h] * scale
            with np.errstate(invalid="ignore"):
                p = np.exp(s - s.max())
            p /= p.sum()
            out[i, h] = p @ vv
            mag[i, h] = p @ np.abs(vv)
            lsum[i, h] = (np.abs(kk) @ np.abs(q[i, h])).max() * scale
    return out, mag, lsum


def attention_bound(out, mag, lsum, keys, D, f32):
    """How far a result may be off, by arithmetic.  Output: rounded to its type, half a step relative.  Weights: rounded to 11
    bits (22 for fp32 rows, the queries to 24), the hardware exponential (2 steps) and the logits' fp32 sums (a step of the
    largest partial sum for each of D terms, twice for the scaling), each relative to a weight, so to sum p |v|, and once
    more through the sum of the weights; fp32 sums over the keys, joined in stretches."""
    out_step = 2.0 ** -24 if f32 else 2.0 ** -8
    weight = 2.0 ** -22 if f32 else 2.0 ** -11
    logit = (D + 4) * 2.0 ** -24 * lsum[..., None] * (2 if f32 else 1)
    relative = weight + 2 * (2.0 ** -22 + 2 * logit + (keys + 64) * 2.0 ** -24)
    return out_step * np.abs(out) + relative * mag * 1.01 + 1e-37


def norm_rope(x, w, pos, eps, freqs, neighbours, norm=True):
    """x [n][heads][D], positions [n]."""
    x = x.astype(np.float64)
    if norm:
        x = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)
    if w is not None:
        x = x * w.astype(np.float64)
    r = 2 * len(freqs)
    t = pos[:, None, None].astype(np.float64) * freqs
    a, b = (slice(0, r, 2), slice(1, r, 2)) if neighbours else (slice(0, r // 2), slice(r // 2, r))
    y = x.copy()
    y[..., a] = x[..., a] * np.cos(t) - x[..., b] * np.sin(t)
    y[..., b] = x[..., b] * np.cos(t) + x[..., a] * np.sin(t)
    return y
