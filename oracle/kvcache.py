"""Oracle of the 8-bit key/value cache: e4m3 codes with a power-of-two scale
per 64 positions of a head, rotary positions in either layout, over part of the
head and stretched, and attention with masks, capped scores and distance bias.

TEST INFRASTRUCTURE ONLY, like the rest of this package: plain numpy in fp64,
sharing no code with the GPU library.
"""
from __future__ import annotations

import numpy as np

BLOCK, BIAS, EMIN, EMAX, LARGEST = 64, 127, -40, 40, 448.0


def e4m3_table():
    """The 256 code values: sign, 4 exponent bits (bias 7), 3 mantissa bits,
    exponent 0 subnormal, all ones NaN."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * np.exp2(e - 10.0))
    v[(b & 127) == 127] = np.nan
    return np.where(b >= 128, -v, v)


TABLE = e4m3_table()


def encode(x):
    """Codes of x (fp64): nearest, ties to the even mantissa; finite values past
    the range become the largest code, infinities and NaN the NaN code 0x7f."""
    x = np.asarray(x, np.float64)
    a = np.minimum(np.abs(np.where(np.isfinite(x), x, 0.0)), LARGEST)
    pos = TABLE[:127]  # ascending
    hi = np.clip(np.searchsorted(pos, a), 0, 126)
    lo = np.maximum(hi - 1, 0)
    up, down = pos[hi] - a, a - pos[lo]
    c = np.where((up < down) | ((up == down) & (hi % 2 == 0)), hi, lo)
    c = np.where(a == pos[hi], hi, c).astype(np.uint8)
    c = np.where(np.signbit(x), c | 128, c)
    return np.where(np.isfinite(x), c, 0x7f).astype(np.uint8)


def exponent(x):
    """The least e in range with the largest finite magnitude of x at most 448 * 2^e."""
    x = np.abs(np.asarray(x, np.float64))
    top = np.max(np.where(np.isfinite(x), x, 0.0), initial=0.0)
    e = EMIN
    while e < EMAX and top > LARGEST * 2.0 ** e:
        e += 1
    return e


class Cache:
    """codes [S][H][ctx][D] and exponents [S][H][ctx / 64] of keys and values."""

    def __init__(self, S, H, ctx, D):
        self.k, self.v = (np.zeros((S, H, ctx, D), np.uint8) for _ in range(2))
        self.ke, self.ve = (np.full((S, H, ctx // BLOCK), BIAS, np.uint8) for _ in range(2))

    def values(self, which):
        c, e = (self.k, self.ke) if which == "k" else (self.v, self.ve)
        return TABLE[c] * np.repeat(np.exp2(e.astype(np.float64) - BIAS), BLOCK, axis=2)[..., None]

    def append(self, s, pos0, k, v):
        """k, v [n][H][D] (fp64) of sequence s from position pos0 on."""
        for c, e, new in ((self.k, self.ke, k), (self.v, self.ve, v)):
            n, H, _ = new.shape
            for b in range(pos0 // BLOCK, (pos0 + n - 1) // BLOCK + 1):
                lo, hi = max(pos0, b * BLOCK), min(pos0 + n, (b + 1) * BLOCK)
                for h in range(H):
                    part = new[lo - pos0:hi - pos0, h]
                    ex = exponent(part)
                    if lo > b * BLOCK:
                        was = int(e[s, h, b]) - BIAS
                        ex = max(ex, was)
                        if ex > was:
                            old = c[s, h, b * BLOCK:lo]
                            c[s, h, b * BLOCK:lo] = encode(TABLE[old] * 2.0 ** (was - ex))
                    c[s, h, lo:hi] = encode(part * 2.0 ** -ex)
                    e[s, h, b] = ex + BIAS


def frequencies(rot, base, factor=1.0, orig=0.0, low=1.0, high=32.0):
    """Angle per position of every pair."""
    f = float(base) ** (-2.0 * np.arange(rot // 2) / max(rot, 1))
    if factor == 1.0:
        return f
    g = np.clip((orig * f / (2 * np.pi) - low) / (high - low), 0, 1) if orig > 0 else 0.0
    return f * ((1 - g) / factor + g)


def rope(x, pos, rot, freq, interleaved=False, mscale=1.0):
    """x [..., D] turned at position pos."""
    x = np.array(x, np.float64)
    i = np.arange(rot // 2)
    a, b = (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)
    c, s = np.cos(pos * freq) * mscale, np.sin(pos * freq) * mscale
    xa, xb = x[..., a].copy(), x[..., b].copy()
    x[..., a], x[..., b] = xa * c - xb * s, xb * c + xa * s
    return x


def visible(i, n, window=0, prefix=0, docs=None):
    """Whether the queries at positions i see keys 0 .. n - 1."""
    i, j = np.asarray(i)[:, None], np.arange(n)
    see = (j <= i) & ((window == 0) | (i - j < window)) | (j < prefix)
    if docs is not None:
        see = see & (docs[i] == docs[j]) & (docs[i] >= 0)
    return see


def attention(q, k, v, start, scale=None, softcap=0.0, window=0, prefix=0, slopes=None, docs=None):
    """q [T][Hq][D] at positions start .. start + T - 1, k, v [H][>= start + T][D]
    (fp64).  Returns (out, mags, dscore): the result, the same sums with |v|, and
    the size of an fp32 score's error in 2^-24: products and sums at most D of
    the sum of their magnitudes, four of the score and its bias for the steps
    after."""
    T, Hq, D = q.shape
    G, n = Hq // k.shape[0], start + T
    i = np.arange(start, n)
    see = visible(i, n, window, prefix, docs)
    scale = 1.0 / np.sqrt(D) if not scale else scale
    out, mags, ds = np.zeros((T, Hq, D)), np.zeros((T, Hq, D)), np.zeros((T, Hq))
    for h in range(Hq):
        K, V = k[h // G, :n], v[h // G, :n]
        with np.errstate(invalid="ignore"):
            s = (q[:, h] @ np.where(see.any(axis=0)[:, None], K, 0.0).T) * scale
            z = D * (np.abs(q[:, h]) @ np.where(see.any(axis=0)[:, None], np.abs(K), 0.0).T) * scale
        if softcap:
            s = softcap * np.tanh(s / softcap)
        away = np.abs(i[:, None] - np.arange(n))
        if slopes is not None:
            s = s - slopes[h] * away
            z = z + 4 * slopes[h] * away
        z = z + (32 if softcap else 4) * np.abs(s)
        for t in range(T):
            w = see[t]
            if not w.any():
                continue
            p = np.exp(s[t, w] - s[t, w].max())
            p /= p.sum()
            out[t, h], mags[t, h], ds[t, h] = p @ V[w], p @ np.abs(V[w]), z[t, w].max()
    return out, mags, ds
