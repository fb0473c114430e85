"""Oracle of the dense path in 8 bits: matrices of e4m3 codes with a power of two
per 128 columns of a row or of 128 rows, the residual's addition and norm, and
products.

TEST INFRASTRUCTURE ONLY, like the rest of this package: plain numpy in fp64,
sharing no code with the GPU library.
"""
from __future__ import annotations

import numpy as np

from oracle.kvcache import BIAS, EMAX, EMIN, LARGEST, TABLE, encode

BLOCK = 128


def exponents(x, block_rows):
    """Per block the least e in range with the largest finite magnitude at most 448 * 2^e."""
    R, n = x.shape
    a = np.where(np.isfinite(x), np.abs(x), 0.0)
    a = np.pad(a, ((0, -R % block_rows), (0, -n % BLOCK)))
    top = a.reshape(-1, block_rows, a.shape[1] // BLOCK, BLOCK).max(axis=(1, 3))
    e = np.full(top.shape, EMIN)
    for _ in range(EMAX - EMIN):
        e = np.where(top > LARGEST * np.exp2(e.astype(np.float64)), e + 1, e)
    return np.minimum(e, EMAX)


def spread(e, rows, n, block_rows):
    return np.exp2(np.repeat(np.repeat(e.astype(np.float64), block_rows, 0)[:rows], BLOCK, 1)[:, :n])


def quantize(x, block_rows=1):
    """x [rows][n] -> (codes, stored exponents)."""
    x = np.asarray(x, np.float64)
    e = exponents(x, block_rows)
    return encode(x / spread(e, *x.shape, block_rows)), (e + BIAS).astype(np.uint8)


def values(codes, exps, block_rows=1):
    e = np.clip(exps.astype(np.int64) - BIAS, EMIN, EMAX)
    return TABLE[codes] * spread(e, *codes.shape, block_rows)


def residual_norm(h, y=None, weight=None, eps=1e-6):
    """(x, v) of rows h [T][d]."""
    x = np.asarray(h, np.float64) + (0.0 if y is None else y)
    with np.errstate(invalid="ignore"):
        v = x / np.sqrt(np.mean(x * x, axis=1, keepdims=True) + eps)
        return x, v if weight is None else v * weight


def dense(x, w, add=None):
    """(y, magnitudes): the product of x [T][n_in] and w [n_out][n_in], and the sums of its terms' magnitudes."""
    y, mags = x @ w.T, np.abs(x) @ np.abs(w).T
    return (y, mags) if add is None else (y + add, mags + np.abs(add))
