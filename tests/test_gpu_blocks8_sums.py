"""The product of two matrices in 8 bits, held to what its sums may be off by: bf16 results before their rounding, and every
block of columns alone."""
import numpy as np
import pytest

from oracle import blocks8 as b8

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")

# sizes of every kernel: few tokens; tiles of 32 x 32, 64 x 64 and 128 x 128, and of 256 tokens with 128, 192 and 256
# outputs, alone and followed by smaller ones; one block of columns to many, whole and ending inside a block
SIZES = [(1, 4112, 130), (16, 400, 300), (30, 1040, 70), (33, 448, 300), (61, 2000, 203), (130, 8192, 200), (129, 1104, 257),
         (300, 16384, 150), (511, 272, 6100), (1030, 1104, 1030), (2000, 144, 8190), (1030, 272, 16400), (1800, 1424, 18504)]


def _product(x, xe, w, we, y, add=None):
    from paper_2509_08342_amd import moesplit as ms
    (T, n_in), n_out = x.shape, w.shape[0]
    ms.ms_dense_q(*[torch.from_numpy(np.ascontiguousarray(v)).cuda() for v in (x, xe, w, we)], T, n_in, n_out, y, add,
                  torch.cuda.current_stream())
    torch.cuda.synchronize()
    return y


def _before_rounding(x, xe, w, we):
    """(a bf16 product as it was before its rounding, to 2^-16 of it; the bf16 product): the rounding's error is the
    product with the rounded one subtracted, which fp32 holds exactly, rounded to bf16 in turn."""
    y = _product(x, xe, w, we, torch.empty(len(x), len(w), dtype=torch.bfloat16, device="cuda"))
    rest = _product(x, xe, w, we, torch.empty_like(y), -y)
    return y.double().cpu().numpy() + rest.double().cpu().numpy(), y.double().cpu().numpy()


def _exponents(c, e, block_rows):
    """The exponent of every value in 8 bits, subnormal codes' that of the smallest normal one; very small for zeros."""
    R, n = c.shape
    f = np.maximum((c >> 3).astype(np.int64) & 15, 1) - 7
    scale = np.log2(b8.spread(e.astype(np.int64) - b8.BIAS, R, n, block_rows)).astype(np.int64)
    return np.where(c & 127, f + scale, -10000)


def _check(x, xe, w, we, spread_of_rows=96):
    """Some results of the product against 64 bits; returns their errors before the rounding and the exact results."""
    T, n_in, n_out = *x.shape, len(w)
    rng = np.random.default_rng(T + n_out)
    t = np.sort(rng.permutation(T)[:spread_of_rows])
    o = np.sort(rng.permutation(n_out)[:max(1, min(spread_of_rows, 2 ** 23 // (len(t) * n_in)))])
    got, rounded = (v[t][:, o] for v in _before_rounding(x, xe, w, we))
    X, W = b8.values(x, xe)[t], b8.values(w, we, 128)[o]
    ref, mags = X @ W.T, np.abs(X) @ np.abs(W).T
    # fp32 sums: the groups of eight columns, 16 and one more to an instruction, and the parts' of a tile's waves
    bound = (n_in / 8 + 8) * 2.0 ** -23 * mags
    if T > 16:  # of eight products, seven are cut by less than 2^-13 of the power of two of the largest exponents
        E = _exponents(x, xe, 1)[t][:, None] + _exponents(w, we, 128)[o][None]
        E = E.reshape(len(t), len(o), n_in // 8, 8).max(axis=-1)
        bound = bound + 7 * 2.0 ** -13 * np.exp2(E.astype(np.float64)).sum(axis=-1)
    read = bound + 2.0 ** -16 * 1.01 * np.abs(ref)
    bad = ~(np.abs(got - ref) <= read)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4], read[bad][:4])
    assert np.all(np.abs(rounded - ref) <= 2.0 ** -8 * np.abs(ref) + 1.01 * bound)
    return got - ref, ref


@pytest.mark.parametrize("T,n_in,n_out", SIZES)
def test_normal_values(T, n_in, n_out):
    """Products of both signs and like sizes: 2e-5 of the results before their rounding (up to 16 tokens the 2^-17 that the
    reading adds)."""
    rng = np.random.default_rng(T)
    x, xe = b8.quantize(rng.standard_normal((T, n_in)))
    w, we = b8.quantize(rng.standard_normal((n_out, n_in)), 128)
    e, ref = _check(x, xe, w, we)
    assert np.sqrt(np.mean(e * e)) <= (2e-5 if T > 16 else 2.0 ** -17) * np.sqrt(np.mean(ref * ref))


@pytest.mark.parametrize("T,n_in,n_out", SIZES[1:])
@pytest.mark.parametrize("kind", ["beside a large one", "subnormal", "any code"])
def test_products_of_unlike_sizes(T, n_in, n_out, kind):
    """Sums that lose the most: one large product and seven small ones of the same sign; rows of subnormal codes and
    zeros; every code and scales far apart."""
    rng = np.random.default_rng(n_in)
    nb = -(-n_in // 128)
    xe, we = np.full((T, nb), b8.BIAS, np.uint8), np.full((-(-n_out // 128), nb), b8.BIAS, np.uint8)
    first = np.arange(n_in) % 8 == 0
    if kind == "beside a large one":
        x = b8.encode(np.where(first, 1.0, 1.875 * np.exp2(-rng.integers(4, 7, (T, 1)))))
        w = b8.encode(np.where(first, 1.0, rng.choice([1.0, 1.375, 1.625, 1.875], (n_out, 1)) * 2.0 ** -6))
    elif kind == "subnormal":
        x = (rng.integers(0, 8, (T, n_in)) | rng.integers(0, 2, (T, n_in)) << 7).astype(np.uint8)
        w = b8.encode(rng.uniform(1, 2, (n_out, n_in)) * np.exp2(rng.integers(-6, 8, (n_out, n_in))))
    else:
        x, w = (rng.integers(0, 127, s).astype(np.uint8) | (rng.integers(0, 2, s) << 7).astype(np.uint8)
                for s in ((T, n_in), (n_out, n_in)))
        xe, we = (e - 4 + rng.integers(0, 9, e.shape).astype(np.uint8) for e in (xe, we))
    _check(x, xe, w, we)


@pytest.mark.parametrize("T,n_in,n_out", SIZES)
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_every_block_of_columns_alone(T, n_in, n_out, dtype):
    """Each token has values in one block of 128 columns only, and scales far apart in all: a block that is left out, read
    twice, from another stage or with another's scale is the whole result."""
    rng = np.random.default_rng(n_out)
    nb = -(-n_in // 128)
    at = (np.arange(T) + np.arange(T) // 16 + nb // 2) % nb
    x = b8.encode(rng.standard_normal((T, n_in)) * 90) * (np.arange(n_in) // 128 == at[:, None])
    xe = (b8.BIAS + rng.integers(-10, 11, (T, nb))).astype(np.uint8)
    w = b8.encode(rng.standard_normal((n_out, n_in)) * 90)
    we = (b8.BIAS + rng.integers(-10, 11, (-(-n_out // 128), nb))).astype(np.uint8)
    y = torch.empty(T, n_out, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    got = _product(x, xe, w, we, y).double().cpu().numpy()
    ref, mags = b8.dense(b8.values(x, xe), b8.values(w, we, 128))
    # a block's groups of eight and what joins them; bf16: eight products lose 7 2^-13 of the largest power of two at most,
    # which is at most eight times (subnormal codes) the sum of theirs, and half a step
    bound = 32 * 2.0 ** -23 * mags
    if dtype == "bf16":
        bound = bound + 7 * 2.0 ** -10 * mags * (T > 16) + 2.0 ** -8 * np.abs(ref)
    bad = ~(np.abs(got - ref) <= 1.01 * bound)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4])
    assert np.mean(np.abs(ref) > 4 * bound) > 0.5  # (most results are far more than what they may be off by)
