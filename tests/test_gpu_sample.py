"""GPU parity of the token drawn from logits against its oracle."""
import numpy as np
import pytest

from oracle import sample as osm

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _ms():
    from paper_2509_08342_amd import moesplit
    return moesplit


def _dev(x, dtype):
    return None if x is None else torch.from_numpy(np.ascontiguousarray(x, dtype)).cuda()


def _run(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, stream=None, offset=0):
    ms = _ms()
    T, n = logits.shape
    buf = torch.full((T * n + offset,), 1e30, dtype=torch.float32, device="cuda")
    buf[offset:] = _dev(logits, np.float32).view(-1)
    opts = ms.sample_opts(_dev(temperature, np.float32), _dev(top_k, np.int32), _dev(top_p, np.float32), _dev(min_p, np.float32))
    idx = torch.full((T + 2,), -7, dtype=torch.int32, device="cuda")
    prob = torch.full((T + 2,), -7.0, dtype=torch.float32, device="cuda")
    need = ms.ms_sample_workspace(T, n)
    ws = torch.full((need + 64,), 0x7f, dtype=torch.uint8, device="cuda")
    ms.ms_sample(buf[offset:].view(T, n), T, n, opts, _dev(u, np.float32), idx[1:-1], prob[1:-1], ws[:need] if need else None,
                 stream or torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert torch.all(ws[need:] == 0x7f)
    idx, prob = idx.cpu().numpy(), prob.cpu().numpy()
    assert idx[0] == idx[-1] == -7 and prob[0] == prob[-1] == -7.0
    return idx[1:-1], prob[1:-1]


def _check(logits, u, temperature=None, top_k=None, top_p=None, min_p=None, **kw):
    """The oracle's token wherever u's mass is not within rounding of a border (weights of 2^-46, 64-bit sums), its share
    to fp32."""
    logits, u = np.asarray(logits, np.float32), np.asarray(u, np.float32)
    idx, prob = _run(logits, u, temperature, top_k, top_p, min_p, **kw)
    at = lambda x, t, d: d if x is None else x[t]  # noqa: E731
    for t in range(len(u)):
        want, share, near = osm.draw(logits[t], u[t], temperature=at(temperature, t, 1.0), top_k=int(at(top_k, t, 0)),
                                     top_p=np.float64(np.float32(at(top_p, t, 1.0))),
                                     min_p=np.float64(np.float32(at(min_p, t, 0.0))))
        if near > 1e-9:
            assert idx[t] == want, (t, idx[t], want, near)
            assert abs(prob[t] - share) <= 2.0 ** -23 * share + 2.0 ** -45


def _settings(rng, T):
    """Rows with every combination of filters on and off, and some greedy."""
    return dict(temperature=np.where(rng.random(T) < 0.1, 0.0, rng.uniform(0.3, 2.0, T)).astype(np.float32),
                top_k=np.where(rng.random(T) < 0.4, 0, rng.integers(1, 90, T)),
                top_p=np.where(rng.random(T) < 0.4, 1.0, rng.uniform(0.05, 0.99, T)).astype(np.float32),
                min_p=np.where(rng.random(T) < 0.5, 0.0, rng.uniform(0.001, 0.5, T)).astype(np.float32))


# vocabularies below, at and past the work-group and its multiples; rows that are not 16-byte aligned
@pytest.mark.parametrize("T,n", [(1, 1), (3, 2), (5, 63), (40, 100), (20, 1024), (9, 1025), (30, 5003), (1, 32000),
                                 (64, 32000), (7, 50257), (2, 200001), (300, 4097), (60, 140001)])
@pytest.mark.parametrize("offset", [0, 1])
def test_settings_of_every_row(T, n, offset):
    rng = np.random.default_rng(T + n)
    logits = 2.5 * rng.standard_normal((T, n))
    logits[rng.random((T, n)) < 10.0 / n] += 6.0
    _check(logits, rng.random(T), **_settings(rng, T), offset=offset)


@pytest.mark.parametrize("which", ["temperature", "top_k", "top_p", "min_p", None])
def test_one_setting_at_a_time(which):
    rng = np.random.default_rng(7)
    T, n = 24, 3001
    logits = 2 * rng.standard_normal((T, n))
    s = _settings(rng, T)
    _check(logits, rng.random(T), **({which: s[which]} if which else {}))


def test_draws_follow_the_weights():
    """Every u on a grid over one row of few tokens: each token at its own share of the grid."""
    rng = np.random.default_rng(2)
    n, T = 50, 4096
    row = 1.5 * rng.standard_normal(n)
    logits = np.tile(row, (T, 1)).astype(np.float32)
    u = (np.arange(T) + 0.5) / T
    _check(logits, u, temperature=np.full(T, 0.8), top_k=np.full(T, 20), top_p=np.full(T, 0.9))


def test_equal_logits():
    """Ties go to the lower index, in whole rows of one value, of few values, and with logits as bf16 has them."""
    rng = np.random.default_rng(4)
    for n in (1, 500, 4096, 40000):
        same = np.full((6, n), 1.25)
        u = np.array([0.0, 0.25, 0.5, 0.999, 0.7, 1 - 2.0 ** -24])
        _check(same, u, top_k=np.array([0, n // 2 + 1, 1, 0, max(n - 3, 1), 7]), top_p=np.array([1, 1, 1, 0.3, 0.6, 1.0]))
    few = rng.integers(0, 4, (12, 30000)) * 0.5
    _check(few, rng.random(12), **_settings(rng, 12))
    coarse = (2.5 * rng.standard_normal((6, 120001))).astype(np.float32).view(np.uint32) & 0xffff0000
    _check(coarse.view(np.float32), rng.random(6), **_settings(rng, 6))


def test_crowded_rows():
    """An outlier, or a mask of large negative numbers, stretches the range of distances; a hot temperature shrinks it."""
    rng = np.random.default_rng(5)
    T, n = 10, 60000
    base = 1e-4 * rng.standard_normal((T, n))
    base[:, 17] = -25.0
    _check(base, rng.random(T), **_settings(rng, T))
    masked = 2 * rng.standard_normal((T, n))
    masked[rng.random((T, n)) < 0.9] = np.float32(-3.4028235e38)
    _check(masked, rng.random(T), **_settings(rng, T))
    hot = 2 * rng.standard_normal((T, n))
    _check(hot, rng.random(T), temperature=np.full(T, 1e4), top_k=np.arange(T) * 700, top_p=np.linspace(0.1, 1, T))


@pytest.mark.parametrize("step", [1 / 4, 1 / 8, 1 / 16, 1 / 64])
@pytest.mark.parametrize("T,n", [(12, 32000), (12, 50257), (6, 131071), (150, 40000)])
def test_many_tokens_to_a_bin(T, n, step):
    """Logits of few values, hundreds or thousands of tokens to each: more in the cuts' bins than are sorted at once,
    more even in one of them."""
    rng = np.random.default_rng(int(1 / step) + n)
    logits = np.round(1.5 * rng.standard_normal((T, n)) / step) * step
    logits[:, ::7] += 2.0 ** -12 * rng.integers(0, 3, (T, (n + 6) // 7))
    s = _settings(rng, T)
    s["temperature"] = np.maximum(s["temperature"], 0.7)
    s["top_k"] = np.where(s["top_k"] > 0, rng.integers(n // 20, n - 1, T), 0)
    s["min_p"] = np.where(s["min_p"] > 0, 2.0 ** -rng.integers(2, 12, T), 0).astype(np.float32)
    _check(logits, rng.random(T), **s)


@pytest.mark.parametrize("T", [1, 2])
def test_the_longest_flat_rows(T):
    rng = np.random.default_rng(T)
    n = 2 ** 19 - 1
    logits = 0.5 * rng.standard_normal((T, n))
    for k, p, m in ((0, 1.0, 0.0), (0, 0.9, 0.0), (400000, 0.5, 0.01), (0, 0.99, 0.3)):
        _check(logits, rng.random(T), top_k=np.full(T, k), top_p=np.full(T, p), min_p=np.full(T, m))


def test_rows_past_32_bits():
    ms = _ms()
    T, n = 8200, 2 ** 19 - 1
    rng = np.random.default_rng(1)
    logits = torch.zeros(T, n, device="cuda")
    last = (2 * rng.standard_normal((3, n))).astype(np.float32)
    logits[-3:] = torch.from_numpy(last).cuda()
    u = rng.random(T).astype(np.float32)
    idx, prob = torch.empty(T, dtype=torch.int32, device="cuda"), torch.empty(T, device="cuda")
    assert ms.ms_sample_workspace(T, n) == 0
    ms.ms_sample(logits, T, n, None, _dev(u, np.float32), idx, prob, None, torch.cuda.current_stream())
    idx, prob = idx.cpu().numpy(), prob.cpu().numpy()
    assert np.all(np.abs(idx[:-3] - np.floor(u[:-3].astype(np.float64) * n)) <= 1) and np.all(np.abs(prob[:-3] * n - 1) < 1e-6)
    for t in range(3):
        want, share, near = osm.draw(last[t], u[T - 3 + t])
        if near > 1e-9:
            assert idx[T - 3 + t] == want and abs(prob[T - 3 + t] - share) <= 2.0 ** -23 * share + 2.0 ** -45
    del logits
    torch.cuda.empty_cache()


def test_extreme_rows():
    inf, nan = np.inf, np.nan
    rows = np.array([[nan, nan, nan, nan, nan], [-inf, -inf, -inf, -inf, -inf], [nan, -inf, 3.0, nan, -inf],
                     [inf, 1.0, inf, -inf, nan], [0.0, -0.0, 0.0, -1.0, -0.0], [-inf, 1.0, 2.0, nan, 2.0],
                     [3e38, -3e38, 3e38, 0.0, 1.0], [1e-40, 2e-40, 0.0, -1e-40, 1e-45]])
    T = len(rows)
    for u in (0.0, 0.3, 0.51, 0.99, 1 - 2.0 ** -24, 1.0, 7.0, -2.0, nan):
        for temp in (1.0, 1e-3, 1e-30, 3e38, inf, 0.0, -1.0, nan):
            _check(rows, np.full(T, u), temperature=np.full(T, temp))
        _check(rows, np.full(T, u), top_k=np.arange(T), top_p=np.full(T, 0.5), min_p=np.full(T, 0.5))


@pytest.mark.parametrize("n", [3000, 32768, 32769, 70001, 300007])
def test_extreme_values_in_long_rows(n):
    """Greedy rows, rows without a logit above -infinity, infinite maxima and ties at the ends of the work-groups' parts,
    rows whose other logits are all far below, NaN among them."""
    rng = np.random.default_rng(n)
    x = (2 * rng.standard_normal((9, n))).astype(np.float32)
    x[0] = np.nan
    x[1] = -np.inf
    x[2, [n - 1, n // 2, 7]] = np.inf
    x[3, rng.random(n) < 0.3] = np.nan
    x[4, [n - 1, n // 3]] = 50.0
    x[5] = -1e30
    x[5, n - 2] = 3.0
    x[6, :n - 1] = -np.inf
    x[7, n // 2:] = -np.inf
    for u in (0.0, 0.4, 0.67, 1 - 2.0 ** -24):
        _check(x, np.full(9, u))
        _check(x, np.full(9, u), temperature=np.zeros(9), top_k=np.full(9, 5))
        _check(x, np.full(9, u), top_k=np.full(9, 2), top_p=np.full(9, 0.9), min_p=np.full(9, 0.2))


def test_filters_at_their_ends():
    """top_k of one, negative and past the row; top_p of nothing, all, more and NaN; min_p of one, more and NaN."""
    rng = np.random.default_rng(6)
    n = 700
    logits = np.tile(rng.standard_normal(n), (6, 1)).astype(np.float32)
    logits[:, [5, 9]] = 4.0  # two largest
    u = np.array([0.0, 0.2, 0.49, 0.51, 0.9, 1 - 2.0 ** -24])
    for k in (1, 2, 3, -5, n - 1, n, n + 1, 2 ** 31 - 1):
        _check(logits, u, top_k=np.full(6, k))
    for p in (0.0, -1.0, 1e-9, 1.0, 1.5, np.nan):
        _check(logits, u, top_p=np.full(6, p))
    for m in (1.0, 2.0, -1.0, 0.999999, np.nan):
        _check(logits, u, min_p=np.full(6, m))


def test_greedy_is_argmax():
    ms = _ms()
    rng = np.random.default_rng(8)
    x = torch.from_numpy(rng.integers(-50, 50, (9, 3001)).astype(np.float32)).cuda()
    ref = torch.empty(9, dtype=torch.int32, device="cuda")
    ms.ms_argmax(x, 9, 3001, ref)
    torch.cuda.synchronize()
    idx, prob = _run(x.cpu().numpy(), rng.random(9), temperature=np.zeros(9), top_k=np.full(9, 40), top_p=np.full(9, 0.1))
    assert np.array_equal(idx, ref.cpu().numpy()) and np.all(prob == 1.0)


@pytest.mark.parametrize("n", [20011, 40009, 60013])
def test_a_row_does_not_depend_on_its_batch(n):
    rng = np.random.default_rng(9)
    T = 400
    logits = (3 * rng.standard_normal((T, n))).astype(np.float32)
    s, u = _settings(rng, T), rng.random(T)
    idx, prob = _run(logits, u, **s)  # a work-group per row; of long rows the smaller batches have several
    for t in (0, 17, 399):
        one = _run(logits[t:t + 1], u[t:t + 1], **{k: v[t:t + 1] for k, v in s.items()})
        assert one[0][0] == idx[t] and one[1][0] == prob[t]
    some = _run(logits[100:140], u[100:140], **{k: v[100:140] for k, v in s.items()})
    assert np.array_equal(some[0], idx[100:140]) and np.array_equal(some[1], prob[100:140])


@pytest.mark.parametrize("T,n", [(1, 32000), (3, 7001), (200, 3001), (1, 40001), (11, 33000), (1, 60001), (9, 150001)])
def test_captured_and_replayed(T, n):
    """A graph replayed with other logits, numbers and settings, the program's own work between the replays; two graphs
    with a workspace each on two streams at once."""
    ms = _ms()
    rng = np.random.default_rng(T)
    sets = [dict(logits=torch.empty(T, n, device="cuda"), u=torch.empty(T, device="cuda"),
                 opts=ms.sample_opts(torch.ones(T, device="cuda"), torch.zeros(T, dtype=torch.int32, device="cuda"),
                                     torch.ones(T, device="cuda"), torch.zeros(T, device="cuda")),
                 idx=torch.empty(T, dtype=torch.int32, device="cuda"), prob=torch.empty(T, device="cuda"),
                 ws=torch.full((max(ms.ms_sample_workspace(T, n), 16),), 0x7f, dtype=torch.uint8, device="cuda"),
                 stream=torch.cuda.Stream(), graph=torch.cuda.CUDAGraph()) for _ in range(2)]
    for s in sets:
        s["logits"].normal_()
        s["u"].uniform_()
    torch.cuda.synchronize()
    for s in sets:
        with torch.cuda.graph(s["graph"], stream=s["stream"]):
            ms.ms_sample(s["logits"], T, n, s["opts"], s["u"], s["idx"], s["prob"], s["ws"], torch.cuda.current_stream())
    for _ in range(4):
        new = []
        for s in sets:
            x, u, v = (2 * rng.standard_normal((T, n))).astype(np.float32), rng.random(T).astype(np.float32), _settings(rng, T)
            for dst, src in zip((s["logits"], s["u"], *s["opts"].tensors),
                                (x, u, v["temperature"], v["top_k"].astype(np.int32), v["top_p"], v["min_p"])):
                dst.copy_(torch.from_numpy(src))
            new.append((x, u, v))
        torch.cuda.synchronize()
        for s in sets:
            with torch.cuda.stream(s["stream"]):
                s["graph"].replay()
        torch.cuda.synchronize()
        for s, (x, u, v) in zip(sets, new):
            idx, prob = _run(x, u, **v)
            assert np.array_equal(s["idx"].cpu().numpy(), idx) and np.array_equal(s["prob"].cpu().numpy(), prob)
        _check(*new[0][:2], **new[0][2])


@pytest.mark.parametrize("min_p,temperature", [(2.0 ** -44, 1.0), (2.0 ** -45, 0.7), (1e-14, 1.0), (2.5e-13, 2.0), (1.0, 3e38)])
def test_a_small_min_p_does_not_depend_on_the_batch(min_p, temperature):
    """Weights that only rounding to whole units of 2^-45 brings up to min_p's are kept, by one work-group a row and by
    several: 20000 tokens of 0.4 units less than it asks for, whose mass moves the drawn token by many of the 900 above them."""
    n, T = 60013, 400
    least = int(np.ceil(np.float32(min_p).astype(np.float64) * 2.0 ** 45))
    rng = np.random.default_rng(least)
    units = np.zeros(n)  # in 2^-45 of the largest
    if min_p < 1:
        units[1:901] = 2500 + 3 * np.arange(900)
        units[901:20901] = least - 0.4
    else:  # all of them round to the largest
        units[1:20901] = 2.0 ** 45 - np.linspace(0, 0.4, 20900)
    units[0] = 2.0 ** 45
    row = np.full(n, -200.0 * temperature if min_p < 1 else -np.inf, np.float64)
    row[:20901] = temperature * np.log(units[:20901] / 2.0 ** 45) if min_p < 1 else -np.linspace(0, 20900, 20901)
    row = rng.permutation(row).astype(np.float32)
    T32 = np.float32(temperature).astype(np.float64)
    w = [int(v) for v in np.rint(2.0 ** 45 * np.exp((row.astype(np.float64) - row.max()) / T32))]
    order = np.lexsort((np.arange(n), -row))
    u = np.float32(1 - 2.0 ** -24)
    kept = [i for i in order if w[i] >= least]
    assert len(kept) == 20901
    M, c = sum(w[i] for i in kept), 0
    for i in kept:
        c += w[i]
        if c * 2 ** 24 > M * (2 ** 24 - 1):
            break
    for rows in (1, T):
        s = dict(temperature=np.full(rows, temperature), min_p=np.full(rows, min_p))
        idx, prob = _run(np.tile(row, (rows, 1)), np.full(rows, u), **s)
        assert (idx == i).all(), (rows, idx[:4], i)
        assert np.all(np.abs(prob - w[i] / M) <= 2.0 ** -23 * w[i] / M)
