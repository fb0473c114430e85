"""GPU parity of the 8-bit key/value cache against its oracle: the append with
rotary positions, the cache read back, attention over it, and a run of them as
a decoder makes it, eager and captured."""
import numpy as np
import pytest

import synth
from oracle import kvcache as kv

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _ms():
    from paper_2509_08342_amd import moesplit
    return moesplit


def _bf16(a):
    from workload import to_device
    raw, f = synth.storage(np.ascontiguousarray(a, np.float32), "bf16")
    return to_device(raw, "bf16"), f.astype(np.float64)


def _cache(ref):
    """The oracle cache's codes and exponents on the GPU."""
    return _ms().kv_cache_q(*[torch.from_numpy(x.copy()).cuda() for x in (ref.k, ref.v, ref.ke, ref.ve)])


def _host(cache):
    return [x.cpu().numpy() for x in cache.tensors]


def _random_cache(rng, S, H, ctx, D, spread=3):
    """Every code but NaN's, scales of neighbouring blocks up to 2^spread apart."""
    c = kv.Cache(S, H, ctx, D)
    for codes, exps in ((c.k, c.ke), (c.v, c.ve)):
        x = rng.standard_normal(codes.shape)
        codes[...] = kv.encode(x * 100)
        exps[...] = kv.BIAS - 7 + rng.integers(-spread, spread + 1, exps.shape)
    return c


def _span(spans):
    return torch.tensor(spans, dtype=torch.int32, device="cuda")


# ------------------------------------------------------------------ append

# every width; one token and many; starts and ends inside and at the ends of 64
# positions; all, part (no multiple of 4, and of 8) and none of the head turned, in
# either layout; stretched positions; sequences of their own spans
@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0,rot,inter,factor,orig,spans", [
    (1, 4, 2, 64, 1, 0, 64, False, 1.0, 0, None),
    (1, 4, 2, 128, 1, 1499, 128, False, 1.0, 0, None),
    (1, 8, 1, 256, 3, 62, 256, False, 4.0, 8192, None),
    (3, 3, 1, 64, 70, 31, 32, True, 4.0, 0, None),
    (2, 4, 4, 128, 64, 64, 44, False, 8.0, 512, None),
    (2, 4, 2, 64, 129, 5, 18, False, 1.0, 0, None),
    (1, 4, 2, 128, 200, 1, 6, True, 2.0, 100, None),
    (1, 2, 2, 256, 65, 127, 0, False, 1.0, 0, None),
    (4, 4, 2, 64, 5, 130, 64, True, 1.0, 0, [(130, 5), (0, 1), (61, 5), (128, 3)]),
    (5, 4, 2, 128, 130, 100, 128, False, 1.0, 0, [(100, 130), (-1, 4), (3, 0), (101, 2), (37, 131)]),
])
def test_append(S, Hq, Hkv, D, T, pos0, rot, inter, factor, orig, spans):
    ms = _ms()
    rng = np.random.default_rng(T + pos0 + D)
    ctx = -(-(pos0 + T) // 64) * 64 + 64
    ref = _random_cache(rng, S, Hkv, ctx, D)
    cache = _cache(ref)
    before = _host(cache)
    qkv = rng.standard_normal((S, T, Hq + 2 * Hkv, D)).astype(np.float32)
    qkv[:, :, Hq] *= 37.0  # the first key head raises its scales, the others keep what is there or start anew
    q = torch.full((S, T, Hq, D), -7.0, dtype=torch.bfloat16, device="cuda")
    ms.ms_rope_kv_q(cache, ms.rope_desc(rot, 1e4, inter, factor, orig, 1.0, 8.0, 1.25), torch.from_numpy(qkv).cuda(), T, Hq,
                    pos0, q, None if spans is None else _span(spans), torch.cuda.current_stream())
    torch.cuda.synchronize()
    k, v, ke, ve = _host(cache)
    qg = q.float().cpu().numpy()
    f = kv.frequencies(rot, 1e4, factor, orig, 1.0, 8.0)
    for s in range(S):
        start, n = (pos0, T) if spans is None else spans[s]
        if not (0 <= start <= pos0 and 1 <= n <= T):
            start, n = 0, 0
        x = qkv[s, :n].astype(np.float64)
        turned = np.stack([kv.rope(x[t], start + t, rot, f, inter, 1.25) for t in range(n)]) if n else x
        # two products and a sum in fp32, of a sine and cosine rounded to it: 8 half steps of the pair's size
        err = 2.0 ** -21 * 1.25 * np.abs(x).max(axis=-1, initial=0, keepdims=True)
        assert np.all(np.abs(qg[s, :n] - turned[:, :Hq]) <= 2.0 ** -8 * np.abs(turned[:, :Hq]) + err[:, :Hq])
        assert np.all(qg[s, n:] == -7.0)
        if n:
            ref.append(s, start, turned[:, Hq:Hq + Hkv], x[:, Hq + Hkv:])
        assert np.array_equal(ke[s], ref.ke[s]) and np.array_equal(ve[s], ref.ve[s])
        rows = np.zeros(ctx, bool)
        rows[start // 64 * 64:start + n] = n > 0
        # values are not turned: the same codes.  Keys: half a step of the code and the turn's error
        assert np.array_equal(v[s], ref.v[s])
        got = kv.TABLE[k[s]] * np.repeat(np.exp2(ke[s].astype(float) - kv.BIAS), 64, axis=1)[..., None]
        unit = np.repeat(np.exp2(ke[s].astype(float) - kv.BIAS), 64, axis=1)[:, start:start + n, None]
        want = turned[:, Hq:Hq + Hkv].transpose(1, 0, 2)
        half = np.maximum(2.0 ** -4 * np.abs(want), 2.0 ** -10 * unit)
        assert np.all(np.abs(got[:, start:start + n] - want) <= half * (1 + 2.0 ** -20) + err[:, Hq:Hq + Hkv].transpose(1, 0, 2))
        assert np.array_equal(k[s][:, ~rows], before[0][s][:, ~rows]) and np.array_equal(v[s][:, ~rows], before[1][s][:, ~rows])
        old = np.arange(ctx)
        old = (old >= start // 64 * 64) & (old < start)
        assert np.array_equal(k[s][:, old], ref.k[s][:, old])


def test_append_token_by_token():
    """A decode of 130 tokens, keys not turned: codes and scales are the oracle's, bit by bit, through every raised scale."""
    ms = _ms()
    rng = np.random.default_rng(11)
    S, H, D, ctx = 2, 2, 64, 192
    ref, cache = kv.Cache(S, H, ctx, D), ms.new_kv_cache_q(S, H, D, ctx)
    q = torch.empty(S, 1, H, D, dtype=torch.bfloat16, device="cuda")
    for p in range(130):
        x = (rng.standard_normal((S, 1, 3 * H, D)) * 2.0 ** rng.integers(-6, 3)).astype(np.float32)
        ms.ms_rope_kv_q(cache, ms.rope_desc(0, 1e4), torch.from_numpy(x).cuda(), 1, H, p, q)
        for s in range(S):
            ref.append(s, p, x[s, :, H:2 * H].astype(np.float64), x[s, :, 2 * H:].astype(np.float64))
    torch.cuda.synchronize()
    for got, want in zip(_host(cache), (ref.k, ref.v, ref.ke, ref.ve)):
        assert np.array_equal(got, want)


def test_append_of_extreme_values():
    """Infinities and NaN become the NaN code and leave the scale to the finite values; magnitudes past the largest scale
    saturate, those below the smallest vanish."""
    ms = _ms()
    H, D, T = 1, 64, 64
    x = np.zeros((1, T, 3, D), np.float32)
    x[0, :, 1] = np.linspace(-3, 3, T * D).reshape(T, D)
    x[0, 5, 1, 7], x[0, 6, 1, 8], x[0, 7, 1, 9] = np.inf, -np.inf, np.nan
    x[0, :, 2] = 1e-16 * np.linspace(-1, 1, T * D).reshape(T, D)
    x[0, 9, 2, 3] = 3e38
    x[0, 10, 2, 4] = 1e-45
    ref, cache = kv.Cache(1, H, 64, D), ms.new_kv_cache_q(1, H, D, 64)
    q = torch.empty(1, T, 1, D, dtype=torch.bfloat16, device="cuda")
    ms.ms_rope_kv_q(cache, ms.rope_desc(0, 1e4), torch.from_numpy(x).cuda(), T, 1, 0, q)
    ref.append(0, 0, x[0, :, 1:2].astype(np.float64), x[0, :, 2:].astype(np.float64))
    torch.cuda.synchronize()
    k, v, ke, ve = _host(cache)
    assert np.array_equal(ke, ref.ke) and np.array_equal(ve, ref.ve) and ve[0, 0, 0] == kv.BIAS + kv.EMAX
    for a, b in ((k, ref.k), (v, ref.v)):
        assert np.array_equal(np.isnan(kv.TABLE[a]), np.isnan(kv.TABLE[b]))
        fine = ~np.isnan(kv.TABLE[b])
        assert np.array_equal(kv.TABLE[a][fine], kv.TABLE[b][fine])


def test_far_positions_turn_by_exact_angles():
    ms = _ms()
    H, D, pos0 = 1, 128, (1 << 20) - 64
    rng = np.random.default_rng(5)
    x = rng.standard_normal((1, 3, 3, D)).astype(np.float32)
    cache = ms.new_kv_cache_q(1, H, D, 1 << 20)
    q = torch.empty(1, 3, 1, D, dtype=torch.bfloat16, device="cuda")
    ms.ms_rope_kv_q(cache, ms.rope_desc(D, 1e4), torch.from_numpy(x).cuda(), 3, 1, pos0, q)
    torch.cuda.synchronize()
    want = np.stack([kv.rope(x[0, t, :1], pos0 + t, D, kv.frequencies(D, 1e4)) for t in range(3)])
    assert np.all(np.abs(q[0].float().cpu().numpy() - want) <= 2.0 ** -8 * np.abs(want) + 2.0 ** -21 * np.abs(x).max())


@pytest.mark.parametrize("S,H,D,ctx,pos0,n", [(1, 1, 64, 64, 0, 1), (2, 3, 64, 256, 63, 130), (1, 2, 128, 192, 0, 192),
                                              (3, 1, 256, 128, 100, 28)])
def test_read(S, H, D, ctx, pos0, n):
    ms = _ms()
    ref = _random_cache(np.random.default_rng(n), S, H, ctx, D, spread=30)
    ref.k[0, 0, pos0, :3] = 0x7f, 0xff, 0x01
    ref.ke[0, 0, pos0 // 64], ref.ve[0, 0, pos0 // 64] = kv.BIAS + kv.EMIN, kv.BIAS + kv.EMAX
    cache = _cache(ref)
    bufs = [torch.full((S * H * n * D + 8,), -7.0, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    k, v = (b[:S * H * n * D].view(S, H, n, D) for b in bufs)
    ms.ms_kv_read_q(cache, pos0, n, k, v, torch.cuda.current_stream())
    torch.cuda.synchronize()
    for got, which, buf in ((k, "k", bufs[0]), (v, "v", bufs[1])):
        want = ref.values(which)[:, :, pos0:pos0 + n]
        assert np.array_equal(got.float().cpu().numpy().astype(np.float64), want, equal_nan=True)
        assert np.all(buf[S * H * n * D:].float().cpu().numpy() == -7.0)


# --------------------------------------------------------------- attention

def _close(got, ref, mags, ds, n, vmax):
    """The result's rounding to bf16; of every probability its fp16 half step and its score's error; and half the
    smallest fp16 step of every key relative to 2^7, to which the largest probability is scaled."""
    bound = 2.0 ** -8 * np.abs(ref) + mags * (2.0 ** -11 + 2 * ds[..., None] * 2.0 ** -24) * 1.01 + n * 2.0 ** -32 * vmax
    bad = ~(np.abs(got - ref) <= bound)
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4], bound[bad][:4])


def _run(cache, q, T, Hq, pos0, opts=None, span=None, out=None, stream=None):
    ms = _ms()
    if out is None:
        out = torch.full_like(q, -7.0)
    need = ms.ms_attention_q_workspace(cache, T, Hq, pos0)
    ws = torch.full((need + 64,), 0x7f, dtype=torch.uint8, device="cuda")  # fp32 of 3e38, past the end too
    ms.ms_attention_q(cache, q, T, Hq, pos0, out, ws[:need] if need else None, opts, span,
                      stream or torch.cuda.current_stream())
    torch.cuda.synchronize()
    assert bool((ws[need:] == 0x7f).all())
    return out


def _check(ref, qf, got, pos0, spans, **kw):
    """got [S][T][Hq][D] against the oracle; rows not in use keep -7."""
    S, T = qf.shape[:2]
    docs = kw.pop("docs", None)
    vals = {w: ref.values(w) for w in "kv"}
    for s in range(S):
        start, n = (pos0, T) if spans is None else spans[s]
        if not (0 <= start <= pos0 and 1 <= n <= T):
            n = 0
        assert np.all(got[s, n:] == -7.0)
        if n:
            o, mags, ds = kv.attention(qf[s, :n], vals["k"][s], vals["v"][s], start, docs=None if docs is None else docs[s], **kw)
            _close(got[s, :n], o, mags, ds, start + n, np.abs(np.nan_to_num(vals["v"][s])).max())


# (S, Hq, Hkv, D, T, pos0): one token, few, a block's worth, prompts; one query head
# per key/value head, three, four, eight, sixteen and 71; contexts that end inside, at and
# just past a tile; long ones that are split
SHAPES = [(1, 1, 1, 64, 1, 0), (1, 4, 2, 64, 1, 63), (2, 4, 2, 64, 1, 64), (1, 32, 8, 128, 1, 1500), (3, 6, 2, 64, 1, 700),
          (1, 8, 1, 256, 1, 333), (1, 16, 1, 128, 1, 4100), (2, 71, 1, 64, 1, 129), (1, 2, 2, 128, 1, 9000),
          (1, 16, 2, 256, 1, 5003), (33, 4, 4, 64, 1, 77),
          (1, 4, 2, 64, 3, 61), (2, 8, 2, 128, 5, 1000), (1, 3, 1, 64, 16, 0), (1, 8, 1, 256, 2, 190), (2, 6, 2, 64, 9, 4000),
          (1, 4, 2, 64, 64, 0), (1, 4, 2, 64, 65, 0), (1, 8, 2, 128, 200, 0), (2, 3, 1, 64, 130, 33), (1, 4, 1, 128, 333, 1000),
          (1, 8, 1, 256, 150, 20), (1, 5, 5, 64, 40, 6000), (1, 16, 16, 64, 257, 0), (1, 32, 2, 128, 600, 3)]


@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0", SHAPES)
def test_attention(S, Hq, Hkv, D, T, pos0):
    rng = np.random.default_rng(T + pos0 + D)
    ctx = -(-(pos0 + T) // 64) * 64 + 64
    ref = _random_cache(rng, S, Hkv, ctx, D)
    q, qf = _bf16(2 * rng.standard_normal((S, T, Hq, D)))
    _check(ref, qf, _run(_cache(ref), q, T, Hq, pos0).float().cpu().numpy(), pos0, None)


# a cap, a bias, windows (one key, inside a tile, several tiles), prefixes (shorter and
# longer than what is there), and all of them
MASKS = [dict(softcap=5.0), dict(slopes=True), dict(window=1), dict(window=37), dict(window=200), dict(prefix=10),
         dict(prefix=150), dict(prefix=100000), dict(window=70, prefix=5), dict(scale=0.25),
         dict(softcap=20.0, slopes=True, window=130, prefix=70, scale=0.1)]


@pytest.mark.parametrize("kw", MASKS, ids=[",".join(m) + str(list(m.values())[0]) for m in MASKS])
@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0", [(2, 4, 2, 64, 1, 700), (1, 6, 1, 128, 1, 3000), (1, 4, 2, 128, 7, 350),
                                               (1, 4, 2, 64, 300, 0), (1, 8, 2, 128, 150, 260), (1, 8, 1, 256, 100, 90)])
def test_attention_masks(S, Hq, Hkv, D, T, pos0, kw):
    ms = _ms()
    rng = np.random.default_rng(T + pos0)
    ctx = -(-(pos0 + T) // 64) * 64
    ref = _random_cache(rng, S, Hkv, ctx, D)
    q, qf = _bf16(2 * rng.standard_normal((S, T, Hq, D)))
    kw = dict(kw)
    if "slopes" in kw:
        kw["slopes"] = (0.5 ** np.arange(1, Hq + 1)).astype(np.float32)
    opts = ms.attn_opts(**{k: torch.from_numpy(x).cuda() if k == "slopes" else x for k, x in kw.items()})
    _check(ref, qf, _run(_cache(ref), q, T, Hq, pos0, opts).float().cpu().numpy(), pos0, None, **kw)


@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0", [(2, 4, 2, 64, 1, 700), (1, 8, 2, 128, 150, 260), (1, 8, 1, 256, 100, 90)])
@pytest.mark.parametrize("cap", [0.01, 1.0, 128.0, 129.0, 5000.0])
@pytest.mark.parametrize("size", [0.1, 2.0, 200.0])
def test_attention_caps(S, Hq, Hkv, D, T, pos0, cap, size):
    """Caps on both sides of where tanh is taken another way, scores far below, around and far above them."""
    rng = np.random.default_rng(int(cap))
    ref = _random_cache(rng, S, Hkv, -(-(pos0 + T) // 64) * 64, D)
    q, qf = _bf16(size * rng.standard_normal((S, T, Hq, D)))
    got = _run(_cache(ref), q, T, Hq, pos0, _ms().attn_opts(softcap=cap)).float().cpu().numpy()
    for s in range(S):
        o, mags, ds = kv.attention(qf[s], ref.values("k")[s], ref.values("v")[s], pos0, softcap=cap)
        # tanh = 1 - 2 / (1 + e): e off by 2^-23 and 2 |x| 2^-23 of itself, of which the slope (1 - tanh^2) / 2 leaves
        # 2^-23, the reciprocal 2^-23 of at most 2, the last rounding 2^-24: 7 steps of 2^-24 of the cap
        _close(got[s], o, mags, ds + 7 * min(cap, 128.0), pos0 + T, np.abs(ref.values("v")).max())


@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0", [(1, 4, 2, 64, 300, 0), (2, 4, 1, 128, 150, 100), (1, 8, 1, 256, 70, 3),
                                               (3, 4, 2, 64, 1, 500), (1, 8, 2, 128, 5, 2000)])
@pytest.mark.parametrize("length", [1, 50, 64, 130])
@pytest.mark.parametrize("more", [{}, dict(window=40, prefix=90, softcap=10.0)])
def test_attention_documents(S, Hq, Hkv, D, T, pos0, length, more):
    """Packed documents, one of them in two places, padding whose queries see nothing (zeros)."""
    ms = _ms()
    rng = np.random.default_rng(length)
    ctx = -(-(pos0 + T) // 64) * 64
    ref = _random_cache(rng, S, Hkv, ctx, D)
    q, qf = _bf16(2 * rng.standard_normal((S, T, Hq, D)))
    docs = np.tile(np.arange(ctx, dtype=np.int32) // length, (S, 1))
    docs[:, : min(20, pos0 + T - 1)] = docs[0, pos0 + T - 1]
    docs[0, max(0, pos0 + T - T // 3):] = -1
    docs[:, pos0 + T:] = docs[0, pos0]  # past the end: never seen
    opts = ms.attn_opts(doc=torch.from_numpy(docs).cuda(), **more)
    got = _run(_cache(ref), q, T, Hq, pos0, opts).float().cpu().numpy()
    _check(ref, qf, got, pos0, None, docs=docs, **more)
    if T >= 3:
        assert not np.any(got[0, T - T // 3:])


@pytest.mark.parametrize("Hq,Hkv,D,T,pos0,spans", [
    (4, 2, 64, 1, 900, [(900, 1), (0, 1), (63, 1), (64, 1), (-1, 1), (901, 1), (5, 0), (450, 1), (7, 2)]),
    (8, 2, 128, 4, 3000, [(3000, 4), (1000, 1), (0, 3), (2999, 4), (-5, -5)]),
    (4, 1, 64, 100, 500, [(500, 100), (0, 100), (321, 3), (2, 64), (600, 100)]),
    (8, 1, 256, 40, 64, [(64, 40), (0, 1), (30, 33)])])
@pytest.mark.parametrize("kw", [{}, dict(window=50, prefix=3)])
def test_attention_spans(Hq, Hkv, D, T, pos0, spans, kw):
    ms = _ms()
    rng = np.random.default_rng(T)
    S, ctx = len(spans), -(-(pos0 + T) // 64) * 64
    ref = _random_cache(rng, S, Hkv, ctx, D)
    q, qf = _bf16(2 * rng.standard_normal((S, T, Hq, D)))
    got = _run(_cache(ref), q, T, Hq, pos0, ms.attn_opts(**kw), _span(spans)).float().cpu().numpy()
    _check(ref, qf, got, pos0, spans, **kw)


@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0", [(1, 4, 2, 64, 1, 700), (1, 8, 2, 128, 1, 5000), (1, 4, 2, 128, 6, 350),
                                               (1, 4, 2, 64, 300, 0), (1, 4, 1, 128, 200, 100), (1, 8, 1, 256, 90, 60)])
def test_attention_does_not_see_what_is_masked(S, Hq, Hkv, D, T, pos0):
    """NaN in the cache past the sequence, and in a key and a value of the call's own tokens: the former reach no query,
    the latter those that see them only."""
    rng = np.random.default_rng(T)
    n = pos0 + T
    ctx = -(-n // 64) * 64 + 64
    ref = _random_cache(rng, S, Hkv, ctx, D)
    ref.k[:, :, n:], ref.v[:, :, n:] = 0x7f, 0xff
    q, qf = _bf16(2 * rng.standard_normal((S, T, Hq, D)))
    _check(ref, qf, _run(_cache(ref), q, T, Hq, pos0).float().cpu().numpy(), pos0, None)
    at, nan_key = pos0 + T // 2, pos0 + T - 1
    clean = [w.copy() for w in (ref.k, ref.v)]
    ref.v[:, :, at, 3] = 0x7f
    ref.k[:, Hkv - 1, nan_key, 5] = 0x7f
    got = _run(_cache(ref), q, T, Hq, pos0).float().cpu().numpy()
    ref.k, ref.v = clean
    vals = {w: ref.values(w) for w in "kv"}
    o, mags, ds = kv.attention(qf[0], vals["k"][0], vals["v"][0], pos0)
    i = np.arange(pos0, n)
    want = np.zeros(o.shape, bool)
    want[i >= at, :, 3] = True
    want[i >= nan_key, (Hkv - 1) * (Hq // Hkv):] = True
    assert np.array_equal(np.isnan(got[0]), want)
    o, got0 = np.where(want, 0.0, o), np.where(want, 0.0, got[0])
    _close(got0, o, mags, ds, n, np.abs(np.nan_to_num(vals["v"])).max())


@pytest.mark.parametrize("T,pos0", [(1, 3000), (4, 500), (150, 200)])
@pytest.mark.parametrize("far", [0, 10, 60])
def test_attention_of_blocks_far_apart_in_scale(T, pos0, far):
    """Values of some blocks 2^far times the others', probabilities that favour either: the small ones still count."""
    rng = np.random.default_rng(far)
    S, Hq, Hkv, D = 1, 8, 2, 128
    ctx = -(-(pos0 + T) // 64) * 64
    ref = _random_cache(rng, S, Hkv, ctx, D, spread=0)
    ref.ve[:, :, ::2] = np.clip(ref.ve[:, :, ::2].astype(int) + far // 2, kv.BIAS + kv.EMIN, kv.BIAS + kv.EMAX)
    ref.ve[:, :, 1::2] = np.clip(ref.ve[:, :, 1::2].astype(int) - (far - far // 2), kv.BIAS + kv.EMIN, kv.BIAS + kv.EMAX)
    for name, sign in (("even", 1.0), ("odd", -1.0)):
        # the first value of a key says which blocks it belongs to; the query's turns that into a score of 0 or -50
        ref.k[:, :, :, 0] = kv.encode(np.where(np.arange(ctx) // 64 % 2 == 0, 100.0, -100.0))
        ref.ke[:, :, :] = kv.BIAS - 7
        qv = 0.5 * rng.standard_normal((S, T, Hq, D))
        qv[..., 0] = sign * 25.0 * np.sqrt(D) / (100.0 / 128)
        q, qf = _bf16(qv)
        _check(ref, qf, _run(_cache(ref), q, T, Hq, pos0).float().cpu().numpy(), pos0, None)


@pytest.mark.parametrize("T,pos0", [(1, 3000), (4, 500), (150, 200)])
@pytest.mark.parametrize("apart", [5, 8, 20, 33, 80])
def test_small_and_zero_values_keep_their_weight(T, pos0, apart):
    """Scores that favour no block, values of every third block 2^apart below the others', the least scale of all with
    zeros in it at 80: what they weigh counts in every row's sum, whichever block comes first."""
    rng = np.random.default_rng(apart)
    S, Hq, Hkv, D = 1, 8, 2, 64
    ctx = -(-(pos0 + T) // 64) * 64
    for first in (0, 1):
        ref = _random_cache(rng, S, Hkv, ctx, D, spread=0)
        ref.ve[:, :, first::3] = max(kv.BIAS - 7 - apart, kv.BIAS + kv.EMIN)
        if apart == 80:
            zero = np.arange(ctx) // 64 % 3 == first
            ref.v[:, :, zero] = 0
        q, qf = _bf16(0.5 * rng.standard_normal((S, T, Hq, D)))
        got = _run(_cache(ref), q, T, Hq, pos0).float().cpu().numpy()
        o, mags, ds = kv.attention(qf[0], ref.values("k")[0], ref.values("v")[0], pos0)
        # the sum's probabilities may be other fp16 numbers than the values' then: half a step of each, 2^13 more of ds / 2;
        # and the 2^-28 of the largest weight for a key that the sum may leave out
        n = pos0 + T
        _close(got[0], o, mags * (1 + n * 2.0 ** -17), ds + 2.0 ** 12, n, np.abs(ref.values("v")).max())


@pytest.mark.parametrize("T,pos0", [(1, 700), (5, 100), (150, 64)])
@pytest.mark.parametrize("exponent", [20, 36, 60])
@pytest.mark.parametrize("sign", [1, -1])
def test_attention_large_scores(T, pos0, exponent, sign):
    """Scores of 1e6 to 1e18, three distinct and exact ones: the largest keys share the weight."""
    rng = np.random.default_rng(T + exponent)
    S, Hq, Hkv, D = 1, 4, 1, 64
    ctx = -(-(pos0 + T) // 64) * 64
    ref = _random_cache(rng, S, Hkv, ctx, D)
    ref.k[...] = kv.encode(sign * (1.25 + rng.integers(0, 3, (S, Hkv, ctx, 1)) / 8.0) * np.ones(D))
    ref.ke[...] = kv.BIAS + exponent - exponent // 2
    q, qf = _bf16(np.full((S, T, Hq, D), 1.5 * 2.0 ** (exponent // 2)))
    got = _run(_cache(ref), q, T, Hq, pos0).float().cpu().numpy()
    o, mags, _ = kv.attention(qf[0], ref.values("k")[0], ref.values("v")[0], pos0)
    _close(got[0], o, mags, np.zeros(o.shape[:2]), ctx, np.abs(ref.values("v")).max())


def test_attention_in_place_and_on_another_stream():
    rng = np.random.default_rng(1)
    for S, Hq, Hkv, D, T, pos0 in [(1, 8, 2, 128, 1, 4000), (2, 4, 2, 64, 5, 300), (1, 4, 2, 64, 200, 100)]:
        ref = _random_cache(rng, S, Hkv, -(-(pos0 + T) // 64) * 64, D)
        q, qf = _bf16(rng.standard_normal((S, T, Hq, D)))
        cache, stream = _cache(ref), torch.cuda.Stream()
        torch.cuda.synchronize()
        _check(ref, qf, _run(cache, q, T, Hq, pos0, out=q, stream=stream).float().cpu().numpy(), pos0, None)


def test_long_caches_pass_32_bits():
    """The second head of a cache of 5 GiB: offsets past 2^32."""
    ms = _ms()
    D, ctx = 256, 10 << 20
    if torch.cuda.mem_get_info()[0] < 12 << 30:
        pytest.skip("needs 12 GiB")
    cache = ms.new_kv_cache_q(1, 2, D, ctx)
    rng = np.random.default_rng(2)
    pos0, T = ctx - 70, 70
    x = rng.standard_normal((1, T, 6, D)).astype(np.float32)
    q = torch.empty(1, T, 2, D, dtype=torch.bfloat16, device="cuda")
    ms.ms_rope_kv_q(cache, ms.rope_desc(0, 1e4), torch.from_numpy(x).cuda(), T, 2, pos0, q)
    k, v = (torch.empty(1, 2, T, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ms.ms_kv_read_q(cache, pos0, T, k, v)
    out = _run(cache, q, T, 2, pos0, ms.attn_opts(window=50)).float().cpu().numpy()
    ref = kv.Cache(1, 2, 128, D)  # the last 128 positions: 58 keys before the call's own, more than the window
    ref.append(0, 58, x[0, :, 2:4].astype(np.float64), x[0, :, 4:].astype(np.float64))
    assert np.array_equal(k[0].float().cpu().numpy().astype(np.float64), ref.values("k")[0][:, 58:])
    assert np.array_equal(v[0].float().cpu().numpy().astype(np.float64), ref.values("v")[0][:, 58:])
    qf = q.float().cpu().numpy().astype(np.float64)
    o, mags, ds = kv.attention(qf[0], ref.values("k")[0], ref.values("v")[0], 58, window=50)
    _close(out[0], o, mags, ds, 128, np.abs(ref.values("v")).max())


# ------------------------------------------------------------ used together

def _steps(ms, cache, qkv, q, out, ws, desc, opts, span, T, Hq, pos0, stream):
    ms.ms_rope_kv_q(cache, desc, qkv, T, Hq, pos0, q, span, stream)
    ms.ms_attention_q(cache, q, T, Hq, pos0, out, ws, opts, span, stream)


def test_prompt_then_decode_eager_and_captured():
    """Three sequences of different prompt lengths, then six tokens each: the eager calls against the oracle, and the same
    decode captured once and replayed with positions that change on the device."""
    ms = _ms()
    rng = np.random.default_rng(8)
    S, Hq, Hkv, D, ctx, P, n_dec = 3, 6, 2, 64, 512, 150, 6
    desc = ms.rope_desc(48, 1e4, True, 4.0, 128, 1.0, 8.0, 1.1)
    kw = dict(softcap=30.0, window=100, prefix=4)
    opts = ms.attn_opts(**kw)
    lens = [150, 64, 97]
    prompt = rng.standard_normal((S, P, Hq + 2 * Hkv, D)).astype(np.float32)
    toks = rng.standard_normal((n_dec, S, 1, Hq + 2 * Hkv, D)).astype(np.float32)
    stream = torch.cuda.Stream()
    results = []
    for captured in (False, True):
        cache = ms.new_kv_cache_q(S, Hkv, D, ctx)
        q, out = (torch.zeros(S, P, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        q1, out1 = (torch.zeros(S, 1, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        need = max(ms.ms_attention_q_workspace(cache, P, Hq, 0), ms.ms_attention_q_workspace(cache, 1, Hq, ctx - 1), 16)
        ws = torch.empty(need, dtype=torch.uint8, device="cuda")
        span = _span([(0, n) for n in lens])
        x, x1 = torch.from_numpy(prompt).cuda(), torch.zeros(S, 1, Hq + 2 * Hkv, D, device="cuda")
        torch.cuda.synchronize()
        with torch.cuda.stream(stream):
            _steps(ms, cache, x, q, out, ws, desc, opts, span, P, Hq, 0, stream)
            got = [out.clone()]
            span.copy_(_span([(n, 1) for n in lens]))
            stream.synchronize()
            graph = None
            if captured:
                graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(graph, stream=stream):
                    _steps(ms, cache, x1, q1, out1, ws, desc, opts, span, 1, Hq, ctx - 1, stream)
            for i in range(n_dec):
                x1.copy_(torch.from_numpy(toks[i]))
                if graph is not None:
                    graph.replay()
                else:
                    _steps(ms, cache, x1, q1, out1, ws, desc, opts, span, 1, Hq, ctx - 1, stream)
                got.append(out1.clone())
                span[:, 0] += 1
            stream.synchronize()
        results.append([g.float().cpu().numpy() for g in got] + _host(cache))
    for a, b in zip(*results):
        assert np.array_equal(a, b)
    f = kv.frequencies(48, 1e4, 4.0, 128, 1.0, 8.0)
    got, (k, v, ke, ve) = results[0][:1 + n_dec], results[0][1 + n_dec:]
    final = kv.Cache(S, Hkv, ctx, D)
    final.k, final.v, final.ke, final.ve = k, v, ke, ve
    for s in range(S):
        # values are not turned: the append in pieces is the oracle's; attention over the cache as it was left
        ref = kv.Cache(1, Hkv, ctx, D)
        z = np.zeros((lens[s], Hkv, D))
        ref.append(0, 0, z, prompt[s, :lens[s], Hq + Hkv:].astype(np.float64))
        for i in range(n_dec):
            ref.append(0, lens[s] + i, z[:1], toks[i, s, :, Hq + Hkv:].astype(np.float64))
        n = lens[s] + n_dec
        assert np.array_equal(v[s, :, :n], ref.v[0, :, :n]) and np.array_equal(ve[s], ref.ve[0])
        pos = lens[s] + n_dec - 1
        qf = kv.rope(toks[-1, s, :, :Hq].astype(np.float64), pos, 48, f, True, 1.1)
        qf = _bf16(qf)[1]
        o, mags, ds = kv.attention(qf, final.values("k")[s], final.values("v")[s], pos, **kw)
        vmax = np.abs(final.values("v")[s]).max()
        # a query's own rounding to bf16 may differ by a step where its turn is rounded: one step of one value's
        # product, 2^-7 |q k| / sqrt(D), in a capped score
        K = np.abs(final.values("k")[s]).max()
        ds = ds + 2.0 ** 24 * 2.0 ** -7 * np.abs(qf).max() * K / np.sqrt(D)
        _close(got[-1][s], o, mags, ds, n, vmax)


# ---------------------------------------------- every way a call is cut up

def _bulk_cache(rng, S, H, ctx, D):
    """Any codes but NaN's, for caches too large to be encoded here."""
    c = kv.Cache(S, H, ctx, D)
    for codes, exps in ((c.k, c.ke), (c.v, c.ve)):
        codes[...] = rng.integers(0, 256, codes.shape, np.uint8)
        codes[(codes & 127) == 127] = 0x31
        exps[...] = kv.BIAS - 7 + rng.integers(-1, 2, exps.shape)
    return c


def _check_some(ref, qf, got, pos0, spans, seqs, **kw):
    docs = kw.pop("docs", None)
    for s in seqs:
        one = kv.Cache.__new__(kv.Cache)
        one.k, one.v, one.ke, one.ve = (x[s:s + 1] for x in (ref.k, ref.v, ref.ke, ref.ve))
        _check(one, qf[s:s + 1], got[s:s + 1], pos0, None if spans is None else spans[s:s + 1], **kw,
               **({} if docs is None else dict(docs=docs[s:s + 1])))


# blocks of 128 rows (512 work-groups of them: one block with empty rows, two, and in two
# shares of the keys, joined by a wave a row); blocks of 64 rows in many shares at every
# width, with enough rows for either join; one token with more than 64 tiles a share; one
# token of many sequences in two shares
@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0", [
    (64, 8, 8, 64, 40, 100), (32, 16, 8, 128, 75, 60), (64, 8, 8, 128, 17, 0), (32, 8, 8, 64, 20, 4300), (32, 8, 8, 128, 20, 4300),
    (1, 16, 16, 256, 140, 3000), (1, 8, 2, 256, 60, 2500), (1, 16, 16, 64, 140, 1500), (1, 16, 16, 128, 140, 1500),
    (1, 4, 1, 128, 20, 5000), (32, 8, 8, 128, 1, 4200), (32, 64, 8, 64, 1, 4200), (32, 8, 8, 256, 1, 4200)])
@pytest.mark.parametrize("kw", [{}, dict(window=1100, prefix=70, softcap=15.0), dict(span=True)])
def test_attention_routes(S, Hq, Hkv, D, T, pos0, kw):
    ms = _ms()
    rng = np.random.default_rng(S + T)
    kw = dict(kw)
    spans = [(max(0, pos0 - 97 * s), max(1, T - s)) for s in range(S)] if kw.pop("span", False) else None
    ref = _bulk_cache(rng, S, Hkv, -(-(pos0 + T) // 64) * 64, D)
    q, qf = _bf16(0.5 * rng.standard_normal((S, T, Hq, D)))
    got = _run(_cache(ref), q, T, Hq, pos0, ms.attn_opts(**kw) if kw else None,
               None if spans is None else _span(spans)).float().cpu().numpy()
    _check_some(ref, qf, got, pos0, spans, sorted({0, 1 % S, S // 2, S - 1}), **kw)


@pytest.mark.parametrize("S,Hq,Hkv,T", [(512, 1, 1, 17), (32, 8, 8, 1), (300, 2, 2, 40)])
def test_attention_documents_over_many_tiles(S, Hq, Hkv, T):
    """More than 64 tiles a share: one document over all of them, documents that leave whole chunks of tiles out, and a
    document at both ends of the context."""
    ms = _ms()
    rng = np.random.default_rng(S)
    pos0, D = 8500, 64
    ctx = -(-(pos0 + T) // 64) * 64
    ref = _bulk_cache(rng, S, Hkv, ctx, D)
    q, qf = _bf16(0.5 * rng.standard_normal((S, T, Hq, D)))
    docs = np.zeros((S, ctx), np.int32)
    docs[1] = np.arange(ctx) // 100
    docs[2, 200:8300] = 7
    docs[3, 30:8510] = np.arange(8480) // 4200 + 1
    docs[4, pos0:] = -1
    opts = ms.attn_opts(doc=torch.from_numpy(docs).cuda())
    got = _run(_cache(ref), q, T, Hq, pos0, opts).float().cpu().numpy()
    _check_some(ref, qf, got, pos0, None, [0, 1, 2, 3, 4, S - 1], docs=docs)
    assert not np.any(got[4])


def test_two_streams_and_replayed_graphs_do_not_meet():
    """Two caches, each its own stream, workspace and captured decode step, replayed in turn and at once with eager work
    between: every step equals the eager calls alone."""
    ms = _ms()
    rng = np.random.default_rng(5)
    S, Hq, Hkv, D, ctx, start, steps = 2, 8, 2, 128, 4096, 3000, 5
    desc = ms.rope_desc(D, 1e4)
    first = torch.from_numpy(rng.standard_normal((2, S, start, Hq + 2 * Hkv, D)).astype(np.float32)).cuda()
    toks = torch.from_numpy(rng.standard_normal((2, steps, S, 1, Hq + 2 * Hkv, D)).astype(np.float32)).cuda()

    class Run:
        def __init__(self, i):
            self.cache, self.span = ms.new_kv_cache_q(S, Hkv, D, ctx), _span([(start, 1)] * S)
            self.x, self.stream, self.graph = torch.zeros_like(toks[0, 0]), torch.cuda.Stream(), None
            self.q, self.out = (torch.zeros(S, 1, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
            self.ws = torch.empty(max(ms.ms_attention_q_workspace(self.cache, 1, Hq, ctx - 1), 16), dtype=torch.uint8, device="cuda")
            q = torch.empty(S, start, Hq, D, dtype=torch.bfloat16, device="cuda")
            ms.ms_rope_kv_q(self.cache, desc, first[i], start, Hq, 0, q)
            torch.cuda.synchronize()

        def calls(self):
            _steps(ms, self.cache, self.x, self.q, self.out, self.ws, desc, None, self.span, 1, Hq, ctx - 1, self.stream)

        def step(self, x):
            with torch.cuda.stream(self.stream):
                self.x.copy_(x)
                self.graph.replay() if self.graph else self.calls()
                got = self.out.clone()
                self.span[:, 0] += 1
            return got

    want = []
    for i in range(2):
        run = Run(i)
        want.append([run.step(toks[i, t]) for t in range(steps)])
        torch.cuda.synchronize()
    for captured in (False, True):
        runs = [Run(0), Run(1)]
        if captured:
            for r in runs:
                r.graph = torch.cuda.CUDAGraph()
                with torch.cuda.graph(r.graph, stream=r.stream):
                    r.calls()
        got = [[r.step(toks[i, t]) for i, r in enumerate(runs)] for t in range(steps)]
        torch.cuda.synchronize()
        for t in range(steps):
            for i in range(2):
                assert torch.equal(got[t][i], want[i][t]), (captured, t, i)


def test_decoder_over_the_8_bit_cache():
    """A two-layer decoder around the experts with kv_bits=8, a prompt and greedy tokens past two scales' blocks, stretched
    positions, a window and capped scores: every layer's codes and its attention against the oracle."""
    from decoder import Decoder
    from gpu_helpers import check_close
    from oracle import decoder as od
    from workload import top_bytes
    ms = _ms()
    shape, attn = synth.ModelShape("dec-tiny", 2, 256, 512, 8, 2, "bf16"), synth.TINY_ATTN
    Hq, Hkv, D, P, n_dec = attn.n_heads, attn.n_kv_heads, attn.head_dim, 126, 4
    kw = dict(softcap=20.0, window=90, prefix=2)
    f = kv.frequencies(D, attn.rope_base, 4.0, 64, 1.0, 8.0)
    with Decoder(shape, attn, seed=4, n_sets=2, max_tokens=P, max_ctx=140, budget_total=2 * 8 * shape.expert_bytes, kv_bits=8,
                 rope=ms.rope_desc(D, attn.rope_base, False, 4.0, 64, 1.0, 8.0), opts=ms.attn_opts(**kw)) as dec:
        dec.stack.configure(0.5, 2 * 4 * top_bytes(dec.stack.rig, 0.5))
        for l in range(2):
            dec.stack.rig.load_tops(l, [0, 1, 2, 3])
        ms.ms_sync(dec.ctx)
        x = torch.empty(P, shape.d_model, dtype=torch.bfloat16, device="cuda")
        x1 = torch.empty(1, shape.d_model, dtype=torch.bfloat16, device="cuda")
        dec.embed_ids(torch.from_numpy(synth.prompt_tokens(attn, 4, P)).cuda(), P, x)
        refs = [kv.Cache(1, Hkv, 192, D) for _ in range(2)]
        for step in range(1 + n_dec):
            T, pos0 = (P if step == 0 else 1), dec.pos
            cap = dec.step(x if step == 0 else x1, T, capture=(0, 1))
            torch.cuda.synchronize()
            for l in range(2):
                xin = cap[l]["x"].astype(np.float64)
                qf, of = dec.f32[l % dec.n_sets]
                qkv = (xin @ qf.astype(np.float64).T).reshape(T, Hq + 2 * Hkv, D)
                turned = np.stack([kv.rope(qkv[t, :Hq + Hkv], pos0 + t, D, f) for t in range(T)])
                refs[l].append(0, pos0, turned[:, Hq:], qkv[:, Hq + Hkv:])
                k, v, ke, ve = _host(dec.kvq[l])
                n = pos0 + T
                blocks = -(-n // 64)
                assert np.array_equal(ke[..., :blocks], refs[l].ke[..., :blocks])
                assert np.array_equal(ve[..., :blocks], refs[l].ve[..., :blocks])
                for got, want in ((k, refs[l].k), (v, refs[l].v)):
                    # a projection's fp32 error moves a value over the middle of two codes: by one code, and rarely
                    a, b = got[:, :, :n].astype(int), want[:, :, :n].astype(int)
                    assert np.abs(a - b)[(a & 127 > 0) & (b & 127 > 0)].max(initial=0) <= 1 and np.mean(a != b) < 1e-3
                ref = kv.Cache(1, Hkv, k.shape[2], D)
                ref.k, ref.v, ref.ke, ref.ve = k, v, ke, ve
                o = kv.attention(od.bf16_round(turned[:, :Hq]), ref.values("k")[0], ref.values("v")[0], pos0, **kw)[0]
                att = od.bf16_round(o.reshape(T, -1)) @ of.astype(np.float64).T
                check_close(cap[l]["h"], od.bf16_round(od.rmsnorm(xin + att)), "bf16", "step %d layer %d h" % (step, l))
            dec.embed_ids(dec.ids, 1, x1)
        assert dec.pos == P + n_dec


# ------------------------------------------------------------- probabilities

def _cancelling(rng, S, Hkv, ctx, D, pos0, cap=0.0):
    """Caches of one query's (all ones) exact products between 0 and -1 and, in every column, five values that cancel to
    about 2^-18 of their terms, at positions that every token sees."""
    one = kv.Cache(1, Hkv, ctx, D)
    one.k[0, :, 1:, 0] = kv.encode(-rng.random((Hkv, ctx - 1)) * np.sqrt(D))
    s = one.values("k")[0, :, :, 0] / np.sqrt(D)
    p = np.exp(cap * np.tanh(s / cap) if cap else s)
    for h in range(Hkv):
        for c in range(D):
            left = 0.0
            for i, at in enumerate(rng.choice(np.arange(1, pos0), 5, replace=False)):
                one.v[0, h, at, c] = kv.encode(256.0 if i == 0 else -left / p[h, at])
                left += p[h, at] * kv.TABLE[one.v[0, h, at, c]]
    ref = kv.Cache(S, Hkv, ctx, D)
    for name in ("k", "v", "ke", "ve"):
        getattr(ref, name)[...] = getattr(one, name)
    return ref


def _check_cancelling(S, Hq, Hkv, D, T, pos0, off, **kw):
    """off: a weight's error.  Beside it, the weights' parts below fp16's steps: 2^-25 of at least 2^6 for each of the five."""
    ref = _cancelling(np.random.default_rng(T + D), S, Hkv, -(-(pos0 + T) // 64) * 64, D, pos0, kw.get("softcap", 0.0))
    q, qf = _bf16(np.ones((S, T, Hq, D)))
    got = _run(_cache(ref), q, T, Hq, pos0, _ms().attn_opts(**kw) if kw else None).float().cpu().numpy()
    o, mags, _ = kv.attention(qf[0], ref.values("k")[0], ref.values("v")[0], pos0, **kw)
    assert np.median(np.abs(o) / mags) < 2.0 ** -15
    for s in (0, S // 2, S - 1):
        assert np.all(np.abs(got[s] - o) <= 2.0 ** -8 * np.abs(o) + off * mags + 5 * 2.0 ** -31 * 448)


# one token, a few tokens, row blocks of 64 and of 128, whole and in shares of the keys
CANCELLING = [(1, 8, 2, 128, 1, 200), (2, 4, 2, 64, 5, 1500), (1, 4, 1, 256, 3, 300), (1, 16, 8, 64, 90, 200),
              (1, 4, 2, 128, 40, 3000), (1, 4, 2, 256, 60, 200), (64, 8, 8, 64, 40, 100), (32, 16, 8, 128, 75, 130)]


@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0", CANCELLING)
def test_probabilities_keep_22_bits(S, Hq, Hkv, D, T, pos0):
    """A weight is off by 2^-22 as two fp16 parts, 2^-22 by the scale's three roundings, 2^-22 by the exponent's (below 8 in
    size) and 2^-23 by its exponential: less than 2^-20 with the sums'.  One fp16 number would leave up to 2^-11."""
    _check_cancelling(S, Hq, Hkv, D, T, pos0, 2.0 ** -20)


@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0", CANCELLING)
@pytest.mark.parametrize("cap", [2.0, 30.0, 128.0, 1000.0])
def test_capped_scores_are_as_exact_as_their_size(S, Hq, Hkv, D, T, pos0, cap):
    """Capped scores of up to 1 whatever the cap: five roundings of the score and its cap, 2^-21, and tanh to 2^-20 of
    itself, beside the 2^-20 of uncapped ones.  Steps of 2^-22 of a cap of 128 would be 2^-15."""
    _check_cancelling(S, Hq, Hkv, D, T, pos0, 2.0 ** -20 + 2.0 ** -20 + 2.0 ** -21, softcap=cap)


@pytest.mark.parametrize("S,Hq,Hkv,D,T,pos0", [(2, 4, 2, 64, 1, 700), (1, 8, 2, 128, 3, 1000), (1, 8, 2, 128, 150, 260),
                                               (1, 8, 1, 256, 100, 90), (64, 8, 8, 64, 40, 100)])
@pytest.mark.parametrize("cap", [0.0, 30.0, 1000.0])
def test_masked_keys_do_not_touch_the_others_roundings(S, Hq, Hkv, D, T, pos0, cap):
    """Keys outside of every window, small or of the largest codes beside visible ones of the same scales: the same results,
    bit by bit."""
    rng = np.random.default_rng(T)
    n = pos0 + T
    ref = kv.Cache(S, Hkv, -(-n // 64) * 64 + 64, D)
    ref.k[...] = kv.encode(rng.standard_normal(ref.k.shape))
    ref.v[...] = kv.encode(rng.standard_normal(ref.v.shape))
    q, _ = _bf16(rng.standard_normal((S, T, Hq, D)))
    opts = _ms().attn_opts(softcap=cap, window=30)
    want = _run(_cache(ref), q, T, Hq, pos0, opts)
    for far in (slice(0, pos0 - 29), slice(n, None)):
        ref.k[:, :, far] = np.where(rng.random(ref.k[:, :, far].shape) < 0.5, 0x7e, 0xfe)
        ref.v[:, :, far] = 0x7e
    assert torch.equal(_run(_cache(ref), q, T, Hq, pos0, opts), want)


# --------------------------------------------------------- turned positions

@pytest.mark.parametrize("Hq,Hkv,D,rot,inter,T,pos0", [(32, 8, 128, 128, False, 2048, 0), (16, 2, 256, 256, True, 3000, 70000),
                                                       (24, 8, 64, 36, False, 1700, 1000000)])
def test_queries_do_not_depend_on_how_a_call_is_cut(Hq, Hkv, D, rot, inter, T, pos0):
    """A prompt, in which work-groups take heads of all kinds, and its tokens one at a time: the same queries, bit by bit."""
    ms = _ms()
    gen = torch.Generator(device="cuda").manual_seed(T)
    ctx = -(-(pos0 + T) // 64) * 64
    cache, desc = ms.new_kv_cache_q(1, Hkv, D, ctx), ms.rope_desc(rot, 1e4, inter, 4.0, 8192, 1.0, 8.0, 1.1)
    x = torch.empty(1, T, Hq + 2 * Hkv, D, device="cuda").normal_(generator=gen)
    q, q1 = (torch.zeros(1, T, Hq, D, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    ms.ms_rope_kv_q(cache, desc, x, T, Hq, pos0, q)
    for t in range(T):
        ms.ms_rope_kv_q(cache, desc, x[:, t], 1, Hq, pos0 + t, q1[:, t])
    torch.cuda.synchronize()
    assert torch.equal(q, q1)


def _code_borders(x, pair):
    """Whether x (of a unit scale) lies so near to the middle of two codes that a turn's 2^-30 of its pair's size may decide:
    sine and cosine to 2^-33 and, at position 2^20, angles to 2^-32, on either side."""
    a = np.abs(x)
    step = np.exp2(np.floor(np.log2(np.maximum(a, 2.0 ** -6))) - 3)
    return np.abs(a / step - np.floor(a / step) - 0.5) * step <= 2.0 ** -30 * pair


# every width, layout and part of the head; one token, inside a block, several blocks
# (the table of angles at its largest: 256 turned values, 64 tokens); far positions
@pytest.mark.parametrize("D,rot,inter,T,pos0", [
    (64, 64, False, 1, 100), (64, 20, False, 70, 30), (64, 64, True, 130, 1 << 20), (128, 128, False, 200, 77),
    (128, 128, False, 64, (1 << 20) - 64), (128, 96, True, 1, 131000), (256, 256, False, 130, 0), (256, 256, True, 64, 64),
    (256, 128, False, 3, 1 << 20)])
@pytest.mark.parametrize("mscale", [1.0, 1.3])
def test_turned_keys_have_the_nearest_codes(D, rot, inter, T, pos0, mscale):
    """Keys whose first value of every pair turns to within an fp32 step of the middle of two codes."""
    ms = _ms()
    rng = np.random.default_rng(D + T)
    H, half = 2, rot // 2
    f = kv.frequencies(rot, 1e4, 4.0, 8192, 1.0, 8.0)
    i = np.arange(half)
    first, second = (2 * i, 2 * i + 1) if inter else (i, i + half)
    y = np.zeros((T, H, D))
    middle = (rng.integers(8, 16, (T, H, half)) + 0.5) * np.exp2(rng.integers(-6, 4, (T, H, half)))
    y[..., first] = middle * rng.choice([-1, 1], middle.shape)
    y[..., second] = rng.uniform(-440, 440, middle.shape)
    y[..., second[0]] = 400.0  # every block's scale is 1
    x = np.stack([kv.rope(y[t], -(pos0 + t), rot, f, inter, 1.0) for t in range(T)]) / mscale
    qkv = np.zeros((1, T, 3 * H, D), np.float32)
    qkv[0, :, H:2 * H] = x
    x = qkv[0, :, H:2 * H].astype(np.float64)
    turned = np.stack([kv.rope(x[t], pos0 + t, rot, f, inter, mscale) for t in range(T)])
    ctx = -(-(pos0 + T) // 64) * 64
    cache = ms.new_kv_cache_q(1, H, D, ctx)
    cache.tensors[2].fill_(kv.BIAS - 20)
    q = torch.empty(1, T, H, D, dtype=torch.bfloat16, device="cuda")
    ms.ms_rope_kv_q(cache, ms.rope_desc(rot, 1e4, inter, 4.0, 8192, 1.0, 8.0, mscale), torch.from_numpy(qkv).cuda(), T, H, pos0, q)
    torch.cuda.synchronize()
    assert bool((cache.tensors[2][:, :, pos0 // 64:] == kv.BIAS).all())
    got = cache.tensors[0][0, :, pos0:pos0 + T].cpu().numpy().transpose(1, 0, 2)
    pair = np.zeros((T, H, D))
    pair[..., first] = pair[..., second] = np.hypot(turned[..., first], turned[..., second])
    near = _code_borders(turned, pair)
    assert np.mean(near[..., first]) < 0.3
    assert np.array_equal(kv.TABLE[got][~near], kv.TABLE[kv.encode(turned)][~near])


# work-groups of two and three heads, head counts that their number does not divide, groups
# of queries alone, with keys and with both of keys and values; appends from inside a
# block on, and sequences of their own spans
@pytest.mark.parametrize("S,Hq,Hkv,D,rot,inter,T,pos0,spans", [
    (1, 24, 8, 64, 64, False, 1700, 37, None), (1, 16, 16, 64, 32, True, 2100, 0, None), (4, 15, 3, 128, 128, False, 1000, 60, None),
    (8, 4, 2, 256, 256, False, 1020, 90, None), (3, 6, 2, 128, 44, False, 2500, 100, [(100, 2500), (63, 1111), (0, 2499)])])
def test_append_of_many_heads_a_work_group(S, Hq, Hkv, D, rot, inter, T, pos0, spans):
    ms = _ms()
    rng = np.random.default_rng(T)
    ctx = -(-(pos0 + T) // 64) * 64 + 64
    ref = _random_cache(rng, S, Hkv, ctx, D)
    cache = _cache(ref)
    qkv = rng.standard_normal((S, T, Hq + 2 * Hkv, D)).astype(np.float32)
    qkv *= np.exp2(rng.integers(-3, 4, (S, T, Hq + 2 * Hkv, 1))).astype(np.float32)
    q = torch.full((S, T, Hq, D), -7.0, dtype=torch.bfloat16, device="cuda")
    ms.ms_rope_kv_q(cache, ms.rope_desc(rot, 1e4, inter, 4.0, 8192, 1.0, 8.0, 1.25), torch.from_numpy(qkv).cuda(), T, Hq, pos0, q,
                    None if spans is None else _span(spans))
    torch.cuda.synchronize()
    f = kv.frequencies(rot, 1e4, 4.0, 8192, 1.0, 8.0)
    k, v, ke, ve = _host(cache)
    qg = q.float().cpu().numpy()
    for s in range(S):
        start, n = (pos0, T) if spans is None else spans[s]
        x = qkv[s, :n].astype(np.float64)
        turned = np.stack([kv.rope(x[t, :Hq + Hkv], start + t, rot, f, inter, 1.25) for t in range(n)])
        err = 2.0 ** -21 * 1.25 * np.abs(x[:, :Hq]).max(axis=-1, keepdims=True)
        assert np.all(np.abs(qg[s, :n] - turned[:, :Hq]) <= 2.0 ** -8 * np.abs(turned[:, :Hq]) + err)
        assert np.all(qg[s, n:] == -7.0)
        ref.append(s, start, turned[:, Hq:], x[:, Hq + Hkv:])
        assert np.array_equal(ke[s], ref.ke[s]) and np.array_equal(ve[s], ref.ve[s])
        assert np.array_equal(v[s], ref.v[s])
        differ = k[s] != ref.k[s]
        if differ.any():  # only values next to the middle of two codes
            h, p, c = np.nonzero(differ)
            unit = np.exp2(ke[s, h, p // 64].astype(float) - kv.BIAS)
            assert np.all((p >= start) & (p < start + n))
            t = turned[p - start, Hq + h, c] / unit
            assert np.all(_code_borders(t, 2 * np.abs(x[p - start, Hq + h]).max(axis=-1) / unit))


@pytest.mark.parametrize("T,pos0", [(1, 300), (40, 100)])
@pytest.mark.parametrize("scale", [1e-40, 2e38])
@pytest.mark.parametrize("size", [0.0, 2.0 ** -124])
def test_scales_at_the_ends_of_fp32(T, pos0, scale, size):
    """The largest scale is as good as any for queries that are small enough, zeros among them; so is one below the least
    normal number."""
    rng = np.random.default_rng(T)
    ref = _random_cache(rng, 1, 2, 192 if T == 40 else 320, 64)
    q, qf = _bf16(size * rng.integers(-2, 3, (1, T, 4, 64)))
    got = _run(_cache(ref), q, T, 4, pos0, _ms().attn_opts(scale=scale)).float().cpu().numpy()
    _check(ref, qf, got, pos0, None, scale=scale)


# ------------------------------------------------------------ the decoder

def test_decoder_steps_allocate_no_device_memory():
    """Its workspace is there from the start and stays: prompts of odd sizes, then tokens past many shares of the context, on
    a stream that is not the current one."""
    from decoder import Decoder
    from workload import top_bytes
    ms = _ms()
    shape, attn = synth.ModelShape("dec-tiny", 2, 256, 512, 8, 2, "bf16"), synth.TINY_ATTN
    with Decoder(shape, attn, seed=4, n_sets=2, max_tokens=400, max_ctx=3000, budget_total=2 * 8 * shape.expert_bytes,
                 keep_f32=False, kv_bits=8) as dec:
        work = dec.work
        assert work.numel() >= max(ms.ms_attention_q_workspace(dec.kvq[0], T, attn.n_heads, 3000 - T) for T in (1, 7, 40, 399))
        assert work.numel() > 0
        dec.stack.configure(0.5, 2 * 4 * top_bytes(dec.stack.rig, 0.5))
        stream = torch.cuda.Stream()
        x = torch.randn(400, shape.d_model, device="cuda").to(torch.bfloat16)
        torch.cuda.synchronize()
        dec.step(x, 400, stream=stream)
        before = torch.cuda.memory_stats()["allocation.all.allocated"]
        for T in [1] * 70 + [399, 40, 7] + [1] * 70 + [400] * 4 + [1] * 9:
            dec.step(x, T, stream=stream)
        stream.synchronize()
        assert torch.cuda.memory_stats()["allocation.all.allocated"] == before and dec.work is work
