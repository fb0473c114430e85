"""Without a GPU: the oracles of the dense path in 8 bits and of the drawn token,
and the calls that the library and its binding refuse."""
import numpy as np
import pytest

from oracle import blocks8 as b8
from oracle import sample as osm

torch = pytest.importorskip("torch")


def _ms():
    from paper_2509_08342_amd import moesplit
    return moesplit


# ------------------------------------------------------------------ oracles

@pytest.mark.parametrize("block_rows", [1, 128])
def test_blocks_hold_their_values(block_rows):
    """Within half a step of the code, and of the least code times the scale; scales the least that hold the block."""
    rng = np.random.default_rng(0)
    x = rng.standard_normal((150, 300)) * np.exp2(rng.integers(-20, 20, (150, 1)))
    c, e = b8.quantize(x, block_rows)
    assert c.shape == x.shape and e.shape == (-(-150 // block_rows), 3)
    unit = b8.spread(e.astype(int) - b8.BIAS, 150, 300, block_rows)
    assert np.all(np.abs(b8.values(c, e, block_rows) - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10 * unit))
    top = np.pad(np.abs(x), ((0, -150 % block_rows), (0, 84))).reshape(-1, block_rows, 3, 128).max(axis=(1, 3))
    s = np.exp2(e.astype(float) - b8.BIAS)
    assert np.all(top <= 448 * s) and np.all(top > 224 * s)


def test_values_at_the_ends():
    x = np.zeros((1, 128))
    x[0, :5] = 448, -449, np.inf, np.nan, 1e-3
    c, e = b8.quantize(x)
    assert e[0, 0] == b8.BIAS + 1 and list(c[0, :4]) == [0x76, 0xf6, 0x7f, 0x7f]
    assert b8.exponents(np.full((1, 1), 1e30), 1)[0, 0] == b8.EMAX and b8.exponents(np.zeros((1, 1)), 1)[0, 0] == b8.EMIN


def test_norm_and_product():
    rng = np.random.default_rng(1)
    h, y, g = rng.standard_normal((3, 20)), rng.standard_normal((3, 20)), rng.standard_normal(20)
    x, v = b8.residual_norm(h, y, g, 0.0)
    assert np.allclose(x, h + y) and np.allclose(np.mean((v / g) ** 2, axis=1), 1.0)
    p, mags = b8.dense(h, y, np.ones((3, 3)))
    assert np.allclose(p, h @ y.T + 1) and np.all(mags >= np.abs(p))


def test_draws():
    """The shares of a small row, by hand; filters keep prefixes of the descending order, ties by index."""
    l = np.log([1.0, 4.0, 2.0, 2.0, 0.5])
    grid = (np.arange(950) + 0.5) / 950
    got = np.bincount([osm.draw(l, u)[0] for u in grid], minlength=5)
    assert list(got) == [100, 400, 200, 200, 50]
    assert [osm.kept(l, top_k=k)[2] for k in (0, 1, 3, 5, 9)] == [5, 1, 3, 5, 5]
    assert list(osm.kept(l)[0]) == [1, 2, 3, 0, 4]
    assert [osm.kept(l, top_p=p)[2] for p in (0.0, 0.4, 0.43, 0.64, 0.99, 1.0)] == [1, 1, 2, 3, 5, 5]
    assert osm.kept(l, top_k=3, top_p=0.7)[2] == 2 and osm.kept(l, min_p=0.3)[2] == 3 and osm.kept(l, min_p=1.0)[2] == 1
    assert osm.draw(l, 0.999, temperature=0.0)[:2] == (1, 1.0)
    assert osm.draw([np.nan, -np.inf], 0.5)[0] == 0 and osm.draw([0.0, np.inf, np.inf], 0.6)[0] == 2


# ----------------------------------------------------------------- refusals

def _status(call, *args, **kw):
    ms = _ms()
    with pytest.raises(ms.MoeSplitError) as e:
        call(*args, **kw)
    return e.value.status


def _z(*shape, dtype=torch.uint8, shift=0):
    n = int(np.prod(shape))
    return torch.zeros(n + 64, dtype=dtype)[shift:shift + n].view(shape)


def test_quant_refusals():
    ms = _ms()
    x, c, e = _z(4, 256, dtype=torch.float32), _z(4, 256), _z(4, 2)
    assert _status(ms.ms_quant_q, x, 4, 256, 2, c, e) == ms.MS_E_INVALID
    assert _status(ms.ms_quant_q, x, 4, 256, 0, c, e) == ms.MS_E_INVALID
    assert _status(ms.ms_quant_q, x, -1, 256, 1, c, e) == ms.MS_E_INVALID
    assert _status(ms.ms_quant_q, x, 4, 0, 1, c, e) == ms.MS_E_INVALID
    assert _status(ms.ms_quant_q, x, 4, 200, 1, c, e) == ms.MS_E_UNSUPPORTED
    assert _status(ms.ms_quant_q, _z(1, 16400, dtype=torch.float32), 1, 16400, 1, _z(1, 16400), _z(1, 129)) == ms.MS_E_UNSUPPORTED
    assert _status(ms.ms_quant_q, _z(4, 256, dtype=torch.float32, shift=1), 4, 256, 1, c, e) == ms.MS_E_INVALID
    assert _status(ms.ms_quant_q, x, 4, 256, 1, _z(4, 256, shift=8), e) == ms.MS_E_INVALID
    assert ms.lib.ms_quant_q(None, ms.MS_F32, 4, 256, 1, c.data_ptr(), e.data_ptr(), None) == ms.MS_E_INVALID
    assert ms.lib.ms_quant_q(x.data_ptr(), 2, 4, 256, 1, c.data_ptr(), e.data_ptr(), None) == ms.MS_E_INVALID
    assert _status(ms.ms_quant_q, x, 4, 256, 1, x.view(torch.uint8).view(-1)[:1024], e) == ms.MS_E_INVALID
    ms.ms_quant_q(_z(0, 256, dtype=torch.float32), 0, 256, 128, _z(0, 256), _z(0, 2))  # nothing to do
    for bad in ((x.half(), c, e), (x[:3], c, e), (x, c[:3], e), (x, c, e[:3]), (x, c.float(), e), (x.t(), c, e)):
        with pytest.raises(ValueError):
            ms.ms_quant_q(bad[0], 4, 256, 1, *bad[1:])


def test_norm_refusals():
    ms = _ms()
    T, d = 3, 256
    bf = lambda **k: _z(T, d, dtype=torch.bfloat16, **k)  # noqa: E731
    h, y, out, c, e = bf(), _z(T, d, dtype=torch.float32), bf(), _z(T, d), _z(T, 2)
    n = ms.ms_residual_norm_q
    assert _status(n, h, y, None, 1e-6, T, d) == ms.MS_E_INVALID  # no output
    assert _status(n, h, y, None, 1e-6, T, d, codes=c) == ms.MS_E_INVALID
    assert _status(n, h, y, None, 1e-6, T, d, out=out, exps=e) == ms.MS_E_INVALID
    assert _status(n, h, y, None, -1e-6, T, d, out=out) == ms.MS_E_INVALID
    assert _status(n, h, y, None, float("nan"), T, d, out=out) == ms.MS_E_INVALID
    assert _status(n, h, y, None, 1e-6, -1, d, out=out) == ms.MS_E_INVALID
    assert _status(n, h, y, None, 1e-6, 1, 100, out=out) == ms.MS_E_UNSUPPORTED
    assert _status(n, bf(shift=1), y, None, 1e-6, T, d, out=out) == ms.MS_E_INVALID
    assert _status(n, h, y, _z(d, dtype=torch.bfloat16, shift=4), 1e-6, T, d, out=out) == ms.MS_E_INVALID
    assert _status(n, h, y, None, 1e-6, T, d, sum_out=out, out=out) == ms.MS_E_INVALID
    both = torch.zeros(2 * T * d, dtype=torch.bfloat16)
    assert _status(n, both[:T * d], y, None, 1e-6, T, d, out=both[d:d + T * d]) == ms.MS_E_INVALID  # another row's values
    assert _status(n, h, y, None, 1e-6, T, d, out=y.view(torch.bfloat16).view(-1)[:T * d]) == ms.MS_E_INVALID
    assert _status(n, h, y, None, 1e-6, T, d, codes=h.view(torch.uint8).view(-1)[:T * d], exps=e) == ms.MS_E_INVALID
    assert ms.lib.ms_residual_norm_q(1 << 44, None, ms.MS_F32, None, 1e-6, 1 << 24, 16, None, 1 << 45, None, None,
                                     None) == ms.MS_E_UNSUPPORTED
    ms.ms_residual_norm_q(_z(0, d, dtype=torch.bfloat16), None, None, 1e-6, 0, d, out=_z(0, d, dtype=torch.bfloat16))
    for bad in (dict(h=h[:2]), dict(h=h.float()), dict(y=y.half()), dict(y=y[:2]), dict(weight=out[0, :100]),
                dict(out=out[:1]), dict(codes=c[:2], exps=e), dict(codes=c, exps=e[:2])):
        a = dict(h=h, y=y, weight=None, out=out)
        a.update(bad)
        with pytest.raises(ValueError):
            n(a.pop("h"), a.pop("y"), a.pop("weight"), 1e-6, T, d, **a)


def test_dense_refusals():
    ms = _ms()
    T, n_in, n_out = 3, 256, 130
    x, xe, w, we = _z(T, n_in), _z(T, 2), _z(n_out, n_in), _z(2, 2)
    y = _z(T, n_out, dtype=torch.float32)
    f = ms.ms_dense_q
    assert _status(f, x, xe, w, we, T, n_in, 0, y) == ms.MS_E_INVALID
    assert _status(f, x, xe, w, we, -1, n_in, n_out, y) == ms.MS_E_INVALID
    assert _status(f, x, xe, w, we, 1, 0, n_out, y) == ms.MS_E_INVALID
    assert _status(f, x, xe, w, we, T, 250, n_out, y) == ms.MS_E_UNSUPPORTED
    assert _status(f, _z(1, 16400), _z(1, 129), _z(1, 16400), _z(1, 129), 1, 16400, 1, y) == ms.MS_E_UNSUPPORTED
    assert _status(f, _z(T, n_in, shift=4), xe, w, we, T, n_in, n_out, y) == ms.MS_E_INVALID
    assert _status(f, x, xe, _z(n_out, n_in, shift=8), we, T, n_in, n_out, y) == ms.MS_E_INVALID
    p = [t.data_ptr() for t in (x, xe, w, we)]
    assert ms.lib.ms_dense_q(p[0], None, p[2], p[3], T, n_in, n_out, y.data_ptr(), ms.MS_F32, None, None) == ms.MS_E_INVALID
    assert ms.lib.ms_dense_q(*p, T, n_in, n_out, y.data_ptr(), 5, None, None) == ms.MS_E_INVALID
    wide = torch.zeros(2 * T * n_out)
    assert _status(f, x, xe, w, we, T, n_in, n_out, wide[:T * n_out], add=wide[1:1 + T * n_out]) == ms.MS_E_INVALID
    room = torch.zeros(T * n_out * 4 + 64, dtype=torch.uint8)  # results over the tokens' codes
    assert _status(f, room[:T * n_in], xe, w, we, T, n_in, n_out, room[:T * n_out * 4].view(torch.float32)) == ms.MS_E_INVALID
    p = [t.data_ptr() for t in (x, xe, w, we)]  # more outputs, and rows, than a launch may have
    assert ms.lib.ms_dense_q(*p, 1, 16, (1 << 25) + 1, 1 << 44, ms.MS_F32, None, None) == ms.MS_E_UNSUPPORTED
    f(_z(0, n_in), _z(0, 2), w, we, 0, n_in, n_out, _z(0, n_out, dtype=torch.float32))
    for bad in (dict(x=x[:2]), dict(xe=xe[:2]), dict(w=w[:100]), dict(we=we[:1]), dict(y=y[:2]), dict(y=y.half()),
                dict(add=y[:2]), dict(add=y.bfloat16()), dict(w=w.t())):
        a = dict(x=x, xe=xe, w=w, we=we, y=y, add=None)
        a.update(bad)
        with pytest.raises(ValueError):
            f(a["x"], a["xe"], a["w"], a["we"], T, n_in, n_out, a["y"], add=a["add"])


def test_sample_refusals():
    ms = _ms()
    l, u, i = _z(2, 50, dtype=torch.float32), _z(2, dtype=torch.float32), _z(2, dtype=torch.int32)
    assert _status(ms.ms_sample, l, -1, 50, None, u, i) == ms.MS_E_INVALID
    assert _status(ms.ms_sample, l, 2, 0, None, u, i) == ms.MS_E_INVALID
    assert _status(ms.ms_sample_workspace, 1, 1 << 19) == ms.MS_E_UNSUPPORTED
    assert _status(ms.ms_sample_workspace, 1, -3) == ms.MS_E_INVALID
    assert ms.lib.ms_sample_workspace(1, 5, None) == ms.MS_E_INVALID
    assert ms.lib.ms_sample(l.data_ptr(), 2, 50, None, None, i.data_ptr(), None, None, 0, None) == ms.MS_E_INVALID
    ms.ms_sample(_z(0, 50, dtype=torch.float32), 0, 50, None, _z(0, dtype=torch.float32), _z(0, dtype=torch.int32))
    for T, n in ((1, 32000), (1, 524287), (3, 150000), (64, 100000)):  # a workspace too small, or not aligned
        need = ms.ms_sample_workspace(T, n)
        if need:
            big = [_z(T, n, dtype=torch.float32), _z(T, dtype=torch.float32), _z(T, dtype=torch.int32)]
            for ws in (None, _z(need - 1), _z(need, shift=8)):
                assert _status(ms.ms_sample, big[0], T, n, None, big[1], big[2], None, ws) == ms.MS_E_INVALID
    opts, prob = ms.sample_opts(u, i, None, u), _z(2, dtype=torch.float32)
    for idx, out in ((l.view(-1)[98:].view(torch.int32), prob), (u.view(torch.int32), None), (i, None), (i, u), (prob.view(torch.int32), prob)):
        assert _status(ms.ms_sample, l, 2, 50, opts, u, idx, out) == ms.MS_E_INVALID  # over the logits, settings, each other
    ws = _z(ms.ms_sample_workspace(1, 200000))
    assert _status(ms.ms_sample, _z(1, 200000, dtype=torch.float32), 1, 200000, None, u[:1], ws[:4].view(torch.int32), None, ws) == ms.MS_E_INVALID
    with pytest.raises(ValueError):
        ms.sample_opts(top_k=u)
    with pytest.raises(ValueError):
        ms.sample_opts(temperature=i)
    for shapes in ((u, u[:1]), (u.view(1, 2), u.view(1, 2)), (u[0], None)):
        with pytest.raises(ValueError):
            ms.sample_opts(temperature=shapes[0], top_p=shapes[1])
    with pytest.raises(ValueError):
        ms.ms_sample(l, 2, 50, ms.sample_opts(temperature=u[:1]), u, i)
    for bad in ((l[:1], u, i), (l, u[:1], i), (l, u, i[:1]), (l.half(), u, i)):
        with pytest.raises(ValueError):
            ms.ms_sample(bad[0], 2, 50, None, *bad[1:])


def test_sample_workspace_over_inputs():
    """A workspace is written before the last look at logits, numbers and settings: it overlaps none of them."""
    ms = _ms()
    T, n = 1, 200000
    need = ms.ms_sample_workspace(T, n)
    assert need > 0
    room = torch.zeros(4 * n + need + 64, dtype=torch.uint8)
    u, i, idx = torch.zeros(T), torch.zeros(T, dtype=torch.int32), torch.zeros(T, dtype=torch.int32)
    logits = torch.zeros(T, n)
    over = [room[:need], room[4 * n - 16:4 * n - 16 + need]]  # the first logits, and the last four
    for ws in over:
        assert _status(ms.ms_sample, room[:4 * n].view(torch.float32), T, n, None, u, idx, None, ws) == ms.MS_E_INVALID
    ws = room[:need]
    at = lambda t: room[need - 4:need].view(t)  # noqa: E731  (in the workspace's last bytes)
    assert _status(ms.ms_sample, logits, T, n, None, at(torch.float32), idx, None, ws) == ms.MS_E_INVALID
    for name, t in (("temperature", torch.float32), ("top_k", torch.int32), ("top_p", torch.float32), ("min_p", torch.float32)):
        assert _status(ms.ms_sample, logits, T, n, ms.sample_opts(**{name: at(t)}), u, idx, None, ws) == ms.MS_E_INVALID
    # unused, it may lie anywhere
    ms.ms_sample(torch.zeros(0, 50), 0, 50, None, u[:0], i[:0], None, room[:16])


def test_tensors_of_another_type_are_refused():
    """Every tensor of the calls as a type of the same size that holds other values."""
    ms = _ms()
    T, d = 3, 256
    z = lambda *shape, dtype: torch.zeros(*shape, dtype=dtype)  # noqa: E731
    bf, f32, u8 = torch.bfloat16, torch.float32, torch.uint8
    ok = dict(h=z(T, d, dtype=bf), y=z(T, d, dtype=bf), weight=z(d, dtype=bf), sum_out=z(T, d, dtype=bf), out=z(T, d, dtype=bf),
              codes=z(T, d, dtype=u8), exps=z(T, 2, dtype=u8))

    def norm(**a):
        a = {**ok, **a}
        ms.ms_residual_norm_q(a.pop("h"), a.pop("y"), a.pop("weight"), 1e-6, T, d, **a)
    for name in ("h", "y", "weight", "sum_out", "out"):
        for other in (torch.float16, torch.int16):
            with pytest.raises(ValueError):
                norm(**{name: ok[name].view(other)})
    for name, others in (("codes", (torch.bool, torch.float8_e5m2, torch.float8_e4m3fnuz)), ("exps", (torch.int8, torch.bool, torch.float8_e4m3fn))):
        for other in others:
            with pytest.raises(ValueError):
                norm(**{name: ok[name].view(other)})
            with pytest.raises(ValueError):
                ms.ms_quant_q(ok["h"], T, d, 1, **{**{k: ok[k] for k in ("codes", "exps")}, name: ok[name].view(other)})
    x, xe, y = ok["codes"], ok["exps"], z(T, T, dtype=f32)
    w, we = z(T, d, dtype=u8), z(1, 2, dtype=u8)
    for bad in ((x.view(torch.float8_e5m2), xe, w, we), (x, xe.view(torch.int8), w, we), (x, xe, w.view(torch.bool), we),
                (x, xe, w, we.view(torch.float8_e5m2))):
        with pytest.raises(ValueError):
            ms.ms_dense_q(*bad, T, d, T, y)
    n = 50
    ok = dict(logits=z(T, n, dtype=f32), u=z(T, dtype=f32), idx=z(T, dtype=torch.int32), prob=z(T, dtype=f32))
    for name, other in (("logits", torch.int32), ("u", torch.int32), ("idx", f32), ("idx", torch.uint32), ("prob", torch.int32)):
        a = {**ok, name: ok[name].view(other)}
        with pytest.raises(ValueError):
            ms.ms_sample(a["logits"], T, n, None, a["u"], a["idx"], a["prob"])
    # nothing to do, of every type that there is
    for c, e in ((u8, u8), (torch.int8, u8), (torch.float8_e4m3fn, torch.float8_e8m0fnu)):
        ms.ms_quant_q(z(0, d, dtype=bf), 0, d, 1, z(0, d, dtype=c), z(0, 2, dtype=e))


def test_cache_tensors_of_another_type_are_refused():
    ms = _ms()
    T, Hq, Hkv, D = 3, 4, 2, 64
    c = ms.new_kv_cache_q(1, Hkv, D, 64, device="cpu")
    rope = ms.rope_desc(D, 1e4)
    half, qkv = torch.zeros(T * Hq * D, dtype=torch.float16), torch.zeros(T * (Hq + 2 * Hkv) * D)
    q = torch.zeros(T * Hq * D, dtype=torch.bfloat16)
    for call in (lambda: ms.ms_rope_kv_q(c, rope, qkv.view(torch.int32), T, Hq, 0, q), lambda: ms.ms_rope_kv_q(c, rope, qkv, T, Hq, 0, half),
                 lambda: ms.ms_attention_q(c, half, T, Hq, 0, q), lambda: ms.ms_attention_q(c, q, T, Hq, 0, half),
                 lambda: ms.ms_kv_read_q(c, 0, T, half, q), lambda: ms.ms_kv_read_q(c, 0, T, q, half)):
        with pytest.raises(ValueError):
            call()


def test_every_launch_asks_for_lds():
    """A work-group without LDS may land on the compute units that copies of experts hold, and waits behind their reads: a
    kernel has LDS in each of its forms, or is launched with some."""
    import os
    import re
    import paper_2509_08342_amd
    has_lds = {"quant_blocks_kernel", "dense_q_tile_kernel", "dense_q_pair_kernel", "dense_q_few_kernel", "sample_kernel",
               "sample_range_kernel", "sample_weigh_kernel", "sample_gather_kernel", "sample_choose_kernel"}
    launched = set()
    for name in ("blocks8.hip", "sample.hip"):
        text = open(os.path.join(os.path.dirname(paper_2509_08342_amd.__file__), "csrc", name)).read().replace("\\\n", " ")
        for m in re.finditer(r"hipLaunchKernelGGL\(", text):
            args, depth, at = [""], 0, m.end()
            while depth >= 0 and len(args) < 5:
                c = text[at]
                depth += (c == "(") - (c == ")")
                args = args + [""] if c == "," and depth == 0 else args[:-1] + [args[-1] + c]
                at += 1
            kernel = re.search(r"\w+_kernel", args[0]).group()
            launched.add(kernel)
            if args[3].strip() != "msk::kGuardLds":
                assert args[3].strip() == "0" and kernel in has_lds, (name, args[:4])
                body = text[text.index("void %s(" % kernel):]
                assert "__shared__" in body[:body.index("\n}\n")], kernel
    assert has_lds < launched and len(launched) == len(has_lds) + 2


def test_calls_larger_than_a_launch_are_refused():
    """One past each limit that the header states (addresses far apart, never read)."""
    ms = _ms()
    a, b, c, d, e = (k << 50 for k in range(1, 6))
    quant = lambda rows, n, R: ms.lib.ms_quant_q(a, ms.MS_BF16, rows, n, R, b, c, None)  # noqa: E731
    assert quant(2 ** 28 - 15, 16, 1) == ms.MS_E_UNSUPPORTED and quant(2 ** 21, 16384, 1) == ms.MS_E_UNSUPPORTED
    assert quant(2 ** 31 - 1, 16, 128) == ms.MS_E_UNSUPPORTED and quant(2 ** 24, 16384, 128) == ms.MS_E_UNSUPPORTED
    assert ms.lib.ms_residual_norm_q(a, None, ms.MS_F32, None, 1e-6, 2 ** 24, 16, b, None, None, None, None) == ms.MS_E_UNSUPPORTED
    dense = lambda T, n_in, n_out: ms.lib.ms_dense_q(a, b, c, d, T, n_in, n_out, e, ms.MS_F32, None, None)  # noqa: E731
    assert dense(1, 16, 2 ** 25 + 1) == ms.MS_E_UNSUPPORTED
    # 2^22 blocks of 128 x 128 of rows that only such tiles take; of shorter ones as many of the largest tiles
    assert dense(2 ** 18, 16384, 2 ** 18) == ms.MS_E_UNSUPPORTED and dense(2 ** 26, 128, 128 * 192) == ms.MS_E_UNSUPPORTED
    assert ms.lib.ms_sample(a, 2 ** 22, 50, None, b, c, d, None, 0, None) == ms.MS_E_UNSUPPORTED
