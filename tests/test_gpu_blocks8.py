"""GPU parity of the dense path in 8 bits against its oracle: matrices of codes
made from rows, the residual's addition and norm with outputs in bf16 and in
codes, and products in every kernel."""
import numpy as np
import pytest

import synth
from oracle import blocks8 as b8

pytestmark = pytest.mark.gpu

torch = pytest.importorskip("torch")


def _ms():
    from paper_2509_08342_amd import moesplit
    return moesplit


def _bf16(a):
    from workload import to_device
    raw, f = synth.storage(np.ascontiguousarray(a, np.float32), "bf16")
    return to_device(raw, "bf16"), f.astype(np.float64)


def _input(a, dtype):
    """(device tensor, exact fp64 values)"""
    if dtype == "bf16":
        return _bf16(a)
    a = np.ascontiguousarray(a, np.float32)
    return torch.from_numpy(a).cuda(), a.astype(np.float64)


def _guarded(shape, fill, dtype, gap=64):
    """A tensor of `shape` between guards of `gap` values, and a check that they are as they were."""
    n = int(np.prod(shape))
    buf = torch.full((n + 2 * gap,), fill, dtype=dtype, device="cuda")

    def check():
        ends = torch.cat((buf[:gap], buf[gap + n:])).float().cpu().numpy()
        assert np.all(ends == float(torch.full((1,), fill, dtype=dtype).float())), "written past the ends"
    return buf[gap:gap + n].view(shape), check


def _same_codes(got, want):
    """Codes alike as numbers: every code of NaN counts as one."""
    a, b = b8.TABLE[got], b8.TABLE[want]
    bad = ~((a == b) | (np.isnan(a) & np.isnan(b)))
    assert not bad.any(), (np.argwhere(bad)[:4].tolist(), a[bad][:4], b[bad][:4])


# -------------------------------------------------------------------- quant

# one value's row to many; widths below, at and past a block and its multiples; rows below, at and past 128
@pytest.mark.parametrize("rows,n", [(1, 16), (1, 128), (3, 144), (127, 112), (128, 256), (129, 2000), (300, 48), (1, 16384),
                                    (61, 4096)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("block_rows", [1, 128])
def test_quant(rows, n, dtype, block_rows):
    ms = _ms()
    rng = np.random.default_rng(rows + n)
    a = rng.standard_normal((rows, n)) * np.exp2(rng.integers(-12, 12, (rows, 1)))
    a[rng.random((rows, n)) < 0.01] *= 300.0
    x, f = _input(a, dtype)
    codes, check = _guarded((rows, n), 0x55, torch.uint8)
    exps, check_exps = _guarded((-(-rows // block_rows), -(-n // 128)), 0x55, torch.uint8, gap=7)
    ms.ms_quant_q(x, rows, n, block_rows, codes, exps, torch.cuda.current_stream())
    torch.cuda.synchronize()
    want, want_exps = b8.quantize(f, block_rows)
    assert np.array_equal(exps.cpu().numpy(), want_exps)
    _same_codes(codes.cpu().numpy(), want)
    check()
    check_exps()


@pytest.mark.parametrize("block_rows", [1, 128])
def test_quant_of_extreme_values(block_rows):
    """Borders of exponents and ties of codes, zeros, subnormals, infinities and NaN, magnitudes past both ends."""
    ms = _ms()
    a = np.zeros((9, 128), np.float32)
    a[1, :3] = 448.0, -448.0, 0.4375
    a[2, :3] = np.nextafter(np.float32(448), np.float32(500)), 1.0, -3.0
    a[3] = np.linspace(-17, 17, 128)
    a[3, 5], a[3, 6], a[3, 7] = np.inf, -np.inf, np.nan
    a[4] = 1e-16 * np.linspace(-1, 1, 128)
    a[5, :4] = 3e38, -1e30, 1.0, np.inf
    a[6, :4] = 1e-45, 1e-40, -1e-39, 0.0
    a[7, :6] = 448, 17, 18, 19, 0.0009765625, 0.00048828125  # ties of codes and of the smallest
    a[8] = np.nan
    for shape in ([(9, 128)] if block_rows == 128 else [(9, 128), (72, 16)]):
        f = a.reshape(shape)
        codes = torch.zeros(shape, dtype=torch.uint8, device="cuda")
        exps = torch.zeros(-(-shape[0] // block_rows), 1, dtype=torch.uint8, device="cuda")
        ms.ms_quant_q(torch.from_numpy(f.copy()).cuda(), *shape, block_rows, codes, exps)
        torch.cuda.synchronize()
        want, want_exps = b8.quantize(f.astype(np.float64), block_rows)
        assert np.array_equal(exps.cpu().numpy(), want_exps)
        _same_codes(codes.cpu().numpy(), want)


# --------------------------------------------------------------------- norm

@pytest.mark.parametrize("T,d", [(1, 16), (1, 4096), (3, 144), (7, 2000), (2, 16384), (33, 8192), (5, 2064), (300, 256), (5, 1024), (4, 528)])
@pytest.mark.parametrize("y_dtype,gain", [("f32", False), ("bf16", True), (None, True), (None, False)])
def test_norm(T, d, y_dtype, gain):
    ms = _ms()
    rng = np.random.default_rng(T + d)
    a = rng.standard_normal((T, d))
    a[:, ::37] *= 20.0
    h, hf = _bf16(a)
    y, yf = (None, None) if y_dtype is None else _input(rng.standard_normal((T, d)) * 0.5, y_dtype)
    w, wf = _bf16(1 + 0.3 * rng.standard_normal(d)) if gain else (None, None)
    outs, checks = zip(*[_guarded((T, d), 0x55 if t == torch.uint8 else -7.0, t)
                         for t in (torch.bfloat16, torch.bfloat16, torch.uint8)])
    exps, check_exps = _guarded((T, -(-d // 128)), 0x55, torch.uint8, gap=5)
    ms.ms_residual_norm_q(h, y, w, 1e-5, T, d, *outs, exps, stream=torch.cuda.current_stream())
    torch.cuda.synchronize()
    x, v = b8.residual_norm(hf, yf, wf, 1e-5)
    want, want_exps = b8.quantize(v)
    assert np.array_equal(exps.cpu().numpy(), want_exps)
    _same_codes(outs[2].cpu().numpy(), want)
    for got, ref in ((outs[0], x), (outs[1], v)):  # half a step of bf16; 64-bit sums differ by far less
        got = got.float().cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - ref) <= 2.0 ** -8 * (1 + 1e-9) * np.abs(ref))
    for check in (*checks, check_exps):
        check()


def test_norm_each_output_alone_and_in_place():
    ms = _ms()
    rng = np.random.default_rng(5)
    T, d = 5, 400
    h, hf = _bf16(rng.standard_normal((T, d)))
    y, yf = _bf16(rng.standard_normal((T, d)))
    x, v = b8.residual_norm(hf, yf)
    ref = [torch.empty(T, d, dtype=torch.bfloat16, device="cuda") for _ in range(2)]
    codes, exps = ms.new_matrix_q(T, d)
    ms.ms_residual_norm_q(h, y, None, 1e-6, T, d, ref[0], ref[1], codes, exps)
    for i in range(2):
        for into in (h, y):
            hh, yy = h.clone(), y.clone()
            target = hh if into is h else yy
            ms.ms_residual_norm_q(hh, yy, None, 1e-6, T, d, **{("sum_out", "out")[i]: target})
            torch.cuda.synchronize()
            assert torch.equal(target, ref[i])
            assert torch.equal(yy if into is h else hh, y if into is h else h)
    hh, yy = h.clone(), y.clone()
    ms.ms_residual_norm_q(hh, yy, None, 1e-6, T, d, sum_out=hh, out=yy)
    c2, e2 = ms.new_matrix_q(T, d)
    ms.ms_residual_norm_q(h, y, None, 1e-6, T, d, codes=c2, exps=e2)
    torch.cuda.synchronize()
    assert torch.equal(hh, ref[0]) and torch.equal(yy, ref[1]) and torch.equal(c2, codes) and torch.equal(e2, exps)


def test_norm_of_extreme_rows():
    """A row of zeros, rows with NaN and infinities, rows whose squares pass fp32."""
    ms = _ms()
    T, d = 6, 272
    a = np.random.default_rng(1).standard_normal((T, d)).astype(np.float32)
    a[0] = 0
    a[1, 3] = np.nan
    a[2, 4] = np.inf
    a[3] *= 2.0 ** 100
    a[4] *= 2.0 ** -100
    h, hf = _bf16(a)
    codes, exps = ms.new_matrix_q(T, d)
    out = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    ms.ms_residual_norm_q(h, None, None, 0.0, T, d, out=out, codes=codes, exps=exps)
    torch.cuda.synchronize()
    got = out.float().cpu().numpy()
    with np.errstate(divide="ignore", invalid="ignore"):
        x, v = b8.residual_norm(hf, eps=0.0)
    assert np.all(np.isnan(got[0]) == np.isnan(v[0])) and np.all(np.isnan(got[1]))
    assert np.isnan(got[2, 4]) and np.all(got[2, 5:] == 0)
    assert np.all(np.abs(got[3:] - v[3:]) <= 2.0 ** -8 * (1 + 1e-9) * np.abs(v[3:]))
    want, want_exps = b8.quantize(v)
    assert np.array_equal(exps.cpu().numpy(), want_exps)
    _same_codes(codes.cpu().numpy(), want)


# ------------------------------------------------------------------ product

def _matrix(rng, rows, n, block_rows, spread=4, nan=0):
    """A random matrix in 8 bits: every code but NaN's, scales of neighbouring blocks far apart."""
    codes = b8.encode(rng.standard_normal((rows, n)) * 90)
    exps = (b8.BIAS - 6 + rng.integers(-spread, spread + 1, (-(-rows // block_rows), -(-n // 128)))).astype(np.uint8)
    return codes, exps


def _dense(T, n_in, n_out, dtype, add=None, shift=0, seed=0, spread=4):
    ms = _ms()
    rng = np.random.default_rng(T + n_in + n_out + seed)
    x, xe = _matrix(rng, T, n_in, 1, spread)
    w, we = _matrix(rng, n_out, n_in, 128, spread)
    t = torch.float32 if dtype == "f32" else torch.bfloat16
    size = rng.standard_normal((T, n_out)) * 30
    a, af = _input(size, dtype)
    buf = torch.full((T * n_out + 66,), -7.0, dtype=t, device="cuda")
    y = buf[shift:shift + T * n_out].view(T, n_out)
    if add == "alias":
        y.copy_(a)
    args = [torch.from_numpy(v).cuda() for v in (x, xe, w, we)]
    ms.ms_dense_q(*args, T, n_in, n_out, y, {None: None, "apart": a, "alias": y}[add], torch.cuda.current_stream())
    torch.cuda.synchronize()
    ref, mags = b8.dense(b8.values(x, xe), b8.values(w, we, 128), af if add else None)
    out = buf.float().cpu().numpy().astype(np.float64)
    assert np.all(out[:shift] == -7.0) and np.all(out[shift + T * n_out:] == -7.0)
    got = out[shift:shift + T * n_out].reshape(T, n_out)
    # fp32: products of two codes are exact, their sums round n_in / 32 + 8 times by at most 2^-23 of the terms' sizes.
    # bf16: every product may lose 2^-12 of the largest of its eight, which is at most their sum: 8 * 2^-12 of the
    # terms' sizes, and the result half a step
    bound = (n_in / 32 + 8) * 2.0 ** -23 * mags
    if dtype == "bf16":
        bound = bound + 2.0 ** -9 * mags + 2.0 ** -8 * np.abs(ref)
    bad = ~(np.abs(got - ref) <= bound * 1.01)
    assert not bad.any(), (bad.sum(), np.argwhere(bad)[:4].tolist(), got[bad][:4], ref[bad][:4], bound[bad][:4])


# few tokens: every number of blocks of 16 outputs and of waves (outputs up to 4096, 8192 and more, by rows of up to
# 2048 and 4096 columns and longer ones), 1, 2 and 4 blocks of tokens; then tiles of 32 x 32 to 256 x 256 with
# remainders, of fewer stages than parts of waves, and two sizes of them in a launch; widths that end inside a block of 128; the longest row
@pytest.mark.parametrize("T,n_in,n_out", [(1, 16, 1), (1, 4096, 6144), (1, 16384, 33), (2, 144, 100), (15, 2000, 129),
                                          (1, 4112, 4099), (16, 4112, 4099), (3, 2064, 8200), (16, 80, 8211),
                                          (16, 1024, 300), (17, 512, 70), (32, 144, 4101), (20, 272, 8210), (33, 448, 30),
                                          (64, 80, 4100), (50, 144, 8205), (30, 2064, 200), (64, 4096, 100), (61, 2000, 1003),
                                          (65, 80, 2500), (130, 8192, 200), (129, 1104, 257), (250, 128, 6144),
                                          (511, 272, 6100), (1000, 256, 4099), (2047, 144, 6140), (300, 16384, 150),
                                          (1500, 80, 6200), (2000, 144, 8190), (1030, 272, 16400), (1300, 400, 11001),
                                          (1300, 80, 11500), (1800, 144, 18504), (60, 2000, 8200), (500, 1200, 6100),
                                          (1030, 1104, 1030), (33, 16384, 40)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dense(T, n_in, n_out, dtype):
    _dense(T, n_in, n_out, dtype)


@pytest.mark.parametrize("T,n_in,n_out", [(1, 256, 13), (9, 144, 64), (40, 400, 130), (300, 256, 515), (1030, 128, 1030)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("add", ["apart", "alias"])
@pytest.mark.parametrize("shift", [0, 1])
def test_dense_add_and_unaligned_results(T, n_in, n_out, dtype, add, shift):
    _dense(T, n_in, n_out, dtype, add, shift)


@pytest.mark.parametrize("T,n_in,n_out", [(1, 512, 64), (70, 512, 200), (600, 384, 700)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dense_scales_at_their_ends(T, n_in, n_out, dtype):
    """Exponents from -40 to 40 on both sides: products from 2^-98 to 2^98."""
    _dense(T, n_in, n_out, dtype, spread=34)


@pytest.mark.parametrize("T,n_in,n_out", [(1, 400, 64), (5, 2064, 50), (70, 400, 200), (600, 400, 700), (2000, 272, 3000)])
@pytest.mark.parametrize("dtype", ["f32", "bf16"])
def test_dense_nan_stays_in_its_row(T, n_in, n_out, dtype):
    """A code of NaN at the end of a row of x (w) makes that token's (output's) results NaN, and no others, though the
    next row's codes follow it in memory."""
    ms = _ms()
    rng = np.random.default_rng(T)
    x, xe = _matrix(rng, T, n_in, 1)
    w, we = _matrix(rng, n_out, n_in, 128)
    t0, o0 = T // 2, n_out // 3
    x[t0, 0] = x[t0, -1] = 0x7f
    w[o0, 0] = w[o0, -1] = 0xff
    y = torch.zeros(T, n_out, dtype=torch.float32 if dtype == "f32" else torch.bfloat16, device="cuda")
    ms.ms_dense_q(*[torch.from_numpy(v).cuda() for v in (x, xe, w, we)], T, n_in, n_out, y)
    torch.cuda.synchronize()
    nan = torch.isnan(y).cpu().numpy()
    want = np.zeros((T, n_out), bool)
    want[t0], want[:, o0] = True, True
    assert np.array_equal(nan, want)


def test_rows_past_32_bits():
    """Rows whose values lie past 2^32 of a matrix, its codes or its results, as the same rows alone."""
    ms = _ms()
    R, n, tail = 2049 * 128, 16384, 128
    s = torch.cuda.current_stream()
    torch.manual_seed(3)
    x = torch.zeros(R, n, dtype=torch.bfloat16, device="cuda")
    x[-tail:] = 3 * torch.randn(tail, n, device="cuda")
    last = x[-tail:].clone()
    for block_rows in (1, 128):
        codes, exps = ms.new_matrix_q(R, n, block_rows)
        c, e = ms.new_matrix_q(tail, n, block_rows)
        ms.ms_quant_q(x, R, n, block_rows, codes, exps, s)
        ms.ms_quant_q(last, tail, n, block_rows, c, e, s)
        assert torch.equal(codes[-tail:], c) and torch.equal(exps[-len(e):], e) and not codes[:-tail].any()
    y, mags = {}, None
    for T in (3, 70, 300):  # weights: the last one's codes and exponents
        a, ae = ms.new_matrix_q(T, n)
        ms.ms_quant_q(last[:1].expand(T, n).contiguous() if T > tail else last[:T].clone(), T, n, 1, a, ae, s)
        out = torch.empty(T, R, dtype=torch.float32, device="cuda")
        ms.ms_dense_q(a, ae, codes, exps, T, n, R, out, stream=s)
        ref, mags = b8.dense(b8.values(a[:3].cpu().numpy(), ae[:3].cpu().numpy()), b8.values(c.cpu().numpy(), e.cpu().numpy(), 128), None)
        assert np.all(np.abs(out[:3, -tail:].cpu().numpy() - ref) <= (n / 32 + 8) * 2.0 ** -23 * mags) and not out[:, :-tail].any()
    del codes, out
    total, out = torch.empty_like(x), torch.empty_like(x)
    codes, exps = ms.new_matrix_q(R, n)
    ms.ms_residual_norm_q(x, None, None, 1e-6, R, n, total, out, codes, exps, s)
    alone = [torch.empty_like(last), torch.empty_like(last), *ms.new_matrix_q(tail, n)]
    ms.ms_residual_norm_q(last, None, None, 1e-6, tail, n, *alone, s)
    for got, want in zip((total, out, codes, exps), alone):
        assert torch.equal(got[-tail:], want)
    del x, total, out, codes
    T, n_in, n_out = 40000, 16, 110000
    a, ae = ms.new_matrix_q(T, n_in)
    w, we = ms.new_matrix_q(n_out, n_in, 128)
    ms.ms_quant_q(torch.randn(T, n_in, device="cuda"), T, n_in, 1, a, ae, s)
    ms.ms_quant_q(torch.randn(n_out, n_in, device="cuda"), n_out, n_in, 128, w, we, s)
    y = torch.empty(T, n_out, dtype=torch.bfloat16, device="cuda")
    ms.ms_dense_q(a, ae, w, we, T, n_in, n_out, y, stream=s)
    ref, mags = b8.dense(b8.values(a.cpu().numpy(), ae.cpu().numpy())[-300:], b8.values(w.cpu().numpy(), we.cpu().numpy(), 128)[-300:], None)
    bad = np.abs(y[-300:, -300:].float().cpu().numpy() - ref) > 1.01 * (2.0 ** -9 * mags + 2.0 ** -8 * np.abs(ref)) + 2.0 ** -19 * mags
    assert not bad.any()
    del y
    torch.cuda.empty_cache()


def test_a_run_of_them():
    """norm -> product -> norm -> ..., eager and as a captured graph with other inputs, on a side stream: every call
    against the oracle on what the call before left."""
    ms = _ms()
    rng = np.random.default_rng(3)
    T, d, n = 5, 512, 384
    s = torch.cuda.Stream()
    h, hf = _bf16(rng.standard_normal((T, d)))
    w1, w2 = 0.05 * rng.standard_normal((n, d)), 0.05 * rng.standard_normal((d, n))
    q1, q2 = (tuple(torch.from_numpy(v).cuda() for v in b8.quantize(w.astype(np.float32), 128)) for w in (w1, w2))
    m1, m2 = ms.new_matrix_q(n, d, 128), ms.new_matrix_q(d, n, 128)
    for (c, e), w in ((m1, w1), (m2, w2)):
        ms.ms_quant_q(torch.from_numpy(w.astype(np.float32)).cuda(), *w.shape, 128, c, e)
    torch.cuda.synchronize()
    for got, want in ((m1, q1), (m2, q2)):
        assert torch.equal(got[0], want[0]) and torch.equal(got[1], want[1])
    xq, zq = ms.new_matrix_q(T, d), ms.new_matrix_q(T, n)
    mid = torch.empty(T, n, dtype=torch.float32, device="cuda")
    mid16 = torch.empty(T, n, dtype=torch.bfloat16, device="cuda")
    y = torch.empty(T, d, dtype=torch.float32, device="cuda")
    out = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
    total = torch.empty_like(out)

    def chain(stream):
        ms.ms_residual_norm_q(h, None, None, 1e-6, T, d, codes=xq[0], exps=xq[1], stream=stream)
        ms.ms_dense_q(*xq, *m1, T, d, n, mid, stream=stream)
        ms.ms_dense_q(*xq, *m1, T, d, n, mid16, stream=stream)
        ms.ms_quant_q(mid, T, n, 1, *zq, stream=stream)
        ms.ms_dense_q(*zq, *m2, T, n, d, y, stream=stream)
        ms.ms_residual_norm_q(h, y, None, 1e-6, T, d, sum_out=total, out=out, stream=stream)

    def check(hf):
        _, v = b8.residual_norm(hf)
        x, xe = b8.quantize(v)
        _same_codes(xq[0].cpu().numpy(), x)
        ref, mags = b8.dense(b8.values(x, xe), b8.values(*[t.cpu().numpy() for t in m1], 128))
        got = mid.cpu().numpy().astype(np.float64)
        assert np.all(np.abs(got - ref) <= 32 * 2.0 ** -23 * mags)
        assert np.all(np.abs(mid16.float().cpu().numpy() - ref) <= 2.0 ** -8 * np.abs(ref) + 2.0 ** -9 * mags)
        z, ze = b8.quantize(got)
        _same_codes(zq[0].cpu().numpy(), z)
        ref, mags = b8.dense(b8.values(z, ze), b8.values(*[t.cpu().numpy() for t in m2], 128))
        yf = y.cpu().numpy().astype(np.float64)
        assert np.all(np.abs(yf - ref) <= 32 * 2.0 ** -23 * mags)
        x, v = b8.residual_norm(hf, yf)
        for t, ref in ((total, x), (out, v)):
            assert np.all(np.abs(t.float().cpu().numpy() - ref) <= 2.0 ** -8 * (1 + 1e-9) * np.abs(ref))

    s.wait_stream(torch.cuda.current_stream())
    chain(s)
    torch.cuda.synchronize()
    check(hf)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=s):
        chain(torch.cuda.current_stream())
    for _ in range(3):
        h2, hf = _bf16(rng.standard_normal((T, d)) * 3)
        h.copy_(h2)
        for t in (mid, y, out):
            t.zero_()
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        check(hf)


# ------------------------------------------------------------- the decoder

def _decoder(P, **kw):
    from decoder import Decoder
    shape, attn = synth.ModelShape("dec-tiny", 2, 256, 512, 8, 2, "bf16"), synth.TINY_ATTN
    return shape, attn, Decoder(shape, attn, seed=4, n_sets=2, max_tokens=P, max_ctx=P + 20,
                                budget_total=2 * 8 * shape.expert_bytes, dense_bits=8, **kw)


def _ready(dec):
    from workload import top_bytes
    ms = _ms()
    dec.stack.configure(0.5, 2 * 4 * top_bytes(dec.stack.rig, 0.5))
    for l in range(2):
        dec.stack.rig.load_tops(l, [0, 1, 2, 3])
    ms.ms_sync(dec.ctx)


@pytest.mark.parametrize("kv_bits", [16, 8])
def test_decoder_in_8_bits(kv_bits):
    """A two-layer decoder around the experts with dense_bits=8, a prompt and drawn tokens: every layer's attention module
    against the oracle from the layer's input, with weights and activations quantized as the library says, and the logits
    from the codes of the last layer's result; the token from those logits."""
    from decoder import Sampling
    from gpu_helpers import check_close
    from oracle import decoder as od
    from oracle import sample as osm
    P, n_dec = 70, 4
    shape, attn, dec = _decoder(P, kv_bits=kv_bits)
    Hq, Hkv, D = attn.n_heads, attn.n_kv_heads, attn.head_dim
    settings = dict(temperature=0.8, top_k=40, top_p=0.95, min_p=0.01)
    with dec:
        _ready(dec)
        draw = Sampling(attn.vocab, seed=7, n=3, **settings)
        quantized = lambda w: b8.values(*b8.quantize(w.astype(np.float64), 128), 128)  # noqa: E731
        weights = [[quantized(w) for w in dec.f32[s]] for s in range(dec.n_sets)]
        x = torch.empty(P, shape.d_model, dtype=torch.bfloat16, device="cuda")
        x1 = torch.empty(1, shape.d_model, dtype=torch.bfloat16, device="cuda")
        dec.embed_ids(torch.from_numpy(synth.prompt_tokens(attn, 4, P)).cuda(), P, x)
        caches = [od.Cache(Hkv, P + 20, D) for _ in range(2)]
        for step in range(1 + n_dec):
            T, pos0 = (P if step == 0 else 1), dec.pos
            cap = dec.step(x if step == 0 else x1, T, capture=(0, 1), sampling=draw)
            torch.cuda.synchronize()
            for l in range(2):
                xin = cap[l]["x"].astype(np.float64)
                w_qkv, w_o = weights[l % dec.n_sets]
                # the library's codes are of the norm before its rounding to bf16, the oracle's of bf16 (a few move by one
                # step), and the 8-bit cache's values are off by 2^-4 at most: of an attention module's result, which the
                # weights leave under a third of the layer's largest value, that is averaged over rows of 64 and more
                a = od.attention(b8.values(*b8.quantize(xin)), w_qkv, w_o, caches[l], pos0, Hq, Hkv, D, attn.rope_base)
                att = b8.dense(b8.values(*b8.quantize(a["o"])), w_o)[0]
                check_close(cap[l]["h"], od.bf16_round(od.rmsnorm(xin + att)), "bf16", "step %d layer %d h" % (step, l))
            last = b8.values(*[t[T - 1:T].cpu().numpy() for t in dec.xq])
            ref, mags = b8.dense(last, quantized(dec.head_f32))
            logits = dec.logits.cpu().numpy().astype(np.float64)
            assert np.all(np.abs(logits - ref) <= 16 * 2.0 ** -23 * mags)
            token, share, near = osm.draw(logits[0], draw.numbers[draw.used - 1].item(), **{
                k: np.float64(np.float32(v)) if k != "top_k" else v for k, v in settings.items()})
            if near > 1e-9:
                assert int(dec.ids[0]) == token and abs(float(dec.prob[0]) - share) <= 2.0 ** -23
            dec.embed_ids(dec.ids, 1, x1)
        assert dec.pos == P + n_dec


def test_decoder_in_8_bits_allocates_nothing_and_repeats():
    """Steps on a stream that is not the current one allocate no device memory; the same seed draws the same tokens."""
    from decoder import Sampling
    _, attn, dec = _decoder(40, kv_bits=8, keep_f32=False)
    with dec:
        _ready(dec)
        prompt = synth.prompt_tokens(attn, 1, 40)
        stream = torch.cuda.Stream()
        torch.cuda.synchronize()
        got = []
        for _ in range(2):
            dec.reset()
            draw = Sampling(attn.vocab, temperature=1.5, top_p=0.9, seed=3, n=4)
            got.append(dec.generate(prompt, 9, stream=stream, sampling=draw)[0])
        assert got[0] == got[1] and all(0 <= t < attn.vocab for t in got[0])
        dec.reset()
        x = torch.randn(1, 256, device="cuda").to(torch.bfloat16)
        torch.cuda.synchronize()
        dec.step(x, 1, stream=stream, sampling=draw)
        before = torch.cuda.memory_stats()["allocation.all.allocated"]
        for _ in range(12):
            dec.step(x, 1, stream=stream, sampling=draw)
        stream.synchronize()
        assert torch.cuda.memory_stats()["allocation.all.allocated"] == before


@pytest.mark.parametrize("kv_bits", [16, 8])
def test_a_decoder_is_ready_for_every_stream(kv_bits, monkeypatch):
    """What its constructor enqueues (codes of the weights, cleared caches) has finished when it returns: the first step may
    be on another stream."""
    from workload import SplitRig
    outputs = SplitRig.outputs

    def late(rig, T):  # among the last things that a decoder makes
        torch.cuda._sleep(200_000_000)
        return outputs(rig, T)
    monkeypatch.setattr(SplitRig, "outputs", late)
    _, _, dec = _decoder(40, kv_bits=kv_bits, keep_f32=False)
    with dec:
        assert torch.cuda.current_stream().query()


@pytest.mark.parametrize("T", [1, 40])
def test_the_residual_sum_takes_the_attention_as_it_is(T):
    """h of the last layer, from its input and the attention's codes left by the step: rounded once, to half a step of bf16,
    with no rounding of the attention's result before the sum."""
    _, attn, dec = _decoder(40)
    with dec:
        _ready(dec)
        x = torch.randn(T, 256, device="cuda").to(torch.bfloat16)
        torch.cuda.synchronize()
        cap = dec.step(x, T, capture=(1,))
        torch.cuda.synchronize()
        o = b8.values(*[t[:T].cpu().numpy() for t in dec.oq])
        w = b8.values(*[t.cpu().numpy() for t in dec.layer_weights(1)[1]], 128)
        att, mags = b8.dense(o, w)
        xin = cap[1]["x"].astype(np.float64)
        total, h = b8.residual_norm(xin, att)
        half = np.exp2(np.floor(np.log2(np.abs(h))) - 8)
        sums = 16 * 2.0 ** -23 * mags * np.abs(h / total)
        bad = np.abs(cap[1]["h"] - h) > half * (1 + 2.0 ** -20) + sums
        assert not bad.any(), (bad.sum(), bad.size)
        assert np.median(np.abs(att / total)) > 2.0 ** -6  # (rounded before the sum, it would show)
