"""The oracle of the 8-bit cache against the definitions, and what the library
refuses before it enqueues anything (no GPU needed)."""
import ctypes

import numpy as np
import pytest

from oracle import kvcache as kv


def test_codes_are_the_nearest_values():
    rng = np.random.default_rng(0)
    x = np.concatenate([rng.standard_normal(2000) * 2.0 ** rng.integers(-12, 9, 2000), kv.TABLE[:127], -kv.TABLE[:127]])
    x = x[np.abs(x) <= 448]
    got = kv.TABLE[kv.encode(x)]
    best = np.min(np.abs(x[:, None] - kv.TABLE[~np.isnan(kv.TABLE)]), axis=1)
    assert np.array_equal(np.abs(got - x), best)
    # half a step: 2^-4 of a normal value, 2^-10 below 2^-6
    assert np.all(np.abs(got - x) <= np.maximum(2.0 ** -4 * np.abs(x), 2.0 ** -10))


def test_codes_at_the_borders():
    ties = np.array([1.0625, 1.1875, 2.0 ** -10, 3 * 2.0 ** -10, 460.0, 1e30, -1e30, np.inf, -np.inf, np.nan])
    assert kv.TABLE[kv.encode(ties[:6])].tolist() == [1.0, 1.25, 0.0, 2.0 ** -8, 448.0, 448.0]
    assert kv.TABLE[kv.encode(ties[6:7])].tolist() == [-448.0]
    assert np.all(np.isnan(kv.TABLE[kv.encode(ties[7:])]))


@pytest.mark.parametrize("top,e", [(448.0, 0), (448.5, 1), (224.0, -1), (0.0, -40), (1e-30, -40), (1e30, 40), (7.0, -6), (7.1, -5)])
def test_exponent_is_the_least_that_holds_the_block(top, e):
    assert kv.exponent([0.0, -top, np.nan, np.inf]) == e


def test_append_in_pieces_ends_at_the_same_scales():
    rng = np.random.default_rng(3)
    k = rng.standard_normal((150, 2, 64)) * np.exp2(rng.integers(-3, 6, (150, 2, 1)).astype(float))
    whole, parts = kv.Cache(1, 2, 192, 64), kv.Cache(1, 2, 192, 64)
    whole.append(0, 0, k, k)
    for a, b in ((0, 5), (5, 64), (64, 65), (65, 150)):
        parts.append(0, a, k[a:b], k[a:b])
    assert np.array_equal(whole.ke[:, :, :2], parts.ke[:, :, :2]) and np.array_equal(whole.ve, parts.ve)
    # rounded twice only where a code fell below the least normal one: at most half a step of it more
    step = np.repeat(np.exp2(whole.ke.astype(float) - kv.BIAS - 10), 64, axis=2)[..., None]
    assert np.all(np.abs(whole.values("k") - parts.values("k"))[:, :, :150] <= 2 * step[:, :, :150])


def test_stretched_positions():
    f = kv.frequencies(128, 1e6)
    assert np.allclose(kv.frequencies(128, 1e6, factor=4.0), f / 4)
    g = kv.frequencies(128, 1e6, factor=4.0, orig=8192, low=1.0, high=32.0)
    turns = 8192 * f / (2 * np.pi)
    assert np.array_equal(g[turns >= 32], f[turns >= 32]) and np.allclose(g[turns <= 1], f[turns <= 1] / 4)
    assert np.all(np.diff(g) < 0)


def _cache(S=2, H=2, D=64, ctx=128):
    from paper_2509_08342_amd import moesplit as ms
    return ms.ms_kv_cache_q(4096, 8192, 12288, 16384, S, H, D, ctx)  # addresses that no refused call reads


def _rope(**kw):
    from paper_2509_08342_amd import moesplit as ms
    return ms.rope_desc(kw.pop("rot_dim", 64), kw.pop("base", 1e4), **kw)


def _status(fn, *args):
    from paper_2509_08342_amd import moesplit as ms
    try:
        fn(*args)
    except ms.MoeSplitError as e:
        return e.status
    return ms.MS_OK


@pytest.mark.parametrize("change,status", [
    (dict(n_seqs=0), 1), (dict(n_kv_heads=-1), 1), (dict(head_dim=0), 1), (dict(head_dim=96), 6), (dict(head_dim=512), 6),
    (dict(max_ctx=100), 1), (dict(max_ctx=0), 1), (dict(k=0), 1), (dict(v_exp=0), 1), (dict(v=8200), 1)])
def test_refused_caches(change, status):
    from paper_2509_08342_amd import moesplit as ms
    c = _cache()
    for name, x in change.items():
        setattr(c, name, x)
    assert _status(ms.ms_rope_kv_q, c, _rope(rot_dim=0), 4096, 1, 4, 0, 4096) == status
    assert _status(ms.ms_kv_read_q, c, 0, 1, 4096, 4096) == status
    assert _status(ms.ms_attention_q, c, 4096, 1, 4, 0, 4096, None) == status


@pytest.mark.parametrize("kw", [dict(rot_dim=3), dict(rot_dim=66), dict(rot_dim=-2), dict(base=1.0), dict(base=float("nan")),
                                dict(base=float("inf")), dict(factor=0.5), dict(factor=float("inf")), dict(orig_ctx=-1.0),
                                dict(orig_ctx=10.0, low=5.0, high=5.0), dict(orig_ctx=10.0, low=-1.0), dict(mscale=0.0),
                                dict(orig_ctx=10.0, high=float("nan")), dict(mscale=float("nan"))])
def test_refused_rotary_descriptions(kw):
    from paper_2509_08342_amd import moesplit as ms
    assert _status(ms.ms_rope_kv_q, _cache(), _rope(**kw), 4096, 1, 4, 0, 4096) == ms.MS_E_INVALID


@pytest.mark.parametrize("T,Hq,pos0,x,y", [(-1, 4, 0, 4096, 4096), (1, 0, 0, 4096, 4096), (1, 3, 0, 4096, 4096),
                                           (1, 4, -1, 4096, 4096), (1, 4, 128, 4096, 4096), (129, 4, 0, 4096, 4096),
                                           (1, 4, 2 ** 31 - 1, 4096, 4096), (1, 4, 0, None, 4096), (1, 4, 0, 4096, None),
                                           (1, 4, 0, 4104, 4096), (1, 4, 0, 4096, 4104)])
def test_refused_calls(T, Hq, pos0, x, y):
    from paper_2509_08342_amd import moesplit as ms
    c = _cache()
    assert _status(ms.ms_rope_kv_q, c, _rope(), x, T, Hq, pos0, y) == ms.MS_E_INVALID
    assert _status(lambda: ms._check(ms.lib.ms_attention_q(ctypes.byref(c), x, T, Hq, pos0, None, None, y, 4096, 1 << 40,
                                                           None))) == ms.MS_E_INVALID
    assert _status(ms.ms_rope_kv_q, c, None, 4096, 1, 4, 0, 4096) == ms.MS_E_INVALID


@pytest.mark.parametrize("pos0,n,k,v", [(-1, 1, 4096, 4096), (0, 129, 4096, 4096), (128, 1, 4096, 4096), (0, -1, 4096, 4096),
                                        (0, 1, None, 4096), (0, 1, 4096, None), (0, 1, 4100, 4096), (2 ** 31 - 1, 1, 4096, 4096)])
def test_refused_reads(pos0, n, k, v):
    from paper_2509_08342_amd import moesplit as ms
    assert _status(ms.ms_kv_read_q, _cache(), pos0, n, k, v) == ms.MS_E_INVALID


@pytest.mark.parametrize("kw", [dict(scale=-1.0), dict(scale=float("nan")), dict(scale=float("inf")), dict(softcap=-1.0),
                                dict(softcap=float("inf")), dict(window=-1), dict(prefix=-1)])
def test_refused_options(kw):
    from paper_2509_08342_amd import moesplit as ms
    assert _status(lambda: ms.ms_attention_q(_cache(), 4096, 1, 4, 0, 1 << 20, None, ms.attn_opts(**kw))) == ms.MS_E_INVALID


def test_documents_that_are_not_aligned_are_refused():
    from paper_2509_08342_amd import moesplit as ms
    opts = ms.attn_opts()
    opts.docs_dev = 4100
    assert _status(lambda: ms.ms_attention_q(_cache(), 4096, 1, 4, 0, 1 << 20, None, opts)) == ms.MS_E_INVALID


def test_calls_of_too_many_rows_are_unsupported():
    from paper_2509_08342_amd import moesplit as ms
    c = _cache(S=1 << 12, H=1, ctx=2048)
    assert ms.ms_attention_q_workspace(c, 1024, 1, 0) >= 0
    assert _status(ms.ms_attention_q_workspace, c, 1025, 1, 0) == ms.MS_E_UNSUPPORTED
    assert _status(ms.ms_attention_q, c, 4096, 1025, 1, 0, 1 << 40, None) == ms.MS_E_UNSUPPORTED
    big = _cache(S=1 << 30, H=1, ctx=64)
    assert _status(ms.ms_rope_kv_q, big, _rope(), 4096, 1, 1, 0, 1 << 40) == ms.MS_E_UNSUPPORTED
    assert _status(ms.ms_kv_read_q, big, 0, 1, 1 << 40, 1 << 41) == ms.MS_E_UNSUPPORTED


def test_workspaces_stay_small():
    """At most 64 shares a row, and none for a prompt that fills the chip."""
    from paper_2509_08342_amd import moesplit as ms
    for T, Hq, pos0 in [(1, 8, 1 << 20), (16, 8, 9000), (100, 64, 100000), (8192, 32, 0), (1, 71, 5000)]:
        for H in (1, Hq):
            n = ms.ms_attention_q_workspace(_cache(S=1, H=H, D=128, ctx=1 << 21), T, Hq, pos0)
            assert n <= T * Hq * 64 * 130 * 4
            assert n == 0 or T * Hq < 1 << 18


def test_out_over_part_of_q_and_small_workspaces_are_refused():
    from paper_2509_08342_amd import moesplit as ms
    c = _cache(S=1, H=1, ctx=1 << 20)
    assert _status(ms.ms_attention_q, _cache(), 4096, 2, 4, 0, 4096 + 256, None) == ms.MS_E_INVALID
    n = ms.ms_attention_q_workspace(c, 1, 4, (1 << 20) - 1)
    if n:
        call = lambda size, at: ms._check(ms.lib.ms_attention_q(  # noqa: E731
            ctypes.byref(c), 4096, 1, 4, (1 << 20) - 1, None, None, 1 << 20, at, size, None))
        assert _status(call, n - 1, 1 << 30) == ms.MS_E_INVALID
        assert _status(call, n, None) == ms.MS_E_INVALID and _status(call, n, (1 << 30) + 8) == ms.MS_E_INVALID


def test_no_tokens_is_no_work():
    from paper_2509_08342_amd import moesplit as ms
    c = _cache()
    assert _status(ms.ms_rope_kv_q, c, _rope(), None, 0, 4, 0, None) == ms.MS_OK
    assert _status(ms.ms_kv_read_q, c, 128, 0, None, None) == ms.MS_OK
    assert _status(ms.ms_attention_q, c, None, 0, 4, 128, None, None) == ms.MS_OK
    assert ms.ms_attention_q_workspace(c, 0, 4, 0) == 0


def test_cache_shapes_are_checked_by_the_binding():
    torch = pytest.importorskip("torch")
    from paper_2509_08342_amd import moesplit as ms
    c = ms.new_kv_cache_q(2, 3, 64, 128, device="cpu")
    assert (c.n_seqs, c.n_kv_heads, c.head_dim, c.max_ctx) == (2, 3, 64, 128)
    k, v, ke, ve = c.tensors
    with pytest.raises(ValueError):
        ms.kv_cache_q(k, v[:1], ke, ve)
    with pytest.raises(ValueError):
        ms.kv_cache_q(k, v, ke, ve[:, :, :1])
    with pytest.raises(ValueError):
        ms.attn_opts(slopes=torch.zeros(4, dtype=torch.bfloat16))
    for fn, args in ((ms.ms_rope_kv_q, (c, _rope(), 4096, 1, 3, 0, 4096)), (ms.ms_attention_q, (c, 4096, 1, 3, 0, 4096, None))):
        with pytest.raises(ValueError):
            fn(*args, span=torch.tensor([[0, 1], [0, 1]]))


@pytest.mark.parametrize("D", [64, 128, 256])
@pytest.mark.parametrize("S,H,G", [(1, 1, 1), (1, 8, 4), (1, 2, 8), (3, 5, 3), (32, 8, 8), (70, 4, 1)])
def test_no_position_needs_a_smaller_workspace_than_one_before(S, H, G, D):
    """So the last position that T tokens may start at tells what a decode ever needs."""
    from paper_2509_08342_amd import moesplit as ms
    c = _cache(S=S, H=H, D=D, ctx=1 << 17)
    for T in (1, 2, 5, 16, 17, 40, 129, 500, 2048):
        if S * T * H * G <= 1 << 22:
            sizes = [ms.ms_attention_q_workspace(c, T, H * G, p) for p in [*range(0, 9000, 64), *range(9000, (1 << 17) - T, 1009)]]
            assert all(a <= b for a, b in zip(sizes, sizes[1:])), T
            assert sizes[-1] > 0 or S * H > 256 or T > 1


def test_tensor_shapes_are_checked_by_the_binding():
    """A kernel would read or write past a tensor that is too small, or other sequences' numbers of one laid out otherwise."""
    torch = pytest.importorskip("torch")
    from paper_2509_08342_amd import moesplit as ms
    S, Hq, Hkv, D, ctx, T = 2, 6, 3, 64, 128, 3
    c = ms.new_kv_cache_q(S, Hkv, D, ctx, device="cpu")

    def t(*shape, dtype=torch.bfloat16):
        return torch.zeros(*shape, dtype=dtype)

    qkv, q = t(S, T, Hq + 2 * Hkv, D, dtype=torch.float32), t(S, T, Hq, D)
    short = q.flatten()[:-1]
    for args in [(qkv.flatten()[:-1], T, Hq, 0, q), (qkv, T, Hq, 0, short), (qkv.to(torch.bfloat16), T, Hq, 0, q),
                 (qkv, T, Hq, 0, qkv)]:
        with pytest.raises(ValueError):
            ms.ms_rope_kv_q(c, _rope(), *args)
    k = t(S, Hkv, 70, D)
    for args in [(0, 71, k, k), (0, 70, k, k[:, :, :69].contiguous()), (0, 70, k.float(), k)]:
        with pytest.raises(ValueError):
            ms.ms_kv_read_q(c, *args)
    for args in [(q, T + 1, Hq, 0, q), (q, T, Hq, 0, short), (q.float(), T, Hq, 0, q), (q, T, Hq, 0, q.float())]:
        with pytest.raises(ValueError):
            ms.ms_attention_q(c, *args)
    for span in (t(S, 3, dtype=torch.int32), t(S - 1, 2, dtype=torch.int32), t(2 * S, dtype=torch.int32)):
        with pytest.raises(ValueError):
            ms.ms_attention_q(c, q, T, Hq, 0, q, span=span)
        with pytest.raises(ValueError):
            ms.ms_rope_kv_q(c, _rope(), qkv, T, Hq, 0, q, span=span)
    for opts in (dict(doc=t(S, T, dtype=torch.int32)), dict(doc=t(ctx, dtype=torch.int32)), dict(doc=t(1, ctx, dtype=torch.int32)),
                 dict(slopes=t(Hkv, dtype=torch.float32))):
        with pytest.raises(ValueError):
            ms.ms_attention_q(c, q, T, Hq, 0, q, opts=ms.attn_opts(**opts))


@pytest.mark.parametrize("mscale", [3.5e38, 1e300])
def test_scales_of_cosine_and_sine_past_fp32_are_refused(mscale):
    """Sines that are infinite in fp32 would make NaN of finite values."""
    from paper_2509_08342_amd import moesplit as ms
    assert _status(ms.ms_rope_kv_q, _cache(), _rope(mscale=mscale), 4096, 1, 4, 0, 4096) == ms.MS_E_INVALID


def test_scales_that_pass_fp32_in_powers_of_two_are_refused():
    """exp(scale x) is taken as 2^(scale log2(e) x): an infinite factor would make NaN of a product of zero."""
    from paper_2509_08342_amd import moesplit as ms
    assert _status(lambda: ms.ms_attention_q(_cache(), 4096, 1, 4, 0, 1 << 20, None, ms.attn_opts(scale=3e38))) == ms.MS_E_INVALID


def test_workspace_sizes_and_what_they_guard():
    """A result, an exponent and a sum for every row and share: 64 shares of a token behind 2^20 positions of one head, none
    for a call that fills the chip; and a workspace that is smaller, missing or not aligned is refused."""
    from paper_2509_08342_amd import moesplit as ms
    c = _cache(S=1, H=1, ctx=1 << 20)
    n = ms.ms_attention_q_workspace(c, 1, 4, (1 << 20) - 1)
    assert n == 4 * 64 * (64 + 2) * 4
    call = lambda size, at: ms._check(ms.lib.ms_attention_q(  # noqa: E731
        ctypes.byref(c), 4096, 1, 4, (1 << 20) - 1, None, None, 1 << 20, at, size, None))
    for size, at in ((n - 1, 1 << 30), (0, 1 << 30), (n, None), (n, (1 << 30) + 8)):
        assert _status(call, size, at) == ms.MS_E_INVALID
    assert ms.ms_attention_q_workspace(_cache(S=1 << 12, H=1, ctx=2048), 1024, 1, 0) == 0


def test_every_launch_asks_for_lds():
    """A work-group without LDS may land on the compute units that copies of experts hold, and waits behind their reads."""
    import os
    import re
    import paper_2509_08342_amd
    text = open(os.path.join(os.path.dirname(paper_2509_08342_amd.__file__), "csrc", "kvcache.hip")).read()
    lds = [re.split(r",(?![^(<]*[)>])", re.sub(r"\s+", " ", call))[3].strip()
           for call in re.findall(r"hipLaunchKernelGGL\((.*?)\);", text, re.S)]
    assert len(lds) == text.count("hipLaunchKernelGGL(") and set(lds) <= {"lds", "tile_lds(D)", "msk::kGuardLds"}, lds
