"""ctypes binding of libmoesplit (include/moesplit.h), same names as the C ABI.

Argument marshalling only: every step of the layer runs in the library's HIP
kernels.  Device buffers are passed as torch tensors (their data_ptr()) or raw
integers; streams as torch.cuda.Stream objects, raw handles or None.  The
binding raises ImportError if the built library is missing; there is no
fallback implementation.
"""
from __future__ import annotations

import ctypes
import os

import numpy as np

# MOESPLIT_LIB names another build of the same library (the sanitized host
# build of build.py --sanitize); there is no fallback when it is missing.
_LIB_PATH = os.environ.get("MOESPLIT_LIB") or os.path.join(os.path.dirname(os.path.abspath(__file__)),
                                                          "libmoesplit.so")

MS_OK, MS_E_INVALID, MS_E_BUDGET, MS_E_STATE, MS_E_HIP, MS_E_NOMEM, MS_E_UNSUPPORTED = range(7)
STATUS_NAMES = {0: "MS_OK", 1: "MS_E_INVALID", 2: "MS_E_BUDGET", 3: "MS_E_STATE", 4: "MS_E_HIP",
                5: "MS_E_NOMEM", 6: "MS_E_UNSUPPORTED"}
MS_F32, MS_BF16 = 0, 1
MS_FWD_PREDICT_NEXT = 1
MS_FWD_MATRIX_CORES = 2
MS_FWD_NO_MATRIX_CORES = 4
(MS_IV_ROUTER, MS_IV_GROUP, MS_IV_FFN_RESIDENT, MS_IV_FFN_STREAMED, MS_IV_COMBINE,
 MS_IV_COPY_MISS, MS_IV_COPY_PREFETCH, MS_IV_COPY_TOP, MS_IV_PREDICT, MS_IV_FFN_DOWN) = range(10)
INTERVAL_NAMES = ["router", "group", "ffn_resident", "ffn_streamed", "combine",
                  "copy_miss", "copy_prefetch", "copy_top", "predict", "ffn_down"]


class ms_model_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_int32) for n in (
        "n_layers", "d_model", "d_ff", "n_experts", "top_k", "n_shared", "d_ff_shared",
        "dtype", "renormalize", "max_tokens", "n_buffer_slots", "ffn_splits", "expert_bits")]


class ms_sizes(ctypes.Structure):
    _fields_ = [("chunk_bytes", ctypes.c_uint64), ("n_chunks", ctypes.c_int32),
                ("expert_bytes", ctypes.c_uint64), ("fixed_pool_bytes", ctypes.c_uint64),
                ("buffer_bytes", ctypes.c_uint64)]


class ms_layer_stats(ctypes.Structure):
    _fields_ = [(n, ctypes.c_uint64) for n in (
        "forwards", "tokens", "selected", "experts_active", "alpha", "beta", "gamma",
        "buffer_hits", "bytes_miss", "bytes_prefetch", "bytes_prefetch_used",
        "bytes_prefetch_dropped", "predicted_hits", "predictions", "cache_inserts")]

    def as_dict(self):
        return {n: int(getattr(self, n)) for n, _ in self._fields_}


class ms_plan_problem(ctypes.Structure):
    _fields_ = [("n_layers", ctypes.c_int32), ("n_experts", ctypes.c_int32), ("top_k", ctypes.c_int32),
                ("expert_bytes", ctypes.c_uint64), ("t_att_us", ctypes.c_double), ("t_moe_us", ctypes.c_double),
                ("t_head_us", ctypes.c_double), ("t_load_us", ctypes.c_double),
                ("hit", ctypes.c_void_p), ("pred", ctypes.c_void_p), ("pred_hit", ctypes.c_void_p)]


class ms_kv_cache_q(ctypes.Structure):
    _fields_ = [("k", ctypes.c_void_p), ("v", ctypes.c_void_p), ("k_exp", ctypes.c_void_p), ("v_exp", ctypes.c_void_p),
                ("n_seqs", ctypes.c_int32), ("n_kv_heads", ctypes.c_int32), ("head_dim", ctypes.c_int32),
                ("max_ctx", ctypes.c_int32)]


class ms_rope_desc(ctypes.Structure):
    _fields_ = [(n, ctypes.c_double) for n in ("base", "factor", "orig_ctx", "low", "high", "mscale")] + [
        ("rot_dim", ctypes.c_int32), ("interleaved", ctypes.c_int32)]


class ms_attn_opts(ctypes.Structure):
    _fields_ = [("scale", ctypes.c_float), ("softcap", ctypes.c_float), ("window", ctypes.c_int32),
                ("prefix", ctypes.c_int32), ("slopes_dev", ctypes.c_void_p), ("docs_dev", ctypes.c_void_p)]


class ms_sample_opts(ctypes.Structure):
    _fields_ = [(n, ctypes.c_void_p) for n in ("temperature_dev", "top_k_dev", "top_p_dev", "min_p_dev")]
    rows = None  # of the tensors


MS_CACHE_STATIC, MS_CACHE_LCP, MS_CACHE_LRU, MS_CACHE_LFU, MS_CACHE_RND = range(5)
MS_COPY_KERNEL, MS_COPY_DMA = range(2)


class ms_interval(ctypes.Structure):
    _fields_ = [("kind", ctypes.c_int32), ("layer", ctypes.c_int32), ("t0_ms", ctypes.c_double),
                ("t1_ms", ctypes.c_double), ("bytes", ctypes.c_uint64)]


def _load():
    if not os.path.exists(_LIB_PATH):
        raise ImportError(
            "libmoesplit.so is not built (%s); run __graft_entry__.build() or "
            "python paper_2509_08342_amd/build.py" % _LIB_PATH)
    lib = ctypes.CDLL(_LIB_PATH)
    P, I32, U64, F32 = ctypes.c_void_p, ctypes.c_int32, ctypes.c_uint64, ctypes.c_float
    sig = {
        "ms_query_sizes": [ctypes.POINTER(ms_model_desc), ctypes.POINTER(ms_sizes)],
        "ms_split_plan": [ctypes.POINTER(ms_model_desc), U64, F32, ctypes.POINTER(I32),
                          ctypes.POINTER(U64), ctypes.POINTER(I32)],
        "ms_create": [ctypes.POINTER(ms_model_desc), P, U64, I32, ctypes.POINTER(P)],
        "ms_set_router": [P, I32, P, P],
        "ms_set_expert": [P, I32, I32, P, P, P],
        "ms_set_expert_q": [P, I32, I32, P, P, P, P, P, P],
        "ms_alias_expert": [P, I32, I32, I32, I32],
        "ms_set_shared_expert": [P, I32, I32, P, P, P],
        "ms_configure": [P, P, P, P],
        "ms_load_top": [P, I32, I32],
        "ms_evict_top": [P, I32, I32],
        "ms_residency": [P, I32, P],
        "ms_predict": [P, I32, P, I32, P, P, P],
        "ms_prefetch": [P, I32, P, I32],
        "ms_forward": [P, I32, P, I32, P, P, P, I32, P],
        "ms_forward_noalloc": [P, I32, P, I32, P, P, P, I32, P],
        "ms_sync": [P],
        "ms_drop_buffer": [P],
        "ms_stats": [P, I32, ctypes.POINTER(ms_layer_stats)],
        "ms_reset_stats": [P],
        "ms_residual_norm": [P, P, P, I32, P, P],
        "ms_plan_stats": [P, I32, P, P, P, P],
        "ms_reset_plan_stats": [P],
        "ms_lcp_priority": [P, I32, P],
        "ms_plan_solve": [ctypes.POINTER(ms_plan_problem), U64, ctypes.c_double, P, I32, P, P, P, P, P],
        "ms_cache_update": [P, P, P],
        "ms_set_cache_policy": [P, I32, ctypes.c_double, ctypes.c_double, U64],
        "ms_set_copy_engine": [P, I32],
        "ms_dense": [P, P, I32, I32, I32, P, P, P],
        "ms_rope_kv": [P, I32, I32, I32, I32, I32, ctypes.c_double, P, P, P, I32, P],
        "ms_attention": [P, P, P, I32, I32, I32, I32, I32, I32, P, P],
        "ms_argmax": [P, I32, I32, P, P],
        "ms_embed": [P, P, I32, I32, I32, P, P],
        "ms_rope_kv_q": [ctypes.POINTER(ms_kv_cache_q), ctypes.POINTER(ms_rope_desc), P, I32, I32, I32, P, P, P],
        "ms_kv_read_q": [ctypes.POINTER(ms_kv_cache_q), I32, I32, P, P, P],
        "ms_attention_q_workspace": [ctypes.POINTER(ms_kv_cache_q), I32, I32, I32, ctypes.POINTER(U64)],
        "ms_attention_q": [ctypes.POINTER(ms_kv_cache_q), P, I32, I32, I32, P, ctypes.POINTER(ms_attn_opts), P, P, U64, P],
        "ms_quant_q": [P, I32, I32, I32, I32, P, P, P],
        "ms_residual_norm_q": [P, P, I32, P, ctypes.c_double, I32, I32, P, P, P, P, P],
        "ms_dense_q": [P, P, P, P, I32, I32, I32, P, I32, P, P],
        "ms_sample_workspace": [I32, I32, ctypes.POINTER(U64)],
        "ms_sample": [P, I32, I32, ctypes.POINTER(ms_sample_opts), P, P, P, P, U64, P],
        "ms_timeline_begin": [P, P, I32],
        "ms_timeline_end": [P, ctypes.POINTER(ms_interval), I32, ctypes.POINTER(I32)],
    }
    for name, args in sig.items():
        fn = getattr(lib, name)
        fn.argtypes = args
        fn.restype = ctypes.c_int
    lib.ms_destroy.argtypes = [P]
    lib.ms_destroy.restype = None
    lib.ms_last_error.argtypes = [P]
    lib.ms_last_error.restype = ctypes.c_char_p
    return lib


lib = _load()


class MoeSplitError(RuntimeError):
    def __init__(self, status, msg):
        super().__init__("%s: %s" % (STATUS_NAMES.get(status, status), msg))
        self.status = status


def _ptr(x):
    """Device/host address of a tensor, numpy array or integer (None -> NULL)."""
    if x is None:
        return None
    address = getattr(x, "data_ptr", None)  # a tensor
    if address is not None:
        assert x.is_contiguous()
        return address()
    if isinstance(x, int):
        return x
    if isinstance(x, np.ndarray):
        assert x.flags.c_contiguous
        return x.ctypes.data
    raise TypeError("cannot take the address of %r" % type(x))


def _stream(s):
    if s is None:
        return None
    if isinstance(s, int):
        return s
    return s.cuda_stream


def model_desc(shape, max_tokens, n_buffer_slots=0, ffn_splits=0):
    """ms_model_desc from a synth.ModelShape-like object."""
    return ms_model_desc(shape.n_layers, shape.d_model, shape.d_ff, shape.n_experts, shape.top_k,
                         shape.n_shared, shape.d_ff_shared,
                         MS_BF16 if shape.dtype == "bf16" else MS_F32, shape.renormalize,
                         max_tokens, n_buffer_slots, ffn_splits, getattr(shape, "expert_bits", 0))


def _check(st, ctx=None, what=""):
    if st != MS_OK:
        msg = lib.ms_last_error(ctx).decode() if ctx else what
        raise MoeSplitError(st, msg or what)


# --------------------------------------------------------------- functions

def ms_query_sizes(desc):
    out = ms_sizes()
    _check(lib.ms_query_sizes(ctypes.byref(desc), ctypes.byref(out)), what="ms_query_sizes")
    return out


def ms_split_plan(desc, budget_bytes, r):
    units, tb, slots = ctypes.c_int32(), ctypes.c_uint64(), ctypes.c_int32()
    _check(lib.ms_split_plan(ctypes.byref(desc), int(budget_bytes), float(r), ctypes.byref(units),
                             ctypes.byref(tb), ctypes.byref(slots)), what="ms_split_plan")
    return units.value, tb.value, slots.value


def ms_create(desc, dev_pool, pool_bytes, host_store_experts=0):
    h = ctypes.c_void_p()
    _check(lib.ms_create(ctypes.byref(desc), _ptr(dev_pool), int(pool_bytes), int(host_store_experts),
                         ctypes.byref(h)), what="ms_create")
    return h


def ms_destroy(ctx):
    lib.ms_destroy(ctx)


def ms_last_error(ctx):
    return lib.ms_last_error(ctx).decode()


def ms_set_router(ctx, layer, w_r, bias=None):
    w_r = np.ascontiguousarray(w_r)
    b = None if bias is None else np.ascontiguousarray(bias, np.float32)
    _check(lib.ms_set_router(ctx, layer, _ptr(w_r), _ptr(b)), ctx)


def ms_set_expert(ctx, layer, e, w_gate, w_up, w_down):
    arrs = [np.ascontiguousarray(a) for a in (w_gate, w_up, w_down)]
    _check(lib.ms_set_expert(ctx, layer, e, *[_ptr(a) for a in arrs]), ctx)


def ms_set_expert_q(ctx, layer, e, codes, meta):
    """codes: (gate [F][d*b/8], up [F][d*b/8], down [d][F*b/8]) uint8;
    meta: (gate [F][d/64][2], up, down [d][F/64][2]) uint16 fp16 patterns."""
    cs = [np.ascontiguousarray(a, np.uint8) for a in codes]
    ms_ = [np.ascontiguousarray(a, np.uint16) for a in meta]
    _check(lib.ms_set_expert_q(ctx, layer, e, _ptr(cs[0]), _ptr(ms_[0]), _ptr(cs[1]), _ptr(ms_[1]),
                               _ptr(cs[2]), _ptr(ms_[2])), ctx)


def ms_alias_expert(ctx, layer, e, src_layer, src_e):
    _check(lib.ms_alias_expert(ctx, layer, e, src_layer, src_e), ctx)


def ms_set_shared_expert(ctx, layer, s, w_gate, w_up, w_down):
    arrs = [np.ascontiguousarray(a) for a in (w_gate, w_up, w_down)]
    _check(lib.ms_set_shared_expert(ctx, layer, s, *[_ptr(a) for a in arrs]), ctx)


def ms_configure(ctx, budget_bytes, r):
    b = np.ascontiguousarray(budget_bytes, np.uint64)
    rr = np.ascontiguousarray(r, np.float32)
    slots = np.zeros(len(b), np.int32)
    _check(lib.ms_configure(ctx, _ptr(b), _ptr(rr), _ptr(slots)), ctx)
    return slots


def ms_load_top(ctx, layer, e):
    _check(lib.ms_load_top(ctx, layer, e), ctx)


def ms_evict_top(ctx, layer, e):
    _check(lib.ms_evict_top(ctx, layer, e), ctx)


def ms_residency(ctx, layer, n_experts):
    out = np.zeros(n_experts, np.uint8)
    _check(lib.ms_residency(ctx, layer, _ptr(out)), ctx)
    return out


def ms_predict(ctx, layer, h_dev, T, stream, n_experts):
    order = np.zeros(n_experts, np.int32)
    score = np.zeros(n_experts, np.float32)
    _check(lib.ms_predict(ctx, layer, _ptr(h_dev), T, _stream(stream), _ptr(order), _ptr(score)), ctx)
    return order, score


def ms_prefetch(ctx, layer, experts):
    ex = np.ascontiguousarray(experts, np.int32)
    _check(lib.ms_prefetch(ctx, layer, _ptr(ex), len(ex)), ctx)


def ms_forward(ctx, layer, h_dev, T, y_dev, idx_dev, w_dev, flags=0, stream=None):
    _check(lib.ms_forward(ctx, layer, _ptr(h_dev), T, _ptr(y_dev), _ptr(idx_dev), _ptr(w_dev), flags,
                          _stream(stream)), ctx)


def ms_forward_noalloc(ctx, layer, h_dev, T, y_dev, idx_dev, w_dev, flags=0, stream=None):
    _check(lib.ms_forward_noalloc(ctx, layer, _ptr(h_dev), T, _ptr(y_dev), _ptr(idx_dev), _ptr(w_dev), flags,
                                  _stream(stream)), ctx)


def ms_sync(ctx):
    _check(lib.ms_sync(ctx), ctx)


def ms_drop_buffer(ctx):
    _check(lib.ms_drop_buffer(ctx), ctx)


def ms_residual_norm(ctx, h_dev, y_dev, T, out_dev, stream=None):
    _check(lib.ms_residual_norm(ctx, _ptr(h_dev), _ptr(y_dev), T, _ptr(out_dev), _stream(stream)), ctx)


def ms_plan_stats(ctx, layer, n_experts):
    """(hit [N+1], pred [N], pred_hit [N][N+1], (q, q_pred)) of one layer."""
    N = n_experts
    hit = np.zeros(N + 1)
    pred = np.zeros(N)
    ph = np.zeros((N, N + 1))
    tok = np.zeros(2, np.uint64)
    _check(lib.ms_plan_stats(ctx, layer, _ptr(hit), _ptr(pred), _ptr(ph), _ptr(tok)), ctx)
    return hit, pred, ph, (int(tok[0]), int(tok[1]))


def ms_reset_plan_stats(ctx):
    _check(lib.ms_reset_plan_stats(ctx), ctx)


def ms_lcp_priority(ctx, layer, n_experts):
    out = np.zeros(n_experts)
    _check(lib.ms_lcp_priority(ctx, layer, _ptr(out)), ctx)
    return out


def ms_plan_solve(n_layers, n_experts, top_k, expert_bytes, t_att_us, t_moe_us, t_head_us, t_load_us,
                  hit, pred, pred_hit, v_e_bytes, zeta=0.01, start_budgets=None, max_iter=100000):
    """Algorithm 1 over per-layer statistics (arrays [L][N+1], [L][N],
    [L][N][N+1]); returns dict(budgets, theta, cache, exposed_us, iters)."""
    L, N = n_layers, n_experts
    hit = np.ascontiguousarray(hit, np.float64).reshape(L, N + 1)
    pred = np.ascontiguousarray(pred, np.float64).reshape(L, N)
    pred_hit = np.ascontiguousarray(pred_hit, np.float64).reshape(L, N, N + 1)
    prob = ms_plan_problem(L, N, top_k, int(expert_bytes), float(t_att_us), float(t_moe_us), float(t_head_us),
                           float(t_load_us), hit.ctypes.data, pred.ctypes.data, pred_hit.ctypes.data)
    start = None if start_budgets is None else np.ascontiguousarray(start_budgets, np.uint64)
    budgets = np.zeros(L, np.uint64)
    theta = np.zeros(L)
    cache = np.zeros(L, np.int32)
    exposed = np.zeros(L)
    iters = ctypes.c_int32()
    _check(lib.ms_plan_solve(ctypes.byref(prob), int(v_e_bytes), float(zeta), _ptr(start), int(max_iter),
                             _ptr(budgets), _ptr(theta), _ptr(cache), _ptr(exposed), ctypes.byref(iters)),
           what="ms_plan_solve")
    return dict(budgets=budgets, theta=theta, cache=cache, exposed_us=exposed, iters=iters.value)


def ms_cache_update(ctx, budgets, r):
    b = np.ascontiguousarray(budgets, np.uint64)
    rr = np.ascontiguousarray(r, np.float32)
    _check(lib.ms_cache_update(ctx, _ptr(b), _ptr(rr)), ctx)


def ms_set_cache_policy(ctx, policy, rho=0.25, omega=128.0, seed=0):
    _check(lib.ms_set_cache_policy(ctx, int(policy), float(rho), float(omega), int(seed)), ctx)


def ms_set_copy_engine(ctx, engine):
    _check(lib.ms_set_copy_engine(ctx, int(engine)), ctx)


def ms_stats(ctx, layer):
    out = ms_layer_stats()
    _check(lib.ms_stats(ctx, layer, ctypes.byref(out)), ctx)
    return out.as_dict()


def ms_reset_stats(ctx):
    _check(lib.ms_reset_stats(ctx), ctx)


def ms_timeline_begin(ctx, stream, capacity=1 << 16):
    _check(lib.ms_timeline_begin(ctx, _stream(stream), capacity), ctx)


def ms_timeline_end(ctx, cap=1 << 16):
    buf = (ms_interval * cap)()
    n = ctypes.c_int32()
    _check(lib.ms_timeline_end(ctx, buf, cap, ctypes.byref(n)), ctx)
    return [dict(kind=INTERVAL_NAMES[buf[i].kind], layer=buf[i].layer, t0_ms=buf[i].t0_ms,
                 t1_ms=buf[i].t1_ms, bytes=int(buf[i].bytes)) for i in range(n.value)]


# ------------------------------------------------- decoder loop (stateless)

def ms_dense(x, w, T, n_in, n_out, y, add=None, stream=None):
    _check(lib.ms_dense(_ptr(x), _ptr(w), int(T), int(n_in), int(n_out), _ptr(y),
                        None if add is None else _ptr(add), _stream(stream)), what="ms_dense")


def ms_rope_kv(qkv, T, Hq, Hkv, D, pos0, base, q_out, k_cache, v_cache, max_ctx, stream=None):
    _check(lib.ms_rope_kv(_ptr(qkv), int(T), int(Hq), int(Hkv), int(D), int(pos0), float(base), _ptr(q_out),
                          _ptr(k_cache), _ptr(v_cache), int(max_ctx), _stream(stream)), what="ms_rope_kv")


def ms_attention(q, k_cache, v_cache, T, Hq, Hkv, D, pos0, max_ctx, out, stream=None):
    _check(lib.ms_attention(_ptr(q), _ptr(k_cache), _ptr(v_cache), int(T), int(Hq), int(Hkv), int(D), int(pos0),
                            int(max_ctx), _ptr(out), _stream(stream)), what="ms_attention")


def ms_argmax(x, T, n, idx_out, stream=None):
    _check(lib.ms_argmax(_ptr(x), int(T), int(n), _ptr(idx_out), _stream(stream)), what="ms_argmax")


def ms_embed(ids, table, n_vocab, T, d, out, stream=None):
    _check(lib.ms_embed(_ptr(ids), _ptr(table), int(n_vocab), int(T), int(d), _ptr(out), _stream(stream)),
           what="ms_embed")


# --------------------------------------------------- 8-bit key/value cache

KV_BLOCK = 64  # positions that share a scale


def kv_cache_q(k, v, k_exp, v_exp):
    """ms_kv_cache_q of uint8 tensors: codes [n_seqs][Hkv][max_ctx][D] and
    exponents [n_seqs][Hkv][max_ctx / 64] (new_kv_cache_q allocates them).  The
    struct keeps the tensors alive."""
    S, Hkv, ctx, D = k.shape
    for x, shape in ((k, (S, Hkv, ctx, D)), (v, (S, Hkv, ctx, D)), (k_exp, (S, Hkv, ctx // KV_BLOCK)),
                     (v_exp, (S, Hkv, ctx // KV_BLOCK))):
        if tuple(x.shape) != shape or x.element_size() != 1:
            raise ValueError("kv_cache_q: one-byte tensors of %r and %r expected" % ((S, Hkv, ctx, D),
                                                                                 (S, Hkv, ctx // KV_BLOCK)))
    c = ms_kv_cache_q(_ptr(k), _ptr(v), _ptr(k_exp), _ptr(v_exp), S, Hkv, D, ctx)
    c.tensors = (k, v, k_exp, v_exp)
    return c


def new_kv_cache_q(n_seqs, n_kv_heads, head_dim, max_ctx, device="cuda"):
    """A zeroed 8-bit cache (max_ctx a multiple of 64)."""
    import torch
    codes = [torch.zeros(n_seqs, n_kv_heads, max_ctx, head_dim, dtype=torch.uint8, device=device) for _ in range(2)]
    exps = [torch.full((n_seqs, n_kv_heads, max_ctx // KV_BLOCK), 127, dtype=torch.uint8, device=device)
            for _ in range(2)]
    return kv_cache_q(*codes, *exps)


def rope_desc(rot_dim, base, interleaved=False, factor=1.0, orig_ctx=0.0, low=1.0, high=32.0, mscale=1.0):
    return ms_rope_desc(float(base), float(factor), float(orig_ctx), float(low), float(high), float(mscale),
                        int(rot_dim), int(bool(interleaved)))


def attn_opts(scale=0.0, softcap=0.0, window=0, prefix=0, slopes=None, doc=None):
    """slopes: device fp32 [Hq]; doc: device int32 [n_seqs][max_ctx]."""
    for x, name in ((slopes, "torch.float32"), (doc, "torch.int32")):
        if x is not None and str(getattr(x, "dtype", name)) != name:
            raise ValueError("attn_opts: %s expected" % name)
    o = ms_attn_opts(float(scale), float(softcap), int(window), int(prefix), _ptr(slopes), _ptr(doc))
    o.tensors = (slopes, doc)
    return o


def _span(x, cache):
    if str(getattr(x, "dtype", "torch.int32")) != "torch.int32":
        raise ValueError("span: torch.int32 expected")
    if cache is not None and getattr(x, "shape", None) not in (None, (cache.n_seqs, 2)):
        raise ValueError("span: [%d][2] expected" % cache.n_seqs)
    return _ptr(x)


class _Values(dict):
    """Bytes of a value by the type of the tensor that holds it; without end for types that hold other values (a type's
    name is looked at once)."""

    def __init__(self, size, *names):
        super().__init__()
        self.size, self.names = size, names

    def __missing__(self, dtype):
        self[dtype] = size = self.size if str(dtype) in self.names else float("inf")
        return size


_F32, _BF16, _I32 = _Values(4, "torch.float32"), _Values(2, "torch.bfloat16"), _Values(4, "torch.int32")
_CODES = _Values(1, "torch.uint8", "torch.int8", "torch.float8_e4m3fn")
_EXPONENTS = _Values(1, "torch.uint8", "torch.float8_e8m0fnu")


def _rows(x, name, kind, values):
    """x's address; a tensor is contiguous and holds at least `values` of a kind (_Values), in whatever shape."""
    try:
        if x.is_contiguous() and x.nbytes >= values * kind[x.dtype]:  # (none of a size without end: NaN)
            return x.data_ptr()
    except AttributeError:  # an address
        return _ptr(x)
    raise ValueError("%s: %d contiguous values of %s expected" % (name, values, " or ".join(kind.names)))


def ms_rope_kv_q(cache, rope, qkv, T, Hq, pos0, q_out, span=None, stream=None):
    n, kv = (cache.n_seqs * T * cache.head_dim, 2 * cache.n_kv_heads) if cache is not None else (0, 0)
    st = lib.ms_rope_kv_q(cache, rope, _rows(qkv, "qkv", _F32, n * (Hq + kv)), T, Hq, pos0,
                          None if span is None else _span(span, cache), _rows(q_out, "q_out", _BF16, n * Hq), _stream(stream))
    if st:
        _check(st, what="ms_rope_kv_q")


def ms_kv_read_q(cache, pos0, n, k_out, v_out, stream=None):
    values = cache.n_seqs * n * cache.head_dim * cache.n_kv_heads if cache is not None else 0
    st = lib.ms_kv_read_q(cache, pos0, n, _rows(k_out, "k_out", _BF16, values), _rows(v_out, "v_out", _BF16, values), _stream(stream))
    if st:
        _check(st, what="ms_kv_read_q")


def ms_attention_q_workspace(cache, T, Hq, pos0):
    n = ctypes.c_uint64()
    _check(lib.ms_attention_q_workspace(cache, T, Hq, pos0, ctypes.byref(n)), what="ms_attention_q_workspace")
    return n.value


def ms_attention_q(cache, q, T, Hq, pos0, out, workspace=None, opts=None, span=None, stream=None):
    """workspace: a device tensor of at least ms_attention_q_workspace bytes."""
    n = cache.n_seqs * T * cache.head_dim * Hq if cache is not None else 0
    if opts is not None and cache is not None:
        slopes, doc = getattr(opts, "tensors", (None, None))
        if slopes is not None and getattr(slopes, "shape", None) not in (None, (Hq,)):
            raise ValueError("attn_opts: slopes of %r expected" % ((Hq,),))
        if doc is not None and getattr(doc, "shape", None) not in (None, (cache.n_seqs, cache.max_ctx)):
            raise ValueError("attn_opts: doc of %r expected" % ((cache.n_seqs, cache.max_ctx),))
    st = lib.ms_attention_q(cache, _rows(q, "q", _BF16, n), T, Hq, pos0, None if span is None else _span(span, cache), opts,
                            _rows(out, "out", _BF16, n), _ptr(workspace), 0 if workspace is None else workspace.nbytes,
                            _stream(stream))
    if st:
        _check(st, what="ms_attention_q")


# ------------------------------------------------- the dense path in 8 bits

BLOCK_Q = 128  # columns that share a scale, and rows of a weight's block

_VALUE_TYPES = {"torch.float32": (MS_F32, _F32), "torch.bfloat16": (MS_BF16, _BF16)}


def _value_type(x, name):
    """(MS_F32 or MS_BF16, its kind) of a tensor."""
    try:
        t = _VALUE_TYPES.get(x.dtype)
        if t is None:  # the first of its type
            t = _VALUE_TYPES[x.dtype] = _VALUE_TYPES[str(x.dtype)]
        return t
    except (AttributeError, KeyError):
        raise ValueError("%s: a float32 or bfloat16 tensor expected" % name) from None


def new_matrix_q(rows, n, block_rows=1, device="cuda"):
    """(codes [rows][n], exponents) of a matrix in 8 bits; block_rows 1, or 128 for weights."""
    import torch
    return (torch.empty(rows, n, dtype=torch.uint8, device=device),
            torch.empty(-(-rows // block_rows), -(-n // BLOCK_Q), dtype=torch.uint8, device=device))


def _blocks(n):
    return -(-n // BLOCK_Q)


def ms_quant_q(x, rows, n, block_rows, codes, exps, stream=None):
    dtype, kind = _value_type(x, "x")
    st = lib.ms_quant_q(_rows(x, "x", kind, rows * n), dtype, rows, n, block_rows, _rows(codes, "codes", _CODES, rows * n),
                        _rows(exps, "exps", _EXPONENTS, -(-rows // max(block_rows, 1)) * _blocks(n)), _stream(stream))
    if st:
        _check(st, what="ms_quant_q")


def ms_residual_norm_q(h, y, weight, eps, T, d, sum_out=None, out=None, codes=None, exps=None, stream=None):
    dtype, kind = (MS_F32, _F32) if y is None else _value_type(y, "y")
    n = T * d
    st = lib.ms_residual_norm_q(_rows(h, "h", _BF16, n), None if y is None else _rows(y, "y", kind, n), dtype,
                                None if weight is None else _rows(weight, "weight", _BF16, d), eps, T, d,
                                None if sum_out is None else _rows(sum_out, "sum_out", _BF16, n),
                                None if out is None else _rows(out, "out", _BF16, n),
                                None if codes is None else _rows(codes, "codes", _CODES, n),
                                None if exps is None else _rows(exps, "exps", _EXPONENTS, T * _blocks(d)), _stream(stream))
    if st:
        _check(st, what="ms_residual_norm_q")


def ms_dense_q(x, x_exp, w, w_exp, T, n_in, n_out, y, add=None, stream=None):
    """y (and add): float32 or bfloat16."""
    dtype, kind = _value_type(y, "y")
    if add is not None and add.dtype != y.dtype:
        raise ValueError("add: the type of y expected")
    st = lib.ms_dense_q(_rows(x, "x", _CODES, T * n_in), _rows(x_exp, "x_exp", _EXPONENTS, T * _blocks(n_in)), _rows(w, "w", _CODES, n_out * n_in),
                        _rows(w_exp, "w_exp", _EXPONENTS, _blocks(n_out) * _blocks(n_in)), T, n_in, n_out, _rows(y, "y", kind, T * n_out),
                        dtype, None if add is None else _rows(add, "add", kind, T * n_out), _stream(stream))
    if st:
        _check(st, what="ms_dense_q")


# ---------------------------------------------------------------- sampling

def sample_opts(temperature=None, top_k=None, top_p=None, min_p=None):
    """Settings of every row: device tensors [T], float32 (top_k: int32), or None."""
    ts = (temperature, top_k, top_p, min_p)
    for x, name in zip(ts, ("torch.float32", "torch.int32", "torch.float32", "torch.float32")):
        if x is not None and str(getattr(x, "dtype", name)) != name:
            raise ValueError("sample_opts: %s expected" % name)
    shapes = {tuple(x.shape) for x in ts if hasattr(x, "shape")}
    if len(shapes) > 1 or any(len(x) != 1 for x in shapes):
        raise ValueError("sample_opts: a value per row expected")
    o = ms_sample_opts(*[_ptr(x) for x in ts])
    for rows, in shapes:
        o.rows = rows
    o.tensors = ts
    return o


def ms_sample_workspace(T, n):
    out = ctypes.c_uint64()
    _check(lib.ms_sample_workspace(T, n, ctypes.byref(out)), what="ms_sample_workspace")
    return out.value


def ms_sample(logits, T, n, opts, u, idx_out, prob_out=None, workspace=None, stream=None):
    """workspace: a device tensor of at least ms_sample_workspace bytes."""
    if opts is not None and opts.rows not in (None, T):
        raise ValueError("sample_opts: [%d] expected" % T)
    st = lib.ms_sample(_rows(logits, "logits", _F32, T * n), T, n, opts, _rows(u, "u", _F32, T), _rows(idx_out, "idx_out", _I32, T),
                       None if prob_out is None else _rows(prob_out, "prob_out", _F32, T), _ptr(workspace),
                       0 if workspace is None else workspace.nbytes, _stream(stream))
    if st:
        _check(st, what="ms_sample")
