"""The operators of the decoder loop's dense path in 8 bits and of its token:
blocks of e4m3 codes made from rows (ms_quant_q), the residual's addition and
root-mean-square norm with an output in such blocks (ms_residual_norm_q), the
matrix product of two of them (ms_dense_q), and a token drawn from logits
(ms_sample), as plain torch operations and as the library's calls.

A matrix in 8 bits holds e4m3 codes and a power of two for every 128 columns
of a row (activations) or of 128 rows (weights).  Sizes are those of the
repository's decoder (width 4096, 6144 outputs for queries, keys and values,
32000 tokens in the vocabulary), of its other layers (width 2048, 1408) and
generic ones.
"""
import math

import torch

own = False

BLOCK = 128
EXP_BIAS, EXP_MIN, EXP_MAX = 127, -40, 40
LARGEST = 448.0  # of e4m3
EPS = 1e-6
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


def listed():
    return [
        # the attention's output of one token, on its way to the output projection
        quant("quant-token", 1, 4096, "bf16", 1),
        # the head's weights, once when a model is loaded
        quant("quant-head", 32000, 4096, "bf16", 128),
        # between the modules of a layer: one decode token; a prompt, with a gain and the running sum kept
        norm("norm-token", 1, 4096, "f32"),
        norm("norm-prompt2048", 2048, 4096, "bf16", gain=True, total=True),
        # a decode token's queries, keys and values, and its logits
        dense("dense-token-qkv", 1, 4096, 6144, "f32"),
        dense("dense-token-head", 1, 4096, 32000, "f32"),
        # a decode batch over odd widths (the last block of 128 is not full), added to what is there
        dense("dense-batch61", 61, 2000, 5003, "f32", add=True),
        # prompts: results for the rotation in fp32; a wide projection whose results go on in bf16
        dense("dense-prompt2048-qkv", 2048, 4096, 6144, "f32"),
        dense("dense-prompt4096-wide", 4096, 4096, 14336, "bf16"),
        # one token of a chat; a serving batch whose rows have settings of their own; many rows of pure temperature
        sample("sample-token", 1, 32000, top_k=50, top_p=0.9),
        sample("sample-batch64", 64, 131071, top_k=1000, top_p=0.95, min_p=0.01, mixed=True),
        sample("sample-rows500", 500, 32000, min_p=0.02),
    ]


def named(name, **c):
    return dict(name=name, **c) if name else c


def quant(name, rows, n, dtype, block_rows):
    return named(name, kind="quant", rows=rows, n=n, dtype=dtype, block_rows=block_rows)


def norm(name, T, d, dtype, gain=False, total=False):
    return named(name, kind="norm", T=T, d=d, dtype=dtype, gain=gain, total=total)


def dense(name, T, n_in, n_out, dtype, add=False):
    return named(name, kind="dense", T=T, n_in=n_in, n_out=n_out, dtype=dtype, add=add)


def sample(name, T, n, top_k=0, top_p=1.0, min_p=0.0, mixed=False):
    return named(name, kind="sample", T=T, n=n, top_k=top_k, top_p=top_p, min_p=min_p, mixed=mixed)


def draw(rng):
    """Rows of 16 to 8192 values, one to 4096 of them (weights: up to 32000);
    products of one to 4096 tokens; tokens from vocabularies of 100 to 200000."""
    def log_uniform(lo, hi):
        return min(hi, int(math.exp(rng.uniform(math.log(lo), math.log(hi + 1)))))

    def width(lo, hi):  # in steps of 16: rows start at 16 bytes
        return 16 * log_uniform(lo // 16, hi // 16)

    kind = rng.random()
    dtype = rng.choice(["bf16", "f32"])
    if kind < 0.15:
        block_rows = rng.choice([1, 128])
        n = width(16, 8192)
        return quant(None, log_uniform(1, min(32000, (1 << 26) // n)), n, dtype, block_rows)
    if kind < 0.35:
        d = width(256, 8192)
        return norm(None, rng.choice([1, log_uniform(2, min(4096, (1 << 24) // d))]), d, dtype, gain=rng.random() < 0.5,
                    total=rng.random() < 0.5)
    if kind < 0.7:
        T, n_in = rng.choice([1, log_uniform(2, 4096), log_uniform(2, 4096)]), width(128, 8192)
        most = min(32000, 4096 * 4096 * 14336 // (T * n_in))
        return dense(None, T, n_in, log_uniform(min(64, most), most), dtype, add=rng.random() < 0.4)
    T = rng.choice([1, log_uniform(2, 512)])
    n = log_uniform(100, min(200000, (1 << 24) // T))
    return sample(None, T, n, top_k=rng.choice([0, 0, log_uniform(1, 2000)]), top_p=rng.choice([1.0, 0.5, 0.9, 0.99]),
                  min_p=rng.choice([0.0, 0.0, 0.01, 0.1]), mixed=rng.random() < 0.4)


# ------------------------------------------------------------------ inputs

def prepare(case, seed):
    gen = torch.Generator(device="cuda")
    gen.manual_seed(0x0DE85E00 + seed)

    def normal(*shape):
        return torch.empty(shape, dtype=torch.float32, device="cuda").normal_(0.0, 1.0, generator=gen)

    def uniform(*shape):
        return torch.rand(shape, dtype=torch.float32, device="cuda", generator=gen)

    def rows(T, d):
        """Activations: a few channels are many times the others."""
        return normal(T, d) * torch.where(uniform(d) < 0.01, 12.0, 1.0)

    st = dict(case=case)
    if case["kind"] == "quant":
        R, n, b = case["rows"], case["n"], case["block_rows"]
        x = normal(R, n).mul_(0.02) if b > 1 else rows(R, n)
        st["x"] = x.to(DTYPES[case["dtype"]])
        st.update(blocks(R, n, b))
    elif case["kind"] == "norm":
        T, d = case["T"], case["d"]
        st["h"], st["y"] = rows(T, d).to(torch.bfloat16), (0.5 * normal(T, d)).to(DTYPES[case["dtype"]])
        st["gain"] = (1.0 + 0.2 * normal(d)).to(torch.bfloat16) if case["gain"] else None
        st["out"] = torch.empty(T, d, dtype=torch.bfloat16, device="cuda")
        st["sum"] = torch.empty(T, d, dtype=torch.bfloat16, device="cuda") if case["total"] else None
        st.update(blocks(T, d, 1))
    elif case["kind"] == "dense":
        T, n_in, n_out = case["T"], case["n_in"], case["n_out"]
        st["x"], st["x_exp"] = encoded(rows(T, n_in), 1)
        st["w"], st["w_exp"] = encoded(normal(n_out, n_in).mul_(0.02), BLOCK)
        st["add"] = normal(T, n_out).to(DTYPES[case["dtype"]]) if case["add"] else None
        st["y"] = torch.empty(T, n_out, dtype=DTYPES[case["dtype"]], device="cuda")
    else:
        T, n = case["T"], case["n"]
        st["logits"] = 2.5 * normal(T, n)
        st["logits"] += torch.where(uniform(T, n) < 20.0 / n, 8.0, 0.0)  # the words that fit
        st["u"] = uniform(T)
        row = torch.arange(T, device="cuda")
        st["temperature"] = 0.7 + 0.6 * uniform(T)
        top_k = torch.full((T,), case["top_k"], dtype=torch.int32, device="cuda")
        top_p, min_p = (torch.full((T,), case[x], dtype=torch.float32, device="cuda") for x in ("top_p", "min_p"))
        if case["mixed"]:  # one row in four greedy, and filters off in some
            st["temperature"][row % 4 == 3] = 0.0
            top_k[row % 3 == 1], top_p[row % 5 == 1], min_p[row % 2 == 0] = 0, 1.0, 0.0
        st["top_k"], st["top_p"], st["min_p"] = top_k, top_p, min_p
        st["idx"] = torch.empty(T, dtype=torch.int32, device="cuda")
        st["prob"] = torch.empty(T, dtype=torch.float32, device="cuda")
    if own:
        st["handle"] = handle(st)
    return st


def blocks(rows, n, block_rows):
    return dict(codes=torch.empty(rows, n, dtype=torch.float8_e4m3fn, device="cuda"),
                exps=torch.empty(-(-rows // block_rows), -(-n // BLOCK), dtype=torch.uint8, device="cuda"))


def encoded(x, block_rows):
    """x [rows][n] as e4m3 codes and a stored exponent for every block: the
    least e in range with the block's largest magnitude at most 448 * 2^e."""
    R, n = x.shape
    a = torch.nn.functional.pad(x.abs(), (0, -n % BLOCK, 0, -R % block_rows))
    a = a.view(-(-R // block_rows), block_rows, -(-n // BLOCK), BLOCK).amax(dim=(1, 3))
    m, e = torch.frexp(a)
    e = e - 9 + (m > 0.875).to(e.dtype)  # 448 = 0.875 * 2^9
    e = torch.where(a == 0, EXP_MIN, e).clamp(EXP_MIN, EXP_MAX)
    scaled = x * spread(e, n, R, block_rows, -1).to(x.dtype)
    return scaled.clamp(-LARGEST, LARGEST).to(torch.float8_e4m3fn), (e + EXP_BIAS).to(torch.uint8)


def spread(e, n, rows, block_rows, sign=1):
    """2^(sign e) of every value, from exponents of blocks (powers from their bits)."""
    p = ((sign * e.to(torch.int32) + 127) << 23).view(torch.float32)
    return p.repeat_interleave(block_rows, 0)[:rows].repeat_interleave(BLOCK, 1)[:, :n]


def values(c, e, block_rows):
    """codes [rows][n] and stored exponents -> fp32"""
    return c.to(torch.float32) * spread(e.to(torch.int32) - EXP_BIAS, c.shape[1], c.shape[0], block_rows)


# --------------------------------------------------------------- the calls

def handle(st):
    """What a program that makes these calls keeps."""
    from paper_2509_08342_amd import moesplit as ms
    h = dict(ms=ms)
    if st["case"]["kind"] == "sample":
        T, n = st["logits"].shape
        h["opts"] = ms.sample_opts(st["temperature"], st["top_k"], st["top_p"], st["min_p"])
        h["workspace"] = torch.empty(max(ms.ms_sample_workspace(T, n), 16), dtype=torch.uint8, device="cuda")
    return h


def run(st):
    kind = st["case"]["kind"]
    if own:
        return dict(quant=own_quant, norm=own_norm, dense=own_dense, sample=own_sample)[kind](st)
    return dict(quant=run_quant, norm=run_norm, dense=run_dense, sample=run_sample)[kind](st)


def own_quant(st):
    c = st["case"]
    st["handle"]["ms"].ms_quant_q(st["x"], c["rows"], c["n"], c["block_rows"], st["codes"], st["exps"],
                                  stream=torch.cuda.current_stream())
    return dict(codes=st["codes"], exps=st["exps"])


def own_norm(st):
    c = st["case"]
    st["handle"]["ms"].ms_residual_norm_q(st["h"], st["y"], st["gain"], EPS, c["T"], c["d"], sum_out=st["sum"],
                                          out=st["out"], codes=st["codes"], exps=st["exps"],
                                          stream=torch.cuda.current_stream())
    return dict(sum=st["sum"], out=st["out"], codes=st["codes"], exps=st["exps"])


def own_dense(st):
    c = st["case"]
    st["handle"]["ms"].ms_dense_q(st["x"], st["x_exp"], st["w"], st["w_exp"], c["T"], c["n_in"], c["n_out"], st["y"],
                                  add=st["add"], stream=torch.cuda.current_stream())
    return st["y"]


def own_sample(st):
    h = st["handle"]
    T, n = st["logits"].shape
    h["ms"].ms_sample(st["logits"], T, n, h["opts"], st["u"], st["idx"], st["prob"], h["workspace"],
                      stream=torch.cuda.current_stream())
    return dict(idx=st["idx"], prob=st["prob"])


# ------------------------------------------------------------- plain forms

def run_quant(st):
    codes, exps = encoded(st["x"].float(), st["case"]["block_rows"])
    return dict(codes=codes, exps=exps)


def run_norm(st):
    # in 64 bits: a block's largest value may lie next to a power of two, a value halfway between two codes
    x = st["h"].double() + st["y"].double()
    v = x * torch.rsqrt(x.square().mean(dim=1, keepdim=True) + EPS)
    if st["gain"] is not None:
        v = v * st["gain"].double()
    codes, exps = encoded(v, 1)
    return dict(sum=x.to(torch.bfloat16) if st["case"]["total"] else None, out=v.to(torch.bfloat16), codes=codes, exps=exps)


def run_dense(st):
    y = torch.matmul(values(st["x"], st["x_exp"], 1), values(st["w"], st["w_exp"], BLOCK).t())
    if st["add"] is not None:
        y = y + st["add"].float()
    return y.to(st["y"].dtype)


def run_sample(st):
    # in 64 bits: a drawn number may fall next to a border between two tokens
    l, order = torch.sort(st["logits"], dim=1, descending=True, stable=True)
    n = l.shape[1]
    greedy = st["temperature"] <= 0
    w = torch.exp((l - l[:, :1].double()) / torch.where(greedy, 1.0, st["temperature"]).double()[:, None])
    c = torch.cumsum(w, dim=1)
    k = torch.where((st["top_k"] > 0) & (st["top_k"] < n), st["top_k"], n).long()
    M = torch.gather(c, 1, k[:, None] - 1)
    p = st["top_p"].double()[:, None]
    by_p = torch.gather(c, 1, ((c < p * M).sum(dim=1, keepdim=True)).clamp(max=n - 1))
    by_min = torch.gather(c, 1, (w >= st["min_p"].double()[:, None]).sum(dim=1, keepdim=True) - 1)
    M = torch.minimum(torch.minimum(M, torch.where(p < 1.0, by_p, M)), by_min)
    j = (c <= st["u"].double()[:, None] * M).sum(dim=1, keepdim=True)
    j = torch.where(greedy[:, None], 0, j)
    prob = torch.where(greedy, 1.0, (torch.gather(w, 1, j) / M)[:, 0])
    return dict(idx=torch.gather(order, 1, j)[:, 0].to(torch.int32), prob=prob.to(torch.float32))


# ---------------------------------------------------------------- the work

def work(case):
    """Every input read once and every output written once; a product's multiplications and additions."""
    size = {"bf16": 2, "f32": 4}.get(case.get("dtype"))
    if case["kind"] == "quant":
        values_ = case["rows"] * case["n"]
        return dict(bytes=values_ * (size + 1) + values_ / (BLOCK * case["block_rows"]), flops=2 * values_)
    if case["kind"] == "norm":
        values_ = case["T"] * case["d"]
        return dict(bytes=values_ * (2 + size + 2 + 2 * case["total"] + 1 + 1 / BLOCK) + 2 * case["d"] * case["gain"],
                    flops=6 * values_)
    if case["kind"] == "dense":
        T, n_in, n_out = case["T"], case["n_in"], case["n_out"]
        return dict(bytes=(T + n_out) * n_in + (T + n_out / BLOCK) * n_in / BLOCK + T * n_out * size * (1 + case["add"]),
                    flops=2 * T * n_in * n_out)
    return dict(bytes=4 * case["T"] * case["n"] + 28 * case["T"], flops=4 * case["T"] * case["n"])


# ------------------------------------------------------------------- exact

# the 256 values of e4m3, from the format: sign, 4 exponent bits (bias 7), 3 mantissa bits, no infinities
E4M3 = [(-1.0 if b & 128 else 1.0) * (math.nan if b & 127 == 127 else (b & 7) * 2.0 ** -9 if (b >> 3) & 15 == 0
                                      else (8 + (b & 7)) * 2.0 ** (((b >> 3) & 15) - 10)) for b in range(256)]


def exact(case, seed):
    st = prepare(case, seed)
    if case["kind"] == "quant":
        return nearest(st["x"].double(), case["block_rows"])
    if case["kind"] == "norm":
        x = st["h"].double() + st["y"].double()
        length = (x * x).sum(dim=1) / case["d"] + EPS
        v = x / length.sqrt()[:, None]
        v = v * st["gain"].double() if case["gain"] else v
        return dict(sum=x if case["total"] else None, out=v, **nearest(v, 1))
    if case["kind"] == "dense":
        table = torch.tensor(E4M3, dtype=torch.float64, device="cuda")
        x, w = table[st["x"].view(torch.uint8).long()], table[st["w"].view(torch.uint8).long()]
        out = torch.zeros(case["T"], case["n_out"], dtype=torch.float64, device="cuda")
        for b in range(0, case["n_in"], BLOCK):  # a block of columns after the other
            xs = torch.exp2(st["x_exp"][:, b // BLOCK].double() - EXP_BIAS)
            ws = torch.exp2(st["w_exp"][:, b // BLOCK].double() - EXP_BIAS).repeat_interleave(BLOCK)[:case["n_out"]]
            out += (x[:, b:b + BLOCK] * xs[:, None]) @ (w[:, b:b + BLOCK] * ws[:, None]).T
        return out if st["add"] is None else out + st["add"].double()
    idx, prob = [], []
    for t in range(case["T"]):
        l = st["logits"][t].double()
        T, k, p, m = (st[x][t].item() for x in ("temperature", "top_k", "top_p", "min_p"))
        by = torch.argsort(l, descending=True, stable=True)
        if T <= 0:
            idx.append(by[0].item())
            prob.append(1.0)
            continue
        z = torch.exp((l[by] - l[by[0]]) / T)
        keep = k if 0 < k < len(z) else len(z)
        if p < 1.0:
            mass = torch.cumsum(z[:keep] / z[:keep].sum(), 0)
            keep = min(keep, int(torch.searchsorted(mass, p).item()) + 1)
        if m > 0.0:
            keep = min(keep, int((z / z[0] >= m).sum().item()))
        q = z[:keep] / z[:keep].sum()
        j = min(int(torch.searchsorted(torch.cumsum(q, 0), st["u"][t].double(), right=True).item()), keep - 1)
        idx.append(by[j].item())
        prob.append(q[j].item())
    return dict(idx=torch.tensor(idx, dtype=torch.int32), prob=torch.tensor(prob, dtype=torch.float64))


def nearest(x, block_rows):
    """The code values and exponents that x's blocks have."""
    R, n = x.shape
    e = torch.full((-(-R // block_rows), -(-n // BLOCK)), EXP_MIN, dtype=torch.float64, device="cuda")
    codes = torch.empty_like(x)
    for b in range(0, n, BLOCK):
        top = x[:, b:b + BLOCK].abs().amax(dim=1)
        top = torch.nn.functional.pad(top, (0, -R % block_rows)).view(-1, block_rows).amax(dim=1)
        e[:, b // BLOCK] = torch.where(top > 0, torch.ceil(torch.log2(top / LARGEST)), EXP_MIN).clamp(EXP_MIN, EXP_MAX)
        y = x[:, b:b + BLOCK] / torch.exp2(e[:, b // BLOCK]).repeat_interleave(block_rows)[:R, None]
        step = torch.exp2(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))) - 3)  # subnormals: 2^-9
        codes[:, b:b + BLOCK] = torch.round(y / step) * step
    return dict(codes=codes, exps=(e + EXP_BIAS).to(torch.uint8))
