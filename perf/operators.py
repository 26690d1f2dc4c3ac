"""The microscaled KV cache: writing it, reading it back, scoring its keys and attending over it.

A cache row of d elements is held in blocks of 32.  A block has one scale byte b, which stands for 2^(b - 127), and 32
elements: 8-bit floats (e4m3, "mxfp8") or 4-bit floats (e2m1, "mxfp4", two to a byte, the even element in the low half).
The scale is the smallest power of two 2^e with largest magnitude <= M 2^e (M = 448 or 6), e limited to -64 .. 15; the
elements are the values divided by it, rounded to nearest even.

A case is a dict of plain values:

    entry      "append"   quoka_append_kv_mx: the chunk's new keys and values go into the cache
               "reread"   the same, then quoka_read_kv_mx of the rows just written
               "read"     quoka_read_kv_mx: the cached rows as plain tensors
               "score"    quoka_score_keys_mx: the cached keys against the retained queries
               "dense"    quoka_dense_chunk_attn_mx: a chunk over all cached rows and its own
               "listed"   quoka_sparse_attn_mx: a chunk over a list of cached rows and its own
    batch, n_q, n_kv, d, dtype            the layer; dtype of the queries, of the new rows and of what comes back
    fmt                                   "mxfp8" or "mxfp4"
    chunk                                 queries (new rows) per sequence, 1 = a generation step
    ctx_len, ctx_min, max_ctx             longest / shortest cached length, and what the buffers are laid out for
    n_retain                              score: queries that the keys are scored against
    kv_budget                             listed: rows in the list
    paged, norms                          64-row pages in random order; inverse key norms kept beside the cache
"""
from __future__ import annotations

import math

import torch

own = False

PAGE = 64
BLOCK = 32
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
E_MIN, E_MAX = -64, 15


def _case(name, **kw):
    c = {"name": name, "entry": "dense", "batch": 1, "n_q": 32, "n_kv": 8, "d": 128, "dtype": "bf16", "fmt": "mxfp8", "chunk": 1,
         "ctx_len": 32768, "ctx_min": 0, "max_ctx": 0, "n_retain": 1, "kv_budget": 0, "paged": False, "norms": False}
    c.update(kw)
    c["ctx_min"] = c["ctx_min"] or c["ctx_len"]
    c["max_ctx"] = c["max_ctx"] or c["ctx_len"]
    return c


def listed():
    return [
        # writing the cache: one row per sequence and head of a paged serving batch (latency), with the norms of its keys
        _case("append_step_b16", entry="append", batch=16, ctx_len=8192, ctx_min=1024, paged=True, norms=True),
        # and the rows of a 2048-token chunk in the middle of a prompt
        _case("append_2048", entry="append", chunk=2048, ctx_len=14336, max_ctx=16384, norms=True),
        # a serving batch's chunks into a 4-bit cache, and the values that it now holds for them
        _case("reread_1024_b8_fp4", entry="reread", batch=8, chunk=1024, ctx_len=8192, ctx_min=2000, fmt="mxfp4", paged=True),
        # long cached prefixes handed to a layer that wants plain tensors
        _case("read_32k_b4_fp4", entry="read", batch=4, ctx_len=32768, ctx_min=20011, fmt="mxfp4"),
        # scoring: a 2048-token chunk's 128 retained queries against 32K keys
        _case("score_32k", entry="score", chunk=2048, n_retain=128),
        # and the generation step of a serving batch, whose norms are kept: every key is read for one product
        _case("score_step_b16", entry="score", batch=16, ctx_len=32768, ctx_min=8192, paged=True, norms=True),
        # attention of a generation step: a short conversation (latency), and a serving batch (the cache is read once)
        _case("step_4k", ctx_len=4003, max_ctx=4096),
        _case("step_mix_b16", batch=16, ctx_len=32768, ctx_min=8192, paged=True),
        # five proposed tokens checked at once, eight heads per KV head of head_dim 64, odd lengths, 4 bits
        _case("verify5_d64_fp4", batch=3, n_kv=4, d=64, chunk=5, ctx_len=20011, ctx_min=9001, fmt="mxfp4"),
        # a chunk over a quarter of the keys: odd sizes, head_dim 64, 4 bits
        _case("listed_777_d64_fp4", entry="listed", n_kv=4, d=64, chunk=777, ctx_len=20011, kv_budget=5003, fmt="mxfp4"),
        # the benchmark's chunk over the rows that its budget leaves
        _case("listed_2048_32k", entry="listed", chunk=2048, kv_budget=3932),
        # and over all of them
        _case("dense_2048_32k", chunk=2048),
    ]


# ----------------------------------------------------------------------------------------------- drawn cases
def _log_int(rng, lo, hi):
    return int(round(math.exp(rng.uniform(math.log(lo), math.log(hi)))))


def _cost(c):
    """Rough time of a pass's plain form: flops at 60 TF/s and bytes in 32 bits at 3 TB/s."""
    keys = sum(_keys_of(c, t) + c["chunk"] for t in _ctx_lens(c))
    if c["entry"] in ("dense", "listed"):
        return 4.0 * c["n_q"] * c["chunk"] * c["d"] * keys / 60e12 + 40.0 * c["n_q"] * c["chunk"] * keys / 3e12 + 16.0 * c["n_kv"] * keys * c["d"] / 3e12
    if c["entry"] == "score":
        return 2.0 * c["n_kv"] * c["n_retain"] * c["d"] * keys / 60e12 + 8.0 * c["n_kv"] * c["n_retain"] * keys / 3e12 + 16.0 * c["n_kv"] * keys * c["d"] / 3e12
    rows = keys if c["entry"] == "read" else c["chunk"] * c["batch"]
    return 64.0 * c["n_kv"] * rows * c["d"] / 3e12


def _state_bytes(c):
    return 4 * c["batch"] * (c["max_ctx"] + c["chunk"]) * c["n_kv"] * c["d"]


def draw(rng):
    while True:
        entry = rng.choices(["append", "reread", "read", "score", "dense", "listed"], [3, 2, 2, 4, 6, 4])[0]
        n_kv, group = rng.choice([(8, 4), (8, 4), (2, 4), (4, 8), (8, 1), (16, 2), (5, 3), (2, 16)])
        c = _case("", entry=entry, n_q=n_kv * group, n_kv=n_kv, d=rng.choice([64, 128, 128]), fmt=rng.choice(["mxfp8", "mxfp8", "mxfp4"]),
                  paged=rng.random() < 0.4, ctx_len=_log_int(rng, 1, 131072))
        del c["name"]
        c["batch"] = rng.choice([1, 1, 1, 2, 3, 4, 8, 16])
        if entry in ("append", "reread"):
            c.update(chunk=rng.choice([1, _log_int(rng, 1, 4096)]), norms=rng.random() < 0.5, ctx_len=_log_int(rng, 1, 16384))
            c["dtype"] = "f32" if rng.random() < 0.3 else "bf16"
        elif entry == "read":
            c["dtype"] = "f32" if rng.random() < 0.3 else "bf16"
        elif entry == "score":
            c.update(chunk=rng.choice([1, 1, _log_int(rng, 2, 4096)]), norms=rng.random() < 0.4)
            c["n_retain"] = min(c["chunk"], rng.choice([16, 50, 64, 128, 256, rng.randint(1, 512)]))
        else:
            c["chunk"] = rng.choice([1, 1, rng.randint(2, 8), _log_int(rng, 8, 4096)])
            if entry == "listed":
                c["kv_budget"] = min(c["ctx_len"], _log_int(rng, 64, 16384))
        c["ctx_min"] = max(1, int(c["ctx_len"] * rng.uniform(0.15, 1.0))) if c["batch"] > 1 else c["ctx_len"]
        c["max_ctx"] = c["ctx_len"] if rng.random() < 0.6 else int(c["ctx_len"] * rng.uniform(1.0, 1.5))
        if _cost(c) <= _cost(listed()[-1]) and _state_bytes(c) <= 2.2e9:
            return c


# ----------------------------------------------------------------------------------------------- sizes of a case
def _ctx_lens(c):
    """Cached lengths of the batch: the longest first, the others spread over [ctx_min, ctx_len]."""
    lo, hi = c["ctx_min"], c["ctx_len"]
    return [hi - int((hi - lo) * ((s * 0.6180339887) % 1.0)) for s in range(c["batch"])]


def _keys_of(c, t):
    """Cached rows of a sequence of t that a query attends to."""
    return min(c["kv_budget"], t) if c["entry"] == "listed" else t


def _n_retain(c):
    return min(c["n_retain"], c["chunk"])


# ----------------------------------------------------------------------------------------------- inputs
class _State:
    pass


def _row_bytes(d, fmt):
    return d if fmt == "mxfp8" else d // 2


def _keys(shape, g):
    """Keys ~ N(0, I), one position in twenty three times as long (independently per KV head)."""
    k = torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=g)
    big = torch.rand(shape[:-1], device="cuda", generator=g) < 0.05
    return k.mul_((1.0 + 2.0 * big.float()).unsqueeze(-1))


def prepare(case, seed):
    """Keys and values normal, queries scattered around a mean direction per head: the distributions of the tests."""
    c = case
    st = _State()
    st.c = c
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    dt = DTYPES[c["dtype"]]
    b, n_q, n_kv, d, C, fmt = c["batch"], c["n_q"], c["n_kv"], c["d"], c["chunk"], c["fmt"]
    lens = _ctx_lens(c)
    st.pow2 = torch.tensor([2.0 ** (i - 127) for i in range(255)] + [math.nan], dtype=torch.float32, device="cuda")
    st.fp4 = torch.tensor([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0, -0.0, -0.5, -1.0, -1.5, -2.0, -3.0, -4.0, -6.0], device="cuda")
    st.ctx_len = torch.tensor(lens, dtype=torch.int32, device="cuda")
    st.table = None
    rows = c["max_ctx"] + C
    if c["paged"]:
        need = [-(-(t + C) // PAGE) for t in lens]
        perm = torch.randperm(sum(need), generator=torch.Generator().manual_seed(seed)).to(torch.int32)
        table = torch.full((b, -(-rows // PAGE)), -1, dtype=torch.int32)
        off = 0
        for s, n in enumerate(need):
            table[s, :n] = perm[off:off + n]
            off += n
        st.table = table.cuda()
        shape = (sum(need), n_kv, PAGE, d)
    else:
        shape = (b, n_kv, rows, d)
    st.k, st.k_scale = _quantise(st, _keys(shape, g), fmt)
    st.v, st.v_scale = _quantise(st, torch.empty(shape, dtype=torch.float32, device="cuda").normal_(generator=g), fmt)
    mu = torch.randn(b, n_q, 1, d, device="cuda", generator=g)
    st.q = (mu + 0.7 * torch.randn(b, n_q, C, d, device="cuda", generator=g)).to(dt)
    st.out = torch.empty_like(st.q)
    st.norms = torch.zeros(shape[:3], device="cuda") if c["norms"] else None
    if c["norms"]:
        st.norms += 1.0 / _dequantise(st, st.k, st.k_scale, fmt).square().sum(-1).sqrt().clamp_min(1e-12)
    if c["entry"] in ("append", "reread"):
        st.k_new = _keys((b, n_kv, C, d), g).to(dt)
        st.v_new = torch.empty((b, n_kv, C, d), device="cuda").normal_(generator=g).to(dt)
    if c["entry"] in ("read", "reread"):
        n = max(lens) if c["entry"] == "read" else rows
        st.k_out = torch.zeros(b, n_kv, n if c["entry"] == "read" else C, d, dtype=dt, device="cuda")
        st.v_out = torch.zeros_like(st.k_out)
    if c["entry"] == "score":
        unit = st.q.float() / st.q.float().square().sum(-1, keepdim=True).sqrt()
        st.qbar = unit[:, :, :_n_retain(c)].reshape(b, n_kv, n_q // n_kv, _n_retain(c), d).mean(2).to(dt)
        st.scores = torch.zeros(b, n_kv, c["max_ctx"], device="cuda")
    if c["entry"] == "listed":
        cnt = [_keys_of(c, t) for t in lens]
        cap = min(c["kv_budget"], c["max_ctx"])
        st.k_idx = torch.full((b, n_kv, cap), -1, dtype=torch.int32, device="cuda")
        for s, t in enumerate(lens):
            pick = torch.rand(n_kv, t, device="cuda", generator=g).argsort(-1)[:, :cnt[s]].sort(-1).values
            st.k_idx[s, :, :cnt[s]] = pick.to(torch.int32)
        st.k_cnt = torch.tensor(cnt, dtype=torch.int32, device="cuda")
    st.call = None
    return st


# ----------------------------------------------------------------------------------------------- the plain form
def _quantise(st, x, fmt):
    """(element bytes, scale bytes) of x in 32 bits."""
    x = x.unflatten(-1, (-1, BLOCK))
    amax = x.abs().amax(-1)
    m, ex = torch.frexp(amax)                                       # amax = m 2^ex, 0.5 <= m < 1
    e = torch.where(m <= 0.875, ex - 9, ex - 8) if fmt == "mxfp8" else torch.where(m <= 0.75, ex - 3, ex - 2)
    e = e.clamp(E_MIN, E_MAX)
    e = torch.where(amax == 0, torch.full_like(e, E_MIN), e)
    finite = torch.isfinite(amax)
    e = torch.where(finite, e, torch.zeros_like(e))
    y = torch.where(finite.unsqueeze(-1), x * st.pow2[127 - e].unsqueeze(-1), torch.zeros_like(x)).flatten(-2)
    scale = torch.where(finite, e + 127, torch.full_like(e, 255)).to(torch.uint8)
    if fmt == "mxfp8":
        return y.clamp(-448.0, 448.0).to(torch.float8_e4m3fn).view(torch.uint8), scale
    a = y.abs()
    code = ((a > 0.25).to(torch.uint8) + (a >= 0.75) + (a > 1.25) + (a >= 1.75) + (a > 2.5) + (a >= 3.5) + (a > 5.0))
    code = code.to(torch.uint8) + torch.signbit(y).to(torch.uint8) * 8
    return code[..., 0::2] + code[..., 1::2] * 16, scale


def _dequantise(st, rows, scale, fmt):
    """The values of element and scale bytes, in 32 bits."""
    if fmt == "mxfp8":
        x = rows.view(torch.float8_e4m3fn).float()
    else:
        x = torch.stack([st.fp4[(rows & 15).int()], st.fp4[(rows >> 4).int()]], -1).flatten(-2)
    return (x.unflatten(-1, (-1, BLOCK)) * st.pow2[scale.int()].unsqueeze(-1)).flatten(-2)


def _logical(st, cache, n):
    """Rows [0, n) of every sequence, (b, n_kv, n, ...), whatever the layout."""
    if st.table is None:
        return cache[:, :, :n]
    pages = cache[st.table[:, :-(-n // PAGE)].clamp_min(0).long()]          # (b, pages, n_kv, 64, ...)
    return pages.transpose(1, 2).flatten(2, 3)[:, :, :n]


def _new_rows(st):
    """Where row r of sequence s goes: index tensors (b, 1, C), (1, n_kv, 1), (b, 1, C) into the cache's first three dimensions."""
    n_kv, C = st.c["n_kv"], st.c["chunk"]
    b = st.ctx_len.numel()
    t = st.ctx_len.long()[:, None] + torch.arange(C, device="cuda")
    h = torch.arange(n_kv, device="cuda")[None, :, None]
    if st.table is None:
        return torch.arange(b, device="cuda")[:, None, None], h, t[:, None]
    page = st.table.long().gather(1, t // PAGE)
    return page[:, None], h, (t % PAGE)[:, None]


def _plain_append(st):
    fmt, at = st.c["fmt"], _new_rows(st)
    st.k[at], st.k_scale[at] = _quantise(st, st.k_new.float(), fmt)
    st.v[at], st.v_scale[at] = _quantise(st, st.v_new.float(), fmt)
    if st.norms is not None:
        st.norms[at] = 1.0 / _dequantise(st, st.k[at], st.k_scale[at], fmt).square().sum(-1).sqrt().clamp_min(1e-12)


def _plain_read(st):
    fmt = st.c["fmt"]
    if st.c["entry"] == "reread":
        at = _new_rows(st)
        st.k_out.copy_(_dequantise(st, st.k[at], st.k_scale[at], fmt))
        st.v_out.copy_(_dequantise(st, st.v[at], st.v_scale[at], fmt))
        return
    n = st.k_out.shape[2]
    there = (torch.arange(n, device="cuda") < st.ctx_len[:, None] + st.c["chunk"])[:, None, :, None]
    st.k_out.copy_(torch.where(there, _dequantise(st, _logical(st, st.k, n), _logical(st, st.k_scale, n), fmt), st.k_out.float()))
    st.v_out.copy_(torch.where(there, _dequantise(st, _logical(st, st.v, n), _logical(st, st.v_scale, n), fmt), st.v_out.float()))


def _plain_score(st):
    c = st.c
    n = min(c["ctx_len"], c["max_ctx"])
    k = _dequantise(st, _logical(st, st.k, n), _logical(st, st.k_scale, n), c["fmt"])
    best = (k @ st.qbar.float().transpose(-1, -2)).amax(-1)
    inv = 1.0 / k.square().sum(-1).sqrt().clamp_min(1e-12) if st.norms is None else _logical(st, st.norms, n)
    there = (torch.arange(n, device="cuda") < st.ctx_len[:, None])[:, None]
    st.scores[:, :, :n] = torch.where(there, best * inv, st.scores[:, :, :n])


def _attended(st, cache, scale):
    """(values in 32 bits of the rows that a chunk may see, cached ones first; how many of them are cached rows)."""
    c = st.c
    n = c["ctx_len"] + c["chunk"]
    rows, scales = _logical(st, cache, n), _logical(st, scale, n)
    if c["entry"] == "listed":
        own_rows = (st.ctx_len.long()[:, None] + torch.arange(c["chunk"], device="cuda"))[:, None].expand(-1, c["n_kv"], -1)
        idx = torch.cat([st.k_idx.long().clamp_min(0), own_rows], -1)[..., None]
        rows = rows.gather(2, idx.expand(-1, -1, -1, rows.shape[-1]))
        scales = scales.gather(2, idx.expand(-1, -1, -1, scales.shape[-1]))
    return _dequantise(st, rows, scales, c["fmt"])


def _seen(st, n):
    """(b, C, n): which of the attended rows chunk row r sees."""
    c = st.c
    r, j = torch.arange(c["chunk"], device="cuda")[None, :, None], torch.arange(n, device="cuda")[None, None]
    if c["entry"] == "dense":
        return j <= st.ctx_len[:, None, None] + r
    cap = st.k_idx.shape[-1]
    return torch.where(j < cap, j < st.k_cnt[:, None, None], j - cap <= r)


def _plain_attend(st):
    c = st.c
    b, n_q, C, d = st.q.shape
    k, v = _attended(st, st.k, st.k_scale), _attended(st, st.v, st.v_scale)
    n = k.shape[2]
    seen = _seen(st, n)
    v = torch.where(seen.any(1)[:, None, :, None], v, torch.zeros_like(v))
    s = (st.q.float().reshape(b, c["n_kv"], -1, d) @ k.transpose(-1, -2)).mul_(1.0 / math.sqrt(d))
    s = s.view(b, n_q, C, n).masked_fill_(~seen[:, None], -math.inf)
    s = s.sub_(s.amax(-1, keepdim=True)).exp_()
    total = s.sum(-1, keepdim=True)
    o = (s.view(b, c["n_kv"], -1, n) @ v).view(b, n_q, C, d) / total
    st.out.copy_(o)


# ----------------------------------------------------------------------------------------------- a pass
class _Call:
    pass


def _own_call(st):
    """What a program makes once per cache: the call's parameters, the cache's description, a workspace."""
    from paper_2602_08722_b200 import api

    c = st.c
    call = _Call()
    call.api = api
    fmt = api.KV_MXFP8 if c["fmt"] == "mxfp8" else api.KV_MXFP4
    call.p = api.make_params(st.q, st.k, st.out, st.ctx_len, n_retain=c["n_retain"], kv_budget=c["kv_budget"], max_ctx_len=c["max_ctx"],
                             block_table=st.table, kv_format=fmt)
    if c["norms"] and c["entry"] == "score":
        call.p.k_inv_norm = st.norms.data_ptr()
    call.mx = api.make_mx_cache(fmt, st.k_scale, st.v_scale)
    call.ws = api.alloc_workspace(call.p, mx=call.mx)
    return call


def _own_pass(st):
    if st.call is None:
        st.call = _own_call(st)
    api, p, mx, ws, entry = st.call.api, st.call.p, st.call.mx, st.call.ws, st.c["entry"]
    if entry == "dense":
        api.quoka_dense_chunk_attn_mx(p, mx, st.q, st.k, st.v, st.out, None, ws)
    elif entry == "listed":
        api.quoka_sparse_attn_mx(p, mx, st.q, st.k, st.v, st.k_idx, st.k_cnt, st.out, None, ws)
    elif entry == "score":
        api.quoka_score_keys_mx(p, mx, st.qbar, st.k, st.scores, ws)
    elif entry == "read":
        api.quoka_read_kv_mx(p, mx, st.k, st.v, 0, st.k_out.shape[2], st.k_out, st.v_out, ws)
    else:
        api.quoka_append_kv_mx(p, mx, st.k_new, st.v_new, st.k, st.v, st.norms, ws)
        if entry == "reread":
            api.quoka_read_kv_mx(p, mx, st.k, st.v, api.FROM_CTX_LEN, st.c["chunk"], st.k_out, st.v_out, ws)


def run(st):
    entry = st.c["entry"]
    if own:
        _own_pass(st)
    elif entry in ("dense", "listed"):
        _plain_attend(st)
    elif entry == "score":
        _plain_score(st)
    elif entry == "read":
        _plain_read(st)
    else:
        _plain_append(st)
        if entry == "reread":
            _plain_read(st)
    if entry in ("dense", "listed"):
        return {"out": st.out}
    if entry == "score":
        return {"scores": st.scores}
    if entry in ("read", "reread"):
        return {"k": st.k_out, "v": st.v_out}
    res = {"k_scale": st.k_scale, "v_scale": st.v_scale}
    if st.c["fmt"] == "mxfp8":                                       # (4-bit elements come back as values in "reread")
        res["k"], res["v"] = st.k.view(torch.float8_e4m3fn), st.v.view(torch.float8_e4m3fn)
    if st.norms is not None:
        res["norms"] = st.norms
    return res


# ----------------------------------------------------------------------------------------------- from the definition, 64 bits
def _powers():
    return torch.tensor([2.0 ** i for i in range(-200, 201)], dtype=torch.float64, device="cuda")


def _rounded64(x, fmt):
    """The values of x's blocks as the cache holds them, divided by their scales, and the exponents of these (finite x)."""
    p2 = _powers()
    x = x.double().unflatten(-1, (-1, BLOCK))
    most, digits, lowest = (448.0, 3, -6) if fmt == "mxfp8" else (6.0, 1, 0)
    amax = x.abs().amax(-1, keepdim=True)
    e = torch.full_like(amax, E_MIN, dtype=torch.int64)
    for cand in range(E_MIN, E_MAX):                                  # the smallest exponent that reaches
        e = torch.where(amax > most * 2.0 ** cand, torch.full_like(e, cand + 1), e)
    a = x.abs() / p2[e + 200]
    at = torch.frexp(a)[1].long() - 1                                 # 2^at <= a < 2^(at + 1)
    step = p2[at.clamp(lowest, 9) - digits + 200]
    return (torch.round(a / step) * step).clamp_max(most).copysign(x), e


def _values64(rows, scale, fmt):
    """Element and scale bytes to values, from the bits."""
    p2 = _powers()
    if fmt == "mxfp8":
        c, frac, lowest = rows.int(), 3, -6
        sign, exp, man = c >> 7, (c >> 3) & 15, c & 7
        bias = 7
    else:
        c, frac, lowest = torch.stack([rows & 15, rows >> 4], -1).flatten(-2).int(), 1, 0
        sign, exp, man = c >> 3, (c >> 1) & 3, c & 1
        bias = 1
    m = torch.where(exp > 0, 1.0 + man.double() / 2 ** frac, man.double() / 2 ** frac)
    x = m * p2[torch.where(exp > 0, exp - bias, torch.full_like(exp, lowest)).long() + 200] * (1.0 - 2.0 * sign)
    return (x.unflatten(-1, (-1, BLOCK)) * p2[scale.long() - 127 + 200].unsqueeze(-1)).flatten(-2)


def _cache64(st, s, h, rows, cache, scale):
    """Values of the cache rows `rows` (a tensor) of KV head h of sequence s."""
    if st.table is None:
        return _values64(cache[s, h, rows], scale[s, h, rows], st.c["fmt"])
    page = st.table[s].long()[rows // PAGE]
    return _values64(cache[page, h, rows % PAGE], scale[page, h, rows % PAGE], st.c["fmt"])


def exact(case, seed):
    st = prepare(case, seed)
    c = case
    b, n_kv, C, d, G = c["batch"], c["n_kv"], c["chunk"], c["d"], c["n_q"] // c["n_kv"]
    lens = _ctx_lens(c)
    if c["entry"] in ("append", "reread"):
        (kv, ke), (vv, ve) = _rounded64(st.k_new, c["fmt"]), _rounded64(st.v_new, c["fmt"])
        p2 = _powers()
        k64, v64 = (kv * p2[ke + 200]).flatten(-2), (vv * p2[ve + 200]).flatten(-2)
        if c["entry"] == "reread":
            return {"k": k64, "v": v64}
        res = {"k_scale": None, "v_scale": None}
        at = _new_rows(st)
        if c["fmt"] == "mxfp8":
            res["k"], res["v"] = st.k.view(torch.float8_e4m3fn).double(), st.v.view(torch.float8_e4m3fn).double()
            res["k"][at], res["v"][at] = kv.flatten(-2), vv.flatten(-2)
        if c["norms"]:
            res["norms"] = st.norms.double()
            res["norms"][at] = 1.0 / k64.square().sum(-1).sqrt().clamp_min(1e-12)
        return res
    if c["entry"] == "read":
        res = {"k": torch.zeros(st.k_out.shape, dtype=torch.float64, device="cuda"), "v": torch.zeros(st.k_out.shape, dtype=torch.float64, device="cuda")}
        for s in range(b):
            rows = torch.arange(min(lens[s] + C, st.k_out.shape[2]), device="cuda")
            for h in range(n_kv):
                res["k"][s, h, :rows.numel()] = _cache64(st, s, h, rows, st.k, st.k_scale)
                res["v"][s, h, :rows.numel()] = _cache64(st, s, h, rows, st.v, st.v_scale)
        return res
    if c["entry"] == "score":
        scores = st.scores.double()
        for s in range(b):
            rows = torch.arange(lens[s], device="cuda")
            for h in range(n_kv):
                k = _cache64(st, s, h, rows, st.k, st.k_scale)
                inv = 1.0 / k.square().sum(-1).sqrt().clamp_min(1e-12)
                if st.norms is not None:                              # the norms are inputs
                    inv = (st.norms[s, h, rows] if st.table is None else st.norms[st.table[s].long()[rows // PAGE], h, rows % PAGE]).double()
                scores[s, h, :lens[s]] = (k @ st.qbar[s, h].double().T).amax(-1) * inv
        return {"scores": scores}
    out = torch.empty(st.q.shape, dtype=torch.float64, device="cuda")
    for s in range(b):
        chunk_rows = lens[s] + torch.arange(C, device="cuda")
        for h in range(n_kv):
            cached = st.k_idx[s, h, :int(st.k_cnt[s])].long() if c["entry"] == "listed" else torch.arange(lens[s], device="cuda")
            rows = torch.cat([cached, chunk_rows])
            k, v = _cache64(st, s, h, rows, st.k, st.k_scale), _cache64(st, s, h, rows, st.v, st.v_scale)
            hidden = torch.arange(rows.numel(), device="cuda")[None] - cached.numel() > torch.arange(C, device="cuda")[:, None]
            for g in range(h * G, (h + 1) * G):
                w = (st.q[s, g].double() @ k.T) / math.sqrt(d)
                w = torch.exp(w.masked_fill(hidden, -math.inf) - w.masked_fill(hidden, -math.inf).amax(-1, keepdim=True))
                out[s, g] = (w @ v) / w.sum(-1, keepdim=True)
    return {"out": out}


# ----------------------------------------------------------------------------------------------- what a pass needs
def work(case):
    c = case
    es = 2 if c["dtype"] == "bf16" else 4
    b, n_q, n_kv, d, C = c["batch"], c["n_q"], c["n_kv"], c["d"], c["chunk"]
    row = _row_bytes(d, c["fmt"]) + d // BLOCK
    lens = _ctx_lens(c)
    if c["entry"] in ("append", "reread"):
        nbytes = 2.0 * b * n_kv * C * (d * es + row) + (4.0 * b * n_kv * C if c["norms"] else 0.0)
        if c["entry"] == "reread":
            nbytes += 2.0 * b * n_kv * C * d * es                     # (the rows are read as they are written)
        return {"bytes": nbytes, "flops": 0.0}
    if c["entry"] == "read":
        rows = sum(min(t + C, max(lens)) for t in lens)
        return {"bytes": 2.0 * n_kv * rows * (d * es + row), "flops": 0.0}
    if c["entry"] == "score":
        keys, N = float(sum(lens)), _n_retain(c)
        return {"bytes": n_kv * keys * (row + 4.0 + (4.0 if c["norms"] else 0.0)) + b * n_kv * N * d * es, "flops": 2.0 * n_kv * N * d * keys}
    nbytes = flops = 0.0
    for t in lens:
        keys = _keys_of(c, t)
        nbytes += 2.0 * n_q * C * d * es + 2.0 * n_kv * (keys + C) * row + (4.0 * n_kv * keys if c["entry"] == "listed" else 0.0)
        flops += 4.0 * n_q * C * d * (keys + (C + 1) / 2)
    return {"bytes": nbytes, "flops": flops}
