"""The microscaled cache on the device: written, read back, scored and attended over, against the definition in 64 bits.

Tolerances.  What the cache holds and what is read back is exact.  Scores: as for a bf16 cache (tests/parity.py): products of
Qbar with the cache's values are exact in fp32, the sum of at most 128 of them and the norm are off by at most
128 * 2^-24 * |qbar| |k| each.  Norms: a sum of at most 128 squares in fp32 (7 + 8 roundings on the longest path), its root
and a division: below 16 * 2^-24 relative.  Attention outputs: parity.attention_bound (bf16 softmax weights and outputs).
"""
import numpy as np
import pytest
import torch

from oracle import quoka_oracle as O
from paper_2602_08722_b200 import api, synth
from tests import mx_reference as R
from tests import parity as PA

pytestmark = pytest.mark.gpu
FORMATS = [api.KV_MXFP8, api.KV_MXFP4]
DTYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NORM_RTOL = 16 * 2.0 ** -24


def rows_to_quantise(b, n_kv, n, d, dtype, seed):
    """Normal rows of many magnitudes, and blocks where quantising can go wrong."""
    g = torch.Generator().manual_seed(seed)
    x = torch.randn(b, n_kv, n, d, generator=g) * torch.exp2(torch.randint(-12, 12, (b, n_kv, n, 1), generator=g).float())
    flat = x.view(-1, d // 32, 32)
    special = [
        torch.zeros(32), -torch.zeros(32), torch.full((32,), 2.0 ** -80), torch.full((32,), 3e38), torch.linspace(-6, 6, 32),
        torch.linspace(-448, 448, 32), torch.tensor([1.75 * 2 ** 8] + [2.0 ** -i for i in range(31)]),
        torch.tensor([1.76 * 2 ** 8] + [-(2.0 ** -i) for i in range(31)]), torch.tensor([6.0, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0] * 4),
        torch.tensor([448.0, 17.0, 19.0, 248.0, 2.0 ** -10, 3 * 2.0 ** -10, -2.0 ** -9, 0.0] * 4), torch.full((32,), 448.0 * 2 ** 15),
        torch.full((32,), 6.0 * 2 ** 15 + 2 ** 12), torch.full((32,), 1e-42)]
    for i, blk in enumerate(special):
        if i < flat.shape[0]:
            flat[i, i % (d // 32)] = blk
    for i, bad in enumerate((float("nan"), float("inf"), -float("inf"))):
        at = len(special) + i
        if at < flat.shape[0]:
            flat[at, 0, 7 * i] = bad
    return x.to(DTYPES[dtype])


class Caches:
    """An empty microscaled cache of b sequences, filled with a pattern that must stay where nothing is written."""

    def __init__(self, b, n_kv, d, C, lens, fmt, paged, layout="bhtd"):
        self.lens, self.paged, self.C = lens, paged, C
        rows = max(lens) + C + 5
        dev = "cuda"
        self.table = None
        if paged:
            need = [-(-(t + C) // 64) for t in lens]
            perm = np.random.default_rng(1).permutation(sum(need) + 1)
            self.table_host = np.full((b, -(-(max(lens) + C) // 64)), -1, dtype=np.int32)
            off = 0
            for s, n in enumerate(need):
                self.table_host[s, :n] = perm[off:off + n]
                off += n
            self.table = torch.from_numpy(self.table_host).to(dev)
            shape = (len(perm), n_kv, 64)
        else:
            shape = (b, n_kv, rows)
        k, v, ks, vs = api.alloc_mx_cache(shape, d, fmt)
        self.k, self.v = R.MxProblem._lay_out(k, layout), R.MxProblem._lay_out(v, layout)
        self.k_scale, self.v_scale = ks, vs
        for t in (self.k, self.v, ks, vs):
            t.fill_(0xA5)
        self.norms = torch.full(shape, 7.0, device=dev)

    def where(self, s):
        """Index of the C rows of sequence s, for (n_kv, C, ...) views."""
        t = np.arange(self.lens[s], self.lens[s] + self.C)
        if not self.paged:
            return lambda a: a[s][:, t]
        page = self.table_host[s, t // 64].astype(np.int64)
        return lambda a: a[page, :, t % 64].swapaxes(0, 1)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("b,n_kv,d,C,lens,paged,layout", [
    (1, 1, 128, 1, [0], False, "bhtd"), (3, 2, 64, 1, [5, 64, 127], True, "bhtd"), (2, 5, 128, 77, [0, 63], True, "bhtd"),
    (2, 3, 64, 130, [9, 200], False, "bthd"), (16, 8, 128, 1, list(range(100, 116)), True, "bhtd"), (1, 2, 128, 1025, [31], False, "bthd"),
    (2, 1, 64, 64, [64, 1], True, "bthd")])
def test_append_and_read_back(fmt, dtype, b, n_kv, d, C, lens, paged, layout):
    c = Caches(b, n_kv, d, C, lens, fmt, paged, layout)
    k_new, v_new = (rows_to_quantise(b, n_kv, C, d, dtype, i).cuda() for i in (3, 4))
    q = torch.zeros(b, n_kv, C, d, dtype=DTYPES[dtype], device="cuda")
    ctx = torch.tensor(lens, dtype=torch.int32, device="cuda")
    p = api.make_params(q, c.k, q, ctx, n_retain=16, kv_budget=16, max_ctx_len=max(lens), block_table=c.table, kv_format=fmt)
    mx = api.make_mx_cache(fmt, c.k_scale, c.v_scale)
    ws = api.alloc_workspace(p, mx=mx)
    api.quoka_append_kv_mx(p, mx, k_new, v_new, c.k, c.v, c.norms, ws)
    outs = {}
    for first, n in ((api.FROM_CTX_LEN, C), (max(0, min(lens) - 1), C + 7)):
        ko, vo = (torch.full((b, n_kv, n, d), 9.0, dtype=DTYPES[dtype], device="cuda") for _ in range(2))
        api.quoka_read_kv_mx(p, mx, c.k, c.v, first, n, ko, vo, ws)
        outs[first] = (ko, vo)
    only_k = torch.full((b, n_kv, C, d), 9.0, dtype=DTYPES[dtype], device="cuda")
    api.quoka_read_kv_mx(p, mx, c.k, None, api.FROM_CTX_LEN, C, only_k, None, ws)
    torch.cuda.synchronize()
    assert torch.equal(torch.nan_to_num(only_k, nan=1e30), torch.nan_to_num(outs[-1][0], nan=1e30))
    untouched = []
    for name, new, cache, scale, at in (("k", k_new, c.k, c.k_scale, 0), ("v", v_new, c.v, c.v_scale, 1)):
        codes, want_scale = R.quantise(new.double().cpu().numpy(), fmt)
        vals = R.values(codes, want_scale, fmt)
        bytes_host, scale_host = cache.cpu().numpy().copy(), scale.cpu().numpy().copy()
        for s in range(b):
            sel = c.where(s)
            np.testing.assert_array_equal(sel(scale_host), want_scale[s], err_msg=name)
            np.testing.assert_array_equal(sel(bytes_host), R.pack(codes[s], fmt), err_msg=name)
            got = outs[-1][at][s].double().cpu().numpy()
            want = torch.from_numpy(vals[s]).to(DTYPES[dtype]).double().numpy()
            np.testing.assert_array_equal(got, want)
            first = max(0, min(lens) - 1)
            there = outs[first][at][s].double().cpu().numpy()
            for i in range(C + 7):
                t = first + i - lens[s]
                if 0 <= t < C:
                    np.testing.assert_array_equal(there[:, i], want[:, t])
                elif t >= C:
                    assert (there[:, i] == 9.0).all()         # rows behind the sequence
            if name == "k":
                nn = (vals[s] ** 2).sum(-1)
                got_n, want_n = sel(c.norms.cpu().numpy()), 1.0 / np.fmax(np.sqrt(nn), 1e-12)     # (not finite: as a norm of nothing, as in the bf16 cache)
                fine = ~(nn <= 1e-30)                           # (squares of smaller values are subnormal in fp32)
                assert (np.abs(got_n - want_n)[fine] <= NORM_RTOL * want_n[fine]).all()
        # nothing else was written
        mask = np.zeros(scale_host.shape[:3], bool)
        for s in range(b):
            t = np.arange(lens[s], lens[s] + C)
            if paged:
                mask[c.table_host[s, t // 64].astype(np.int64), :, t % 64] = True
            else:
                mask[s][:, t] = True
        assert (scale_host[~mask] == 0xA5).all() and (bytes_host[~mask] == 0xA5).all()
        untouched.append((c.norms.cpu().numpy()[~mask] == 7.0).all())
    assert all(untouched)
    assert api.quoka_last_device_status(ws) == 0


IMPLS = [api.IMPL_AUTO, api.IMPL_SIMT]


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("b,n_kv,d,lens,N,paged,norms,mode,agg,dtype", [
    (1, 2, 128, [1], 1, False, False, "cosine", "max", "bf16"), (3, 2, 64, [0, 129, 64], 1, True, True, "cosine", "max", "bf16"),
    (2, 5, 128, [700, 255], 7, True, False, "cosine", "max", "bf16"), (2, 1, 128, [1000, 33], 16, False, True, "cosine", "mean", "bf16"),
    (1, 3, 64, [513], 50, False, False, "dot", "max", "bf16"), (1, 2, 128, [2000], 128, False, False, "cosine", "max", "bf16"),
    (2, 1, 128, [640, 1], 300, True, False, "dot", "mean", "bf16"), (1, 1, 64, [400], 512, False, True, "cosine", "max", "bf16"),
    (1, 2, 128, [300], 20, False, False, "cosine", "max", "f32"), (1, 1, 128, [200], 600, False, False, "cosine", "max", "bf16")])
def test_scores(impl, fmt, b, n_kv, d, lens, N, paged, norms, mode, agg, dtype):
    inp = synth.make_chunk_inputs(5, b, 2 * n_kv, n_kv, d, lens, N, dtype)
    P = R.MxProblem(inp, fmt, paged=paged, n_retain=N, kv_budget=8, impl=impl, cached_norms=norms, max_ctx_len=max(lens) + 9)
    P.p.score_mode = {"cosine": api.SCORE_COSINE, "dot": api.SCORE_DOT}[mode]
    P.p.query_agg = {"max": api.AGG_MAX, "mean": api.AGG_MEAN}[agg]
    g = torch.Generator().manual_seed(8)
    qbar = torch.randn(b, n_kv, N, d, generator=g)
    qbar = (qbar / qbar.norm(dim=-1, keepdim=True)).to(DTYPES[dtype])
    scores = torch.full((b, n_kv, P.max_ctx), 7.0, device="cuda")
    api.quoka_score_keys_mx(P.p, P.mx, qbar.cuda(), P.k, scores, P.ws)
    torch.cuda.synchronize()
    assert api.quoka_last_device_status(P.ws) == 0
    for s, T in enumerate(lens):
        assert (scores[s, :, T:] == 7.0).all()
        if T:
            want = O.score_keys(qbar[s].double().numpy(), P.k64[s, :, :T], T, mode, agg)
            got = scores[s, :, :T].double().cpu().numpy()
            assert np.abs(got - want).max() <= PA.SCORE_ATOL * max(1.0, np.abs(want).max())


ATTN = [
    # b, n_q, n_kv, d, lens, C, paged, layout
    (1, 1, 1, 128, [0], 1, False, "bhtd"), (1, 4, 1, 64, [1], 1, False, "bhtd"), (2, 8, 2, 128, [0, 70], 1, True, "bhtd"),
    (3, 8, 2, 128, [700, 64, 1], 1, True, "bthd"), (2, 32, 4, 64, [129, 500], 1, False, "bthd"), (1, 34, 2, 128, [333], 1, False, "bhtd"),
    (2, 6, 2, 64, [127, 128], 2, True, "bhtd"), (2, 16, 4, 128, [61, 300], 4, False, "bhtd"), (1, 10, 2, 128, [800], 3, True, "bthd"),
    (1, 5, 1, 64, [77], 7, False, "bhtd"), (2, 8, 8, 128, [130, 40], 9, True, "bhtd"), (1, 4, 2, 128, [256], 17, False, "bhtd"),
    (1, 32, 8, 128, [1000], 40, False, "bhtd"), (2, 6, 2, 128, [65, 0], 130, True, "bhtd"), (1, 4, 4, 64, [300], 257, False, "bthd"),
    (1, 8, 2, 64, [511], 129, True, "bhtd"), (2, 8, 2, 128, [1500, 900], 300, True, "bhtd"), (1, 3, 1, 128, [0], 200, False, "bhtd"),
]


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("b,n_q,n_kv,d,lens,C,paged,layout", ATTN)
def test_attention(impl, use_list, fmt, b, n_q, n_kv, d, lens, C, paged, layout):
    inp = synth.make_chunk_inputs(11, b, n_q, n_kv, d, lens, C, "bf16")
    P = R.MxProblem(inp, fmt, paged=paged, impl=impl, kv_budget=max(1, max(lens) // 3) if use_list else 16, layout=layout,
                    q_layout="bchd" if layout == "bthd" else "bhcd", max_ctx_len=max(lens) + 2)
    if use_list:
        k_idx, k_cnt = P.listed(3)
        api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, P.lse, P.ws)
    else:
        api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, P.lse, P.ws)
    torch.cuda.synchronize()
    assert api.quoka_last_device_status(P.ws) == 0
    for s in range(b):
        out, lse = P.reference(s, use_list=use_list)
        PA.check_attention(PA.f64(P.out[s]), out, "bf16")
        assert np.abs(PA.f64(P.lse[s]) - lse).max() <= 2e-3


@pytest.mark.parametrize("use_list", [False, True])
def test_attention_of_f32_queries(use_list):
    inp = synth.make_chunk_inputs(12, 2, 6, 2, 64, [200, 90], 33, "f32")
    P = R.MxProblem(inp, api.KV_MXFP8, paged=True, kv_budget=50)
    if use_list:
        k_idx, k_cnt = P.listed(4)
        api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, P.lse, P.ws)
    else:
        api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, P.lse, P.ws)
    for s in range(2):
        out, lse = P.reference(s, use_list=use_list)
        PA.check_attention(PA.f64(P.out[s]), out, "f32")
        assert np.abs(PA.f64(P.lse[s]) - lse).max() <= 2e-4


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("b,n_q,n_kv,d,T,C,bad_k,bad_v", [
    # (position, block) of blocks that are not finite; positions from T on are the chunk's own rows
    (1, 8, 2, 128, 300, 1, [], [(7, 1)]), (1, 8, 2, 128, 300, 1, [(9, 0)], []), (1, 8, 2, 64, 130, 3, [], [(131, 1)]), (1, 8, 2, 128, 70, 3, [(71, 2)], [(72, 0)]),
    (1, 8, 2, 128, 200, 300, [], [(350, 3), (420, 1)]), (1, 8, 2, 64, 90, 270, [(91 + 100, 0)], [(90 + 200, 1)]), (1, 8, 2, 128, 0, 260, [], [(129, 2)]),
    (1, 4, 1, 128, 150, 200, [], [(20, 3)])])
def test_blocks_that_are_not_finite_reach_only_the_rows_that_see_them(impl, use_list, fmt, b, n_q, n_kv, d, T, C, bad_k, bad_v):
    inp = synth.make_chunk_inputs(13, b, n_q, n_kv, d, T, C, "bf16")
    for t, blk in bad_k:
        inp.k[0, 0, t, 32 * blk + 5] = float("inf")
    for t, blk in bad_v:
        inp.v[0, 0, t, 32 * blk + 9] = float("nan")
    P = R.MxProblem(inp, fmt, impl=impl, kv_budget=max(1, T), max_ctx_len=T)
    if use_list:
        k_idx, k_cnt = P.listed(3)                            # (the whole cache)
        api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, P.lse, P.ws)
    else:
        api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, P.lse, P.ws)
    torch.cuda.synchronize()
    with np.errstate(invalid="ignore"):
        k64, v64 = P.k64.copy(), P.v64.copy()
        P.k64, P.v64 = np.nan_to_num(k64), np.nan_to_num(v64)
        out, _ = P.reference(0, use_list=use_list)            # as if these blocks were zero: right for rows that do not see them
    got = PA.f64(P.out[0])
    G = n_q // n_kv
    bad = np.zeros(got.shape, bool)
    for t, blk in bad_k:
        bad[:G, max(0, t - T):] = True
    for t, blk in bad_v:
        bad[:G, max(0, t - T):, 32 * blk:32 * blk + 32] = True
    assert np.isnan(got[bad]).all()
    # rows that see a value that is not finite are right in their other columns: the reference took its block as zeros there
    rows_clean = ~bad
    bound = PA.attention_bound(out, "bf16")
    assert np.isfinite(got[rows_clean]).all()
    assert (np.abs(got - out)[rows_clean] <= bound[rows_clean]).all()


@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n_q,n_kv,d,T,C,bad_k,bad_v", [
    # row blocks whose key tiles are cut into parts (in a cluster, through memory), and shares of several CTAs
    (8, 2, 128, 3000, 64, [], [(2999, 0), (3040, 2)]), (8, 2, 128, 3000, 64, [(3010, 1)], [(17, 3)]), (4, 1, 64, 4000, 100, [], [(4050, 1), (4090, 0)]),
    (8, 2, 128, 2500, 1, [], [(2500, 3)]), (8, 2, 64, 2500, 2, [(2501, 1)], [(2501, 0)]), (16, 4, 128, 2100, 7, [(2103, 0)], [(2105, 1), (40, 2)])])
def test_blocks_that_are_not_finite_in_calls_cut_into_parts(use_list, fmt, n_q, n_kv, d, T, C, bad_k, bad_v):
    test_blocks_that_are_not_finite_reach_only_the_rows_that_see_them(api.IMPL_AUTO, use_list, fmt, 1, n_q, n_kv, d, T, C, bad_k, bad_v)


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("N,norms,agg", [(1, False, "max"), (5, True, "max"), (8, False, "mean"), (40, False, "max"), (40, True, "mean")])
def test_keys_that_are_not_finite_score_minus_infinity(fmt, N, norms, agg):
    inp = synth.make_chunk_inputs(6, 1, 4, 2, 128, [300], N, "bf16")
    inp.k[0, 0, 7, 3] = float("nan")
    inp.k[0, 1, 299, 100] = float("-inf")
    g = torch.Generator().manual_seed(8)
    qbar = torch.randn(1, 2, N, 128, generator=g)
    qbar = (qbar / qbar.norm(dim=-1, keepdim=True)).bfloat16().cuda()
    for impl in IMPLS:
        P = R.MxProblem(inp, fmt, n_retain=N, kv_budget=8, impl=impl)
        if norms:
            P.norms = torch.zeros(P.k.shape[:3], device="cuda")
            n = torch.from_numpy(1.0 / np.fmax(np.sqrt((P.k64 ** 2).sum(-1)), 1e-12)).float()
            P.norms.copy_(n)
            P.p.k_inv_norm = P.norms.data_ptr()
        P.p.query_agg = {"max": api.AGG_MAX, "mean": api.AGG_MEAN}[agg]
        scores = torch.full((1, 2, P.max_ctx), 7.0, device="cuda")
        api.quoka_score_keys_mx(P.p, P.mx, qbar, P.k, scores, P.ws)
        got = scores.double().cpu().numpy()
        for h, t in ((0, 7), (1, 299)):
            assert np.isnan(got[0, h, t]) if agg == "mean" else got[0, h, t] == -np.inf
            got[0, h, t] = 0
        want = O.score_keys(qbar[0].double().cpu().numpy(), np.nan_to_num(P.k64[0, :, :300]), 300, "cosine", agg)
        want[0, 7] = want[1, 299] = 0
        assert np.abs(got[0] - want).max() <= PA.SCORE_ATOL


@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("n_q,n_kv,d,lens,C,paged", [
    (8, 2, 128, [900, 130], 300, True), (32, 8, 128, [2000], 256, False), (8, 2, 64, [700], 200, True), (8, 8, 128, [5000], 40, False)])
def test_long_chunks_are_the_bf16_call_on_what_the_cache_reads_as(use_list, n_q, n_kv, d, lens, C, paged):
    """Every value of the cache is a bf16 number: the tensor-core kernels of chunks give what they give over a bf16 cache of them,
    up to the order in which 16 columns of a product are added up."""
    b = len(lens)
    inp = synth.make_chunk_inputs(31, b, n_q, n_kv, d, lens, C, "bf16")
    for fmt in FORMATS:
        P = R.MxProblem(inp, fmt, paged=paged, kv_budget=max(lens) // 2)
        rows = max(lens) + C
        k, v = (torch.zeros(b, n_kv, rows, d, dtype=torch.bfloat16, device="cuda") for _ in range(2))
        api.quoka_read_kv_mx(P.p, P.mx, P.k, P.v, 0, rows, k, v, P.ws)
        out = torch.empty_like(P.out)
        p = api.make_params(P.q, k, out, P.ctx_len, n_retain=16, kv_budget=max(lens) // 2, max_ctx_len=P.max_ctx)
        ws = api.alloc_workspace(p)
        if use_list:
            k_idx, k_cnt = P.listed(3)
            api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, None, P.ws)
            api.quoka_sparse_attn(p, P.q, k, v, k_idx, k_cnt, out, None, ws)
        else:
            api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, P.ws)
            api.quoka_dense_chunk_attn(p, P.q, k, v, out, None, ws)
        # one bf16 spacing of the output, and the fp32 sums' last bits where they nearly cancel
        diff = (P.out.float() - out.float()).abs()
        assert (diff <= out.float().abs() * 2.0 ** -7 + 1e-4).all(), float(diff.max())


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_workspace_of_the_longest_chunk_serves_the_last_one(fmt):
    inp = synth.make_chunk_inputs(33, 1, 8, 2, 128, [1500], 512, "bf16")
    P = R.MxProblem(inp, fmt, kv_budget=200)
    short = synth.make_chunk_inputs(34, 1, 8, 2, 128, [1500], 3, "bf16")
    S = R.MxProblem(short, fmt, kv_budget=200)
    assert P.ws.numel() >= S.ws.numel()
    want = []
    for ws in (S.ws, P.ws):
        api.quoka_dense_chunk_attn_mx(S.p, S.mx, S.q, S.k, S.v, S.out, None, ws)
        want.append(S.out.clone())
    assert torch.equal(*want)
    with pytest.raises(api.QuokaError) as e:
        api.quoka_dense_chunk_attn_mx(S.p, S.mx, S.q, S.k, S.v, S.out, None, S.ws[: api.quoka_workspace_size(S.p)])
    assert e.value.status == api.ERR_WORKSPACE


@pytest.mark.parametrize("fmt", FORMATS)
def test_empty_batches_entries_and_many_sequences(fmt):
    """More sequences than a warp has lanes, empty caches among them; generation steps and scores."""
    lens = [(37 * i) % 300 if i % 5 else 0 for i in range(45)]
    inp = synth.make_chunk_inputs(35, 45, 4, 2, 64, lens, 1, "bf16")
    P = R.MxProblem(inp, fmt, paged=True, kv_budget=20, n_retain=4)
    scores = torch.full((45, 2, P.max_ctx), 7.0, device="cuda")
    qbar = torch.nn.functional.normalize(torch.randn(45, 2, 1, 64, generator=torch.Generator().manual_seed(1)), dim=-1).bfloat16()
    api.quoka_score_keys_mx(P.p, P.mx, qbar.cuda(), P.k, scores, P.ws)
    k_idx, k_cnt = P.listed(5)
    dense = torch.empty_like(P.out)
    api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, None, P.ws)
    api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, dense, None, P.ws)
    torch.cuda.synchronize()
    assert api.quoka_last_device_status(P.ws) == 0
    for s, T in enumerate(lens):
        assert (scores[s, :, T:] == 7.0).all()
        if T:
            want = O.score_keys(qbar[s].double().numpy(), P.k64[s, :, :T], T)
            assert np.abs(PA.f64(scores[s, :, :T]) - want).max() <= PA.SCORE_ATOL
        PA.check_attention(PA.f64(P.out[s]), P.reference(s, use_list=True)[0], "bf16")
        PA.check_attention(PA.f64(dense[s]), P.reference(s)[0], "bf16")


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("C", [1, 4, 70])
def test_wide_ranges_of_scales(fmt, C):
    """Rows and blocks of very different magnitudes, queries with one large element: nothing of the operands' range shows."""
    inp = synth.make_chunk_inputs(36, 1, 4, 1, 128, [600], C, "bf16")
    r = np.random.default_rng(4)
    for x, lo, hi in ((inp.k, -14, 3), (inp.v, -30, 10)):
        e = torch.from_numpy(r.integers(lo, hi, (1, 1, x.shape[2], 4)).astype(np.float64)).repeat_interleave(32, -1)
        x.copy_((x.double() * 2.0 ** e).bfloat16())
    inp.q[..., 5] *= 64
    P = R.MxProblem(inp, fmt, kv_budget=100)
    api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, P.lse, P.ws)
    out, lse = P.reference(0)
    got = PA.f64(P.out[0])
    # weights and outputs in bf16 (fp16 weights in short chunks): half a spacing of the output and 2^-8 of the weighted magnitudes
    bound = 2.0 ** -8 * np.abs(out) + 2.0 ** -8 * np.abs(P.v64[0, 0, : 600 + C]).max(0)
    assert (np.abs(got - out) <= bound).all()
    # logits up to some hundreds: the sums of 128 products and the exponent's scaling in fp32
    assert np.abs(PA.f64(P.lse[0]) - lse).max() <= 2e-3 + 2.0 ** -18 * np.abs(lse).max()


@pytest.mark.parametrize("impl", IMPLS)
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("paged,C,n_retain,budget", [(True, 96, 24, 100), (False, 1, 8, 40), (True, 130, 200, 64), (True, 3, 2, 33)])
def test_algorithm_2_as_a_loop(impl, fmt, paged, C, n_retain, budget):
    """Append, select, score, select keys, attend: chunk after chunk from an empty cache, each against the oracle on what the
    cache holds, and the fused call against the staged ones."""
    b, n_q, n_kv, d, steps = 2, 8, 2, 128, 4
    pages = -(-steps * C // 64)
    rows = steps * C
    shape = (2 * pages + 1, n_kv, 64) if paged else (b, n_kv, rows)
    k, v, ks, vs = api.alloc_mx_cache(shape, d, fmt)
    table_host = np.random.default_rng(2).permutation(2 * pages).reshape(2, pages).astype(np.int32)
    table = torch.from_numpy(table_host).cuda() if paged else None
    norms = torch.zeros(shape, device="cuda")
    hist_k, hist_v = (np.zeros((b, n_kv, rows, d)) for _ in range(2))
    for i in range(steps):
        T = i * C
        inp = synth.make_chunk_inputs(40 + i, b, n_q, n_kv, d, 0, C, "bf16")
        q, k_new, v_new = inp.q.cuda(), inp.k.cuda(), inp.v.cuda()
        ctx = torch.full((b,), T, dtype=torch.int32, device="cuda")
        out, out_f = torch.empty_like(q), torch.empty_like(q)
        p = api.make_params(q, k, out, ctx, n_retain=n_retain, kv_budget=budget, max_ctx_len=T, block_table=table, impl=impl, kv_format=fmt)
        if not paged:
            assert p.kv_rows == rows
        p.k_inv_norm = norms.data_ptr()
        mx = api.make_mx_cache(fmt, ks, vs)
        ws = api.alloc_workspace(p, mx=mx)
        api.quoka_append_kv_mx(p, mx, k_new, v_new, k, v, norms, ws)
        hist_k[:, :, T:T + C] = R.values(*R.quantise(inp.k.double().numpy(), fmt), fmt)
        hist_v[:, :, T:T + C] = R.values(*R.quantise(inp.v.double().numpy(), fmt), fmt)
        cap, N = api.quoka_kv_budget_cap(p), min(n_retain, C)
        q_idx = torch.zeros(b, n_q, N, dtype=torch.int32, device="cuda")
        qbar = torch.zeros(b, n_kv, N, d, dtype=torch.bfloat16, device="cuda")
        scores = torch.zeros(b, n_kv, max(T, 1), device="cuda")
        k_idx, k_idx_f = (torch.zeros(b, n_kv, cap, dtype=torch.int32, device="cuda") for _ in range(2))
        k_cnt, k_cnt_f = (torch.zeros(b, dtype=torch.int32, device="cuda") for _ in range(2))
        lse = torch.zeros(b, n_q, C, device="cuda")
        api.quoka_select_queries(p, q, q_idx, qbar, ws)
        api.quoka_score_keys_mx(p, mx, qbar, k, scores, ws)
        api.quoka_select_keys(p, scores, k_idx, k_cnt, ws)
        api.quoka_sparse_attn_mx(p, mx, q, k, v, k_idx, k_cnt, out, lse, ws)
        api.quoka_prefill_chunk_mx(p, mx, q, k, v, out_f, k_idx_f, k_cnt_f, ws)
        torch.cuda.synchronize()
        assert api.quoka_last_device_status(ws) == 0
        assert torch.equal(k_idx, k_idx_f) and torch.equal(k_cnt, k_cnt_f)
        assert torch.equal(out, out_f)
        for s in range(b):
            B = O.key_budget(T, budget, 0.0)
            kk, vv = hist_k[s, :, :T + C], hist_v[s, :, :T + C]
            idx = k_idx[s].cpu().numpy()
            if T:
                sc = O.score_keys(PA.f64(qbar[s]), kk, T)
                assert np.abs(PA.f64(scores[s]) - sc).max() <= PA.SCORE_ATOL
                PA.check_key_selection(idx, sc, B)
            want, lse_o = O.sparse_attention(inp.q[s].double().numpy(), kk, vv, T, [idx[h, :B] for h in range(n_kv)])
            PA.check_attention(PA.f64(out[s]), want, "bf16")
            assert np.abs(PA.f64(lse[s]) - lse_o).max() <= 2e-3


@pytest.mark.parametrize("fmt", FORMATS)
def test_calls_capture_into_a_graph_and_run_on_another_stream(fmt):
    inp = synth.make_chunk_inputs(21, 2, 8, 2, 128, [300, 180], 5, "bf16")
    P = R.MxProblem(inp, fmt, paged=True, n_retain=5, kv_budget=64)
    want = []
    for _ in range(2):
        api.quoka_prefill_chunk_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, None, P.ws)
        dense = torch.empty_like(P.out)
        api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, dense, None, P.ws)
        torch.cuda.synchronize()
        want.append((P.out.clone(), dense.clone()))
    assert torch.equal(want[0][0], want[1][0]) and torch.equal(want[0][1], want[1][1])      # the same bits from run to run
    side = torch.cuda.Stream()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        api.quoka_prefill_chunk_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, None, P.ws, stream=side)
        api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, dense, None, P.ws, stream=side)
    for _ in range(3):
        P.out.zero_()
        dense.zero_()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(P.out, want[0][0]) and torch.equal(dense, want[0][1])
    P.ws.fill_(0xEE)                                          # scratch means nothing between calls
    P.ws[:256].zero_()
    graph.replay()
    torch.cuda.synchronize()
    assert torch.equal(P.out, want[0][0]) and torch.equal(dense, want[0][1])


# Chunks that are long enough for their rows to be unpacked first: 2048 query rows per KV head, 8192 over a whole cache of 128 columns.
UNPACKED = [(8, 1, 64, [700, 90], 257, True), (8, 2, 64, [130, 0], 513, False), (16, 1, 64, [333], 300, True), (8, 1, 128, [450, 1], 258, True),
            (12, 2, 128, [200], 345, False), (16, 1, 128, [600, 77], 513, True), (8, 1, 128, [64], 1025, False)]


@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("n_q,n_kv,d,lens,C,paged", UNPACKED)
def test_unpacked_chunks_are_the_bf16_call_on_what_the_cache_reads_as(use_list, n_q, n_kv, d, lens, C, paged):
    test_long_chunks_are_the_bf16_call_on_what_the_cache_reads_as(use_list, n_q, n_kv, d, lens, C, paged)


@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n_q,n_kv,d,T,C,bad_k,bad_v", [
    # blocks in cached rows, in the chunk, at the edges of an unpacking tile (64 rows of 128 columns, 128 of 64), in the last row
    (8, 1, 64, 300, 257, [], [(7, 1), (300 + 250, 0)]), (8, 1, 64, 90, 260, [(95, 0)], [(127, 1), (128, 0)]), (8, 1, 128, 190, 260, [], [(191, 3), (192, 2), (449, 0)]),
    (8, 1, 128, 40, 300, [(339, 1)], [(39, 2)]), (16, 1, 128, 70, 520, [], [(71, 0), (400, 3)]), (8, 1, 128, 0, 1030, [(1000, 1)], [(63, 0), (1029, 2)])])
def test_blocks_that_are_not_finite_in_unpacked_chunks(use_list, fmt, n_q, n_kv, d, T, C, bad_k, bad_v):
    test_blocks_that_are_not_finite_reach_only_the_rows_that_see_them(api.IMPL_AUTO, use_list, fmt, 1, n_q, n_kv, d, T, C, bad_k, bad_v)


@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d,n_q,C", [(64, 8, 300), (128, 16, 530)])
def test_chunks_convert_where_the_workspace_has_no_room_for_unpacked_rows(use_list, fmt, d, n_q, C):
    """quoka_workspace_size's bytes are enough; one byte less than what unpacking takes is too, and nothing behind them is written."""
    inp = synth.make_chunk_inputs(35, 2, n_q, 1, d, [400, 129], C, "bf16")
    P = R.MxProblem(inp, fmt, kv_budget=100, paged=True)
    least, full = api.quoka_workspace_size(P.p), P.ws.numel()
    assert least < full
    args = P.listed(5) if use_list else ()
    call = api.quoka_sparse_attn_mx if use_list else api.quoka_dense_chunk_attn_mx
    for n in (full, full - 1, least):
        ws = torch.full((full + 256,), 0xA5, dtype=torch.uint8, device="cuda")
        P.out.fill_(7.0)
        call(P.p, P.mx, P.q, P.k, P.v, *args, P.out, P.lse, ws[:n])
        assert (ws[n:] == 0xA5).all()
        for s in range(2):
            want, _ = P.reference(s, use_list=use_list)
            assert (np.abs(PA.f64(P.out[s]) - want) <= PA.attention_bound(want, "bf16")).all()


@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n_q,n_kv,d,lens,C,paged", [
    # units that a cluster shares: sequences with fewer granules of 32 keys than the cluster has CTAs, of no keys, one granule more than a CTA takes
    (8, 2, 128, [1700, 0, 33], 1, True), (4, 1, 128, [780], 1, False), (8, 1, 128, [3000, 5], 2, True), (4, 1, 64, [5000, 31, 64], 3, False), (8, 1, 64, [2100, 1], 3, True),
    (16, 2, 64, [1300, 0], 5, False), (32, 8, 128, [4003], 1, True), (32, 8, 128, [1500, 40], 4, False), (5, 5, 64, [1025, 1024, 7], 1, True)])
def test_few_rows_shared_in_clusters(use_list, fmt, n_q, n_kv, d, lens, C, paged):
    inp = synth.make_chunk_inputs(41, len(lens), n_q, n_kv, d, lens, C, "bf16")
    P = R.MxProblem(inp, fmt, paged=paged, kv_budget=max(lens) - 1)
    for _ in range(2):                                        # (the same bits every time)
        if use_list:
            k_idx, k_cnt = P.listed(3)
            api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, P.lse, P.ws)
        else:
            api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, P.lse, P.ws)
        first = P.out.clone() if _ == 0 else first
    assert torch.equal(first, P.out)
    for s in range(len(lens)):
        want, lse = P.reference(s, use_list=use_list)
        assert (np.abs(PA.f64(P.out[s]) - want) <= PA.attention_bound(want, "bf16")).all()
        assert np.abs(PA.f64(P.lse[s]) - lse).max() <= 1e-3


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("d", [64, 128])
def test_every_code_under_every_scale_reads_back(fmt, d, dtype):
    """quoka_read_kv_mx of scales that this library does not write too: the value, rounded once where bf16 or fp32 ends."""
    codes = 256 if fmt == api.KV_MXFP8 else 16
    code = (np.arange(256)[:, None] * 7 + np.arange(d * 8)).reshape(1, 1, 256 * 8, d) % codes
    code[np.isin(code, (0x7F, 0xFF)) & (fmt == api.KV_MXFP8)] = 0
    scale = np.repeat(np.arange(256), 8 * d // 32).reshape(1, 1, 2048, d // 32)
    kc, vc = (torch.from_numpy(R.pack(code.astype(np.uint8), fmt)).cuda() for _ in range(2))
    ks, vs = (torch.from_numpy(scale.astype(np.uint8)).cuda() for _ in range(2))
    q = torch.zeros(1, 1, 1, d, dtype=DTYPES[dtype], device="cuda")
    ctx = torch.tensor([2047], dtype=torch.int32, device="cuda")
    p = api.make_params(q, kc, torch.empty_like(q), ctx, n_retain=1, kv_budget=1, max_ctx_len=2047, kv_format=fmt)
    mx = api.make_mx_cache(fmt, ks, vs)
    k, v = (torch.zeros(1, 1, 2048, d, dtype=DTYPES[dtype], device="cuda") for _ in range(2))
    api.quoka_read_kv_mx(p, mx, kc, vc, 0, 2048, k, v, api.alloc_workspace(p, mx=mx))
    unit = R.values(code.astype(np.uint8), np.full_like(scale, 127).astype(np.uint8), fmt)
    with np.errstate(invalid="ignore", over="ignore"):
        want = unit * np.where(np.repeat(scale, 32, axis=-1) == 255, np.nan, np.exp2(np.repeat(scale, 32, axis=-1) - 127.0))
        want = torch.from_numpy(want).to(torch.float32).to(DTYPES[dtype])
    for got in (k.cpu(), v.cpu()):
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got[~torch.isnan(want)], want[~torch.isnan(want)])


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n_q,n_kv,d,C", [(8, 2, 128, 1), (8, 1, 64, 5), (8, 1, 64, 260), (8, 2, 128, 70)])
def test_a_captured_call_follows_the_lengths_on_the_device(fmt, n_q, n_kv, d, C):
    inp = synth.make_chunk_inputs(23, 2, n_q, n_kv, d, [2500, 2500], C, "bf16")
    P = R.MxProblem(inp, fmt, n_retain=4, kv_budget=300)
    dense = torch.empty_like(P.out)

    def calls(stream=None):
        api.quoka_prefill_chunk_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, None, P.ws, stream=stream)
        api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, dense, None, P.ws, stream=stream)
    calls()
    side, graph = torch.cuda.Stream(), torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=side):
        calls(side)
    for lens in ([2500, 2500], [1, 2500], [0, 31], [777, 300], [299, 0]):
        P.ctx_len.copy_(torch.tensor(lens, dtype=torch.int32))
        graph.replay()
        torch.cuda.synchronize()
        got = P.out.clone(), dense.clone()
        P.out.zero_(), dense.zero_()
        calls()
        torch.cuda.synchronize()
        assert torch.equal(got[0], P.out) and torch.equal(got[1], dense)
        assert torch.isfinite(got[0].float()).all() and torch.isfinite(got[1].float()).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_two_streams_at_once(fmt):
    """Calls on two streams with a workspace each: few rows in clusters beside a chunk whose rows are unpacked."""
    problems = [R.MxProblem(synth.make_chunk_inputs(51, 1, 8, 2, 128, [3000], 1, "bf16"), fmt, n_retain=1, kv_budget=1500),
                R.MxProblem(synth.make_chunk_inputs(52, 2, 8, 1, 64, [1000, 77], 300, "bf16"), fmt, n_retain=8, kv_budget=200, paged=True)]

    def call(P, out, stream=None):
        api.quoka_prefill_chunk_mx(P.p, P.mx, P.q, P.k, P.v, out, None, None, P.ws, stream=stream)
    want = []
    for P in problems:
        call(P, P.out)
        want.append(P.out.clone())
    streams = [torch.cuda.Stream() for _ in problems]
    torch.cuda.synchronize()
    for _ in range(30):
        for P, s in zip(problems, streams):
            call(P, P.out, s)
    torch.cuda.synchronize()
    for P, w in zip(problems, want):
        assert torch.equal(P.out, w) and api.quoka_last_device_status(P.ws) == 0


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("n_q,n_kv,d,C", [(8, 2, 128, 1), (8, 1, 64, 4), (8, 2, 128, 70), (8, 1, 64, 260), (8, 1, 128, 300)])
def test_lists_that_are_empty_short_or_name_a_row_twice(fmt, n_q, n_kv, d, C):
    inp = synth.make_chunk_inputs(27, 3, n_q, n_kv, d, [900, 900, 40], C, "bf16")
    P = R.MxProblem(inp, fmt, kv_budget=850)
    P.listed(9, counts=[0, 801, 40])
    P.idx_host[1, :, 5] = P.idx_host[1, :, 4]
    P.idx_host[1, :, :7] = P.idx_host[1, :, :7][:, ::-1]               # (nor in order)
    k_idx, k_cnt = torch.from_numpy(P.idx_host).cuda(), torch.tensor(P.cnt_host, dtype=torch.int32, device="cuda")
    api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, None, P.ws)
    torch.cuda.synchronize()
    for s in range(3):
        PA.check_attention(PA.f64(P.out[s]), P.reference(s, use_list=True)[0], "bf16")
