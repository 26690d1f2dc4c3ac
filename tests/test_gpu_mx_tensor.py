"""The tcgen05 kernels over a microscaled cache where the default takes others: few query rows, few retained queries (impl = TENSOR)."""
import numpy as np
import pytest
import torch

from oracle import quoka_oracle as O
from paper_2602_08722_b200 import api, synth
from tests import mx_reference as R
from tests import parity as PA

pytestmark = pytest.mark.gpu
FORMATS = [api.KV_MXFP8, api.KV_MXFP4]


@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("b,n_q,n_kv,d,lens,C,paged", [
    (1, 4, 1, 64, [1], 1, False), (2, 8, 2, 128, [0, 70], 1, True), (1, 34, 2, 128, [333], 1, False), (2, 6, 2, 64, [127, 128], 2, True),
    (2, 16, 4, 128, [61, 3000], 4, False), (1, 8, 1, 64, [777], 5, True), (2, 8, 8, 128, [130, 40], 9, True), (1, 6, 2, 128, [1200], 11, False)])
def test_attention(use_list, fmt, b, n_q, n_kv, d, lens, C, paged):
    inp = synth.make_chunk_inputs(91, b, n_q, n_kv, d, lens, C, "bf16")
    P = R.MxProblem(inp, fmt, paged=paged, impl=api.IMPL_TENSOR, kv_budget=max(1, max(lens) // 3) if use_list else 16)
    if use_list:
        k_idx, k_cnt = P.listed(3)
        api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, P.lse, P.ws)
    else:
        api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, P.lse, P.ws)
    assert api.quoka_last_device_status(P.ws) == 0
    for s in range(b):
        out, lse = P.reference(s, use_list=use_list)
        PA.check_attention(PA.f64(P.out[s]), out, "bf16")
        assert np.abs(PA.f64(P.lse[s]) - lse).max() <= 2e-3


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("norms,agg", [(False, "max"), (True, "mean")])
@pytest.mark.parametrize("n_kv,d,lens,N,paged", [(2, 128, [1], 1, False), (1, 64, [513], 1, True), (5, 128, [700, 255], 7, True), (3, 64, [0, 129, 64], 8, True)])
def test_scores(fmt, norms, agg, n_kv, d, lens, N, paged):
    b = len(lens)
    inp = synth.make_chunk_inputs(92, b, 2 * n_kv, n_kv, d, lens, N, "bf16")
    P = R.MxProblem(inp, fmt, paged=paged, n_retain=N, kv_budget=8, impl=api.IMPL_TENSOR, cached_norms=norms)
    P.p.query_agg = {"max": api.AGG_MAX, "mean": api.AGG_MEAN}[agg]
    qbar = torch.nn.functional.normalize(torch.randn(b, n_kv, N, d, generator=torch.Generator().manual_seed(8)), dim=-1).bfloat16()
    scores = torch.full((b, n_kv, P.max_ctx), 7.0, device="cuda")
    api.quoka_score_keys_mx(P.p, P.mx, qbar.cuda(), P.k, scores, P.ws)
    assert api.quoka_last_device_status(P.ws) == 0
    for s, T in enumerate(lens):
        assert (scores[s, :, T:] == 7.0).all()
        if T:
            want = O.score_keys(qbar[s].double().numpy(), P.k64[s, :, :T], T, "cosine", agg)
            assert np.abs(PA.f64(scores[s, :, :T]) - want).max() <= PA.SCORE_ATOL


@pytest.mark.parametrize("fmt", FORMATS)
@pytest.mark.parametrize("impl", [api.IMPL_AUTO, api.IMPL_SIMT, api.IMPL_TENSOR])
@pytest.mark.parametrize("n_q,n_kv,d,C,n_retain,budget,T", [(8, 2, 128, 1, 1, 40, 700), (16, 4, 64, 4, 2, 100, 333), (8, 2, 128, 40, 16, 200, 900),
                                                            (8, 1, 64, 300, 32, 250, 1000), (8, 2, 128, 520, 300, 300, 1100), (8, 2, 128, 30, 512, 50, 0)])
def test_the_fused_call_against_the_oracle(fmt, impl, n_q, n_kv, d, C, n_retain, budget, T):
    """One chunk, from the queries to the output; long ones attend to rows unpacked behind the selection."""
    inp = synth.make_chunk_inputs(93, 1, n_q, n_kv, d, [T], C, "bf16")
    P = R.MxProblem(inp, fmt, paged=T > 0, n_retain=n_retain, kv_budget=budget, impl=impl)
    N, cap = min(n_retain, C), api.quoka_kv_budget_cap(P.p)
    q_idx = torch.zeros(1, n_q, N, dtype=torch.int32, device="cuda")
    qbar = torch.zeros(1, n_kv, N, d, dtype=torch.bfloat16, device="cuda")
    k_idx = torch.full((1, n_kv, cap), 7, dtype=torch.int32, device="cuda")
    k_cnt = torch.zeros(1, dtype=torch.int32, device="cuda")
    api.quoka_select_queries(P.p, P.q, q_idx, qbar, P.ws)
    api.quoka_prefill_chunk_mx(P.p, P.mx, P.q, P.k, P.v, P.out, k_idx, k_cnt, P.ws)
    assert api.quoka_last_device_status(P.ws) == 0
    B = O.key_budget(T, budget, 0.0)
    assert k_cnt.tolist() == [B]
    idx = k_idx[0].cpu().numpy()
    if T:
        PA.check_key_selection(idx, O.score_keys(PA.f64(qbar[0]), P.k64[0, :, :T], T), B)
    want, _ = O.sparse_attention(inp.q[0].double().numpy(), P.k64[0, :, :T + C], P.v64[0, :, :T + C], T, [idx[h, :B] for h in range(n_kv)])
    PA.check_attention(PA.f64(P.out[0]), want, "bf16")


@pytest.mark.parametrize("fmt", FORMATS)
def test_a_refused_fused_call_launches_nothing(fmt):
    inp = synth.make_chunk_inputs(94, 1, 4, 2, 64, [100], 600, "bf16")
    P = R.MxProblem(inp, fmt, n_retain=600, kv_budget=20, impl=api.IMPL_TENSOR)
    before = api.quoka_launch_count()
    with pytest.raises(api.QuokaError) as e:
        api.quoka_prefill_chunk_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, None, P.ws)
    assert e.value.status == api.ERR_UNSUPPORTED and api.quoka_launch_count() == before
    assert (P.out == 7.0).all()


@pytest.mark.parametrize("impl", [api.IMPL_SIMT, api.IMPL_TENSOR])
@pytest.mark.parametrize("n_q,n_kv,d,C", [(8, 2, 128, 1), (8, 1, 64, 5)])
def test_other_kernels_than_the_few_row_ones_do_not_need_their_scratch(impl, n_q, n_kv, d, C):
    """The bf16 call's workspace is enough, and nothing behind it is written."""
    inp = synth.make_chunk_inputs(95, 1, n_q, n_kv, d, [2500], C, "bf16")
    P = R.MxProblem(inp, api.KV_MXFP8, n_retain=4, kv_budget=300, impl=impl)
    n = api.quoka_workspace_size(P.p)
    ws = torch.full((n + (1 << 22),), 0xA5, dtype=torch.uint8, device="cuda")
    ws[:256] = 0
    api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, ws[:n])
    PA.check_attention(PA.f64(P.out[0]), P.reference(0)[0], "bf16")
    api.quoka_prefill_chunk_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, None, ws[:n])
    assert api.quoka_last_device_status(ws) == 0 and (ws[n:] == 0xA5).all()
