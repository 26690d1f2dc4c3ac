"""Lists with as many entries as the cache has rows that are not its rows in order: every kernel attends to what the list names."""
import numpy as np
import pytest
import torch

from oracle import quoka_oracle as O
from paper_2602_08722_b200 import api, synth
from tests import mx_reference as R
from tests import parity as PA

pytestmark = pytest.mark.gpu
# few query rows; chunks that convert; long ones, unpacked over the microscaled cache
SHAPES = [(8, 2, 128, 1), (8, 1, 64, 3), (8, 2, 128, 70), (8, 2, 64, 200), (8, 1, 64, 300), (8, 1, 128, 300)]
T = 300


def lists(n_kv, kind):
    r = np.random.default_rng(5)
    rows = {"twice": lambda: np.sort(r.integers(0, T // 2, T)), "reversed": lambda: np.arange(T)[::-1], "any order, some twice": lambda: r.integers(0, T, T)}[kind]
    return np.stack([rows() for _ in range(n_kv)])[None].astype(np.int32)


@pytest.mark.parametrize("kind", ["twice", "reversed", "any order, some twice"])
@pytest.mark.parametrize("fmt", [api.KV_NATIVE, api.KV_MXFP8, api.KV_MXFP4])
@pytest.mark.parametrize("impl", [api.IMPL_AUTO, api.IMPL_SIMT, api.IMPL_TENSOR])
@pytest.mark.parametrize("n_q,n_kv,d,C", SHAPES)
def test_a_list_as_long_as_the_cache(kind, fmt, impl, n_q, n_kv, d, C):
    inp = synth.make_chunk_inputs(71, 1, n_q, n_kv, d, [T], C, "bf16")
    idx = lists(n_kv, kind)
    k_idx, k_cnt = torch.from_numpy(idx).cuda(), torch.tensor([T], dtype=torch.int32, device="cuda")
    if fmt == api.KV_NATIVE:
        q, k, v = inp.q.cuda(), inp.k.cuda(), inp.v.cuda()
        out = torch.empty_like(q)
        ctx = inp.ctx_len.cuda()
        p = api.make_params(q, k, out, ctx, n_retain=16, kv_budget=T, max_ctx_len=T, impl=impl)
        ws = api.alloc_workspace(p)
        api.quoka_sparse_attn(p, q, k, v, k_idx, k_cnt, out, None, ws)
        k64, v64 = (x[0].double().numpy() for x in (inp.k, inp.v))
    else:
        P = R.MxProblem(inp, fmt, kv_budget=T, max_ctx_len=T, impl=impl)
        out, ws = P.out, P.ws
        api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, out, None, ws)
        k64, v64 = P.k64[0], P.v64[0]
    assert api.quoka_last_device_status(ws) == 0
    want, _ = O.sparse_attention(inp.q[0].double().numpy(), k64[:, :T + C], v64[:, :T + C], T, [idx[0, h] for h in range(n_kv)])
    PA.check_attention(PA.f64(out[0]), want, "bf16")


@pytest.mark.parametrize("fmt", [api.KV_NATIVE, api.KV_MXFP8])
@pytest.mark.parametrize("n_q,n_kv,d,C", SHAPES)
def test_the_rows_in_order_give_the_same_bits_as_in_the_fused_call(fmt, n_q, n_kv, d, C):
    """A budget that covers the cache: the selection's list is the rows in order, which the fused call knows."""
    inp = synth.make_chunk_inputs(72, 1, n_q, n_kv, d, [T], C, "bf16")
    k_idx = torch.arange(T, dtype=torch.int32).repeat(1, n_kv, 1).cuda()
    k_cnt = torch.tensor([T], dtype=torch.int32, device="cuda")
    if fmt == api.KV_NATIVE:
        q, k, v = inp.q.cuda(), inp.k.cuda(), inp.v.cuda()
        out, fused = torch.empty_like(q), torch.empty_like(q)
        ctx = inp.ctx_len.cuda()
        p = api.make_params(q, k, out, ctx, n_retain=16, kv_budget=T, max_ctx_len=T)
        ws = api.alloc_workspace(p)
        api.quoka_sparse_attn(p, q, k, v, k_idx, k_cnt, out, None, ws)
        api.quoka_prefill_chunk(p, q, k, v, fused, None, None, ws)
        if C == 1:                                            # (one launch that attends to what it selects, and adds up in another order)
            assert (out.float() - fused.float()).abs().max() <= 2e-2
            return
    else:
        P = R.MxProblem(inp, fmt, kv_budget=T, max_ctx_len=T)
        out, fused = P.out, torch.empty_like(P.out)
        api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, out, None, P.ws)
        api.quoka_prefill_chunk_mx(P.p, P.mx, P.q, P.k, P.v, fused, None, None, P.ws)
    assert torch.equal(out, fused)


@pytest.mark.parametrize("kind", ["twice", "any order, some twice"])
@pytest.mark.parametrize("fmt", [api.KV_NATIVE, api.KV_MXFP8, api.KV_MXFP4])
@pytest.mark.parametrize("n_q,n_kv,d,C", [(4, 2, 128, 1), (4, 2, 64, 70)])
def test_a_list_as_long_as_the_cache_of_f32_queries(kind, fmt, n_q, n_kv, d, C):
    inp = synth.make_chunk_inputs(73, 1, n_q, n_kv, d, [T], C, "f32")
    idx = lists(n_kv, kind)
    k_idx, k_cnt = torch.from_numpy(idx).cuda(), torch.tensor([T], dtype=torch.int32, device="cuda")
    if fmt == api.KV_NATIVE:
        q, k, v = inp.q.cuda(), inp.k.cuda(), inp.v.cuda()
        out = torch.empty_like(q)
        ctx = inp.ctx_len.cuda()
        p = api.make_params(q, k, out, ctx, n_retain=16, kv_budget=T, max_ctx_len=T)
        api.quoka_sparse_attn(p, q, k, v, k_idx, k_cnt, out, None, api.alloc_workspace(p))
        k64, v64 = (x[0].double().numpy() for x in (inp.k, inp.v))
    else:
        P = R.MxProblem(inp, fmt, kv_budget=T, max_ctx_len=T)
        out = P.out
        api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, out, None, P.ws)
        k64, v64 = P.k64[0], P.v64[0]
    want, _ = O.sparse_attention(inp.q[0].double().numpy(), k64[:, :T + C], v64[:, :T + C], T, [idx[0, h] for h in range(n_kv)])
    PA.check_attention(PA.f64(out[0]), want, "f32")
