"""Values that are not finite in a microscaled cache, and e4m3's codes of NaN."""
import numpy as np
import pytest
import torch

from paper_2602_08722_b200 import api, synth
from tests import mx_reference as R
from tests import parity as PA

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", [api.KV_MXFP8, api.KV_MXFP4])
@pytest.mark.parametrize("impl", [api.IMPL_AUTO, api.IMPL_SIMT])
@pytest.mark.parametrize("use_list", [False, True])
@pytest.mark.parametrize("n_q,n_kv,d,C", [(8, 2, 128, 64), (4, 1, 64, 100), (16, 2, 128, 200), (4, 1, 128, 1), (8, 1, 64, 4)])
def test_a_value_that_is_not_finite_among_keys_that_weigh_nothing(fmt, impl, use_list, n_q, n_kv, d, C):
    """The rows that see it have NaN in its 32 columns, however the keys are cut into parts; their other columns are right."""
    T, bad, blk = 4000, 17, 1
    inp = synth.make_chunk_inputs(81, 1, n_q, n_kv, d, [T], C, "bf16")
    inp.q[..., 0] = 8
    inp.k[..., 0] = 0
    inp.k[:, :, :3200, 0] = -150 * d ** 0.5 / 8                  # weights below 2^-200
    inp.v[0, 0, bad, 32 * blk + 3] = float("nan")
    P = R.MxProblem(inp, fmt, kv_budget=T, max_ctx_len=T, impl=impl)
    k_idx, k_cnt = P.listed(3)
    if use_list:
        api.quoka_sparse_attn_mx(P.p, P.mx, P.q, P.k, P.v, k_idx, k_cnt, P.out, None, P.ws)
    else:
        api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, P.ws)
    got = PA.f64(P.out[0])
    marked = np.zeros(got.shape, bool)
    marked[:n_q // n_kv, :, 32 * blk:32 * blk + 32] = True
    assert np.isnan(got[marked]).all()
    P.v64 = np.nan_to_num(P.v64)
    want, _ = P.reference(0)
    assert (np.abs(got - want)[~marked] <= PA.attention_bound(want, "bf16")[~marked]).all()


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("d", [64, 128])
def test_codes_of_nan_read_back_as_nan(d, dtype):
    """e4m3's two codes that are no number (0x7F, 0xFF), in every place of a block, under every scale."""
    code = ((np.arange(2048)[:, None] * 5 + np.arange(d)) % 256).astype(np.uint8).reshape(1, 1, 2048, d)
    code[0, 0, :256] = 0x38                                   # ones, and one code of NaN in each place
    for i in range(256):
        code[0, 0, i, i % d] = 0x7F if i < 128 else 0xFF
    scale = np.repeat(np.arange(256), 8 * d // 32).reshape(1, 1, 2048, d // 32).astype(np.uint8)
    scale[0, 0, :256] = 127
    kc, vc = (torch.from_numpy(code).cuda() for _ in range(2))
    ks, vs = (torch.from_numpy(scale).cuda() for _ in range(2))
    q = torch.zeros(1, 1, 1, d, dtype=dtype, device="cuda")
    ctx = torch.tensor([2047], dtype=torch.int32, device="cuda")
    p = api.make_params(q, kc, torch.empty_like(q), ctx, n_retain=1, kv_budget=1, max_ctx_len=2047, kv_format=api.KV_MXFP8)
    mx = api.make_mx_cache(api.KV_MXFP8, ks, vs)
    k, v = (torch.zeros(1, 1, 2048, d, dtype=dtype, device="cuda") for _ in range(2))
    api.quoka_read_kv_mx(p, mx, kc, vc, 0, 2048, k, v, api.alloc_workspace(p, mx=mx))
    element = torch.from_numpy(code).view(torch.float8_e4m3fn).float().numpy().astype(np.float64)
    with np.errstate(invalid="ignore", over="ignore"):
        s = np.repeat(scale, 32, axis=-1)
        want = torch.from_numpy(element * np.where(s == 255, np.nan, np.exp2(s - 127.0))).to(torch.float32).to(dtype)
    assert torch.isnan(want).sum() > 256
    for got in (k.cpu(), v.cpu()):
        assert torch.equal(torch.isnan(got), torch.isnan(want))
        assert torch.equal(got[~torch.isnan(want)], want[~torch.isnan(want)])


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("code", [0x7F, 0xFF])
def test_codes_of_nan_in_the_scalar_kernels(code, dtype):
    """A value of that code makes its column NaN in the rows that see it, a key of it those rows, and its score minus infinity."""
    T, C, d = 40, 5, 64
    inp = synth.make_chunk_inputs(82, 1, 2, 2, d, [T], C, dtype)
    P = R.MxProblem(inp, api.KV_MXFP8, kv_budget=8, n_retain=C, impl=api.IMPL_SIMT)
    P.v[0, 0, 7, 33] = code
    P.k[0, 1, 9, 2] = code
    api.quoka_dense_chunk_attn_mx(P.p, P.mx, P.q, P.k, P.v, P.out, None, P.ws)
    got = PA.f64(P.out[0])
    bad = np.zeros(got.shape, bool)
    bad[0, :, 33] = True
    bad[1] = True
    assert (np.isnan(got) == bad).all()
    want, _ = P.reference(0)
    assert (np.abs(got - want)[~bad] <= PA.attention_bound(want, dtype)[~bad]).all()
    qbar = torch.nn.functional.normalize(torch.randn(1, 2, C, d, generator=torch.Generator().manual_seed(1)), dim=-1).to(P.q.dtype).cuda()
    scores = torch.zeros(1, 2, P.max_ctx, device="cuda")
    api.quoka_score_keys_mx(P.p, P.mx, qbar, P.k, scores, P.ws)
    assert (torch.isinf(scores[0]).nonzero().cpu().tolist()) == [[1, 9]] and scores[0, 1, 9] < 0
