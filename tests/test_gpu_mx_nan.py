"""Values that are not finite in a microscaled cache."""
import numpy as np
import pytest

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
