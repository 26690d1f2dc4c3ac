"""What the calls over a microscaled cache refuse, before anything is launched (no GPU needed)."""
import pytest

from tests.test_abi import good_params, lib  # noqa: F401  (the fixture)
from tests.test_mx_abi import calls, good_mx


@pytest.mark.parametrize("n_retain,C_,d", [(513, 700, 128), (600, 600, 64), (8192, 1025, 128)])
def test_the_fused_call_refuses_before_its_first_launch(lib, n_retain, C_, d):  # noqa: F811
    """More retained queries than the tensor-core scoring takes, with IMPL_TENSOR: refused as a whole."""
    from paper_2602_08722_b200 import api
    p, mx = good_params(), good_mx(api)
    p.impl, p.head_dim, p.chunk_len, p.n_retain = api.IMPL_TENSOR, d, C_, n_retain
    p.kv_rows = p.max_ctx_len + C_
    before = api.quoka_launch_count()
    fused = calls(lib, p, mx)[-1]
    assert fused() == api.ERR_UNSUPPORTED
    assert api.quoka_launch_count() == before
