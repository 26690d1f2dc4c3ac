"""What the calls over a microscaled cache refuse, before anything is launched (no GPU needed)."""
import ctypes as C

import pytest

from tests.test_abi import good_params, lib  # noqa: F401  (the fixture)
from tests.test_mx_abi import calls, good_mx


def head_major(p, elements):
    """Heads outermost: n_kv_heads times `elements`, of which a page, or a sequence, has a short stride."""
    p.n_q_heads, p.n_kv_heads = 8, 8
    p.kv_stride_h = elements
    p.kv_stride_t = 128


@pytest.mark.parametrize("paged", [False, True])
def test_caches_that_32_bit_places_do_not_reach(lib, paged):  # noqa: F811
    """Places are counted in 32 bits of 16 (microscaled) or 8 elements (bf16): a cache beyond that is not for the tensor-core kernels, whichever of
    its strides is the longest.  (Shown with IMPL_TENSOR, which refuses; the default takes the scalar kernels.)"""
    from paper_2602_08722_b200 import api
    p, mx = good_params(), good_mx(api)
    p.impl = api.IMPL_TENSOR
    if paged:
        pages = 1 << 20
        p.page_size, p.max_pages_per_seq, p.block_table, p.kv_rows = 64, 128, 0x1000, pages
        p.kv_stride_b = 64 * 128
        head_major(p, pages * 64 * 128)                       # 2^33 elements a head, 2^36 in all
    else:
        p.kv_rows = 1 << 26
        p.kv_stride_b = (1 << 26) * 128
        head_major(p, (1 << 26) * 128)
    before = api.quoka_launch_count()
    _, _, score, sparse, dense, fused = calls(lib, p, mx)
    for call in (score, sparse, dense, fused):
        assert call() == api.ERR_UNSUPPORTED
    pp = C.byref(p)
    assert lib.quoka_dense_chunk_attn(pp, 0x1000, 0x2000, 0x3000, 0x7000, None, 0x4000, 1 << 40, None) == api.ERR_UNSUPPORTED
    assert lib.quoka_prefill_chunk(pp, 0x1000, 0x2000, 0x3000, 0x7000, None, None, 0x4000, 1 << 40, None) == api.ERR_UNSUPPORTED
    assert api.quoka_launch_count() == before


@pytest.mark.parametrize("paged", [False, True])
def test_the_largest_caches_that_they_do_reach(lib, paged):  # noqa: F811
    """Just inside: 2^32 - 2 units of 16 elements, of a microscaled cache (not refused for its size: what is refused here is a workspace)."""
    from paper_2602_08722_b200 import api
    p, mx = good_params(), good_mx(api)
    p.impl, p.n_q_heads, p.n_kv_heads = api.IMPL_TENSOR, 8, 8
    last = (2 ** 32 - 2) * 16
    if paged:
        p.page_size, p.max_pages_per_seq, p.block_table, p.kv_rows = 64, 128, 0x1000, 1 << 16
        p.kv_stride_b = 64 * 128
        p.kv_stride_t = 128
        p.kv_stride_h = (last - 128 - 63 * 128 - (p.kv_rows - 1) * p.kv_stride_b) // 7 // 32 * 32
    else:
        p.kv_stride_b, p.kv_stride_t = 8 * 4352 * 128, 128
        p.kv_stride_h = (last - 128 - (p.kv_rows - 1) * 128) // 7 // 32 * 32
    assert calls(lib, p, mx, ws_bytes=255)[-1]() == api.ERR_WORKSPACE
    p.kv_stride_h += 32 * 16
    assert calls(lib, p, mx, ws_bytes=255)[-1]() == api.ERR_UNSUPPORTED


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
