"""The calls on a microscaled cache refuse bad arguments on the host and launch nothing (no GPU needed)."""
import ctypes as C

import pytest

from tests.test_abi import good_params, lib  # noqa: F401  (the fixture)


def good_mx(api):
    return api.QuokaMxCache(api.KV_MXFP8, 0x10000, 0x20000)


def calls(lib, p, mx, ws=0x4000, ws_bytes=1 << 33, ptr=0x1000):  # noqa: F811
    pp, pm = C.byref(p), None if mx is None else C.byref(mx)
    return [
        lambda: lib.quoka_append_kv_mx(pp, pm, ptr, 0x2000, 0x3000, 0x5000, None, ws, ws_bytes, None),
        lambda: lib.quoka_read_kv_mx(pp, pm, ptr, 0x2000, 0, 5, 0x3000, 0x5000, ws, ws_bytes, None),
        lambda: lib.quoka_score_keys_mx(pp, pm, ptr, 0x2000, 0x3000, ws, ws_bytes, None),
        lambda: lib.quoka_sparse_attn_mx(pp, pm, ptr, 0x2000, 0x3000, 0x5000, 0x6000, 0x7000, None, ws, ws_bytes, None),
        lambda: lib.quoka_dense_chunk_attn_mx(pp, pm, ptr, 0x2000, 0x3000, 0x7000, None, ws, ws_bytes, None),
        lambda: lib.quoka_prefill_chunk_mx(pp, pm, ptr, 0x2000, 0x3000, 0x7000, None, None, ws, ws_bytes, None),
    ]


@pytest.mark.parametrize("field,value,status", [
    ("head_dim", 96, 2), ("n_kv_heads", 3, 1), ("batch", 0, 1), ("page_size", 16, 2), ("dtype", 7, 1), ("kv_rows", 100, 1),
    ("chunk_len", 0, 1), ("impl", 9, 1), ("kv_stride_t", 136, 1), ("kv_stride_h", 4352 * 128 + 16, 1), ("kv_stride_b", 8, 1),
    ("ctx_len", None, 1), ("max_ctx_len", -1, 1)])
def test_bad_params(lib, field, value, status):  # noqa: F811
    from paper_2602_08722_b200 import api
    p, mx = good_params(), good_mx(api)
    setattr(p, field, value)
    before = api.quoka_launch_count()
    n = C.c_size_t(0)
    assert lib.quoka_workspace_size_mx(C.byref(p), C.byref(mx), C.byref(n)) == status
    for call in calls(lib, p, mx):
        assert call() == status
    assert api.quoka_launch_count() == before


@pytest.mark.parametrize("field,value", [("format", 0), ("format", 3), ("k_scale", None), ("v_scale", None), ("k_scale", 0x10004), ("v_scale", 0x20008)])
def test_bad_descriptions_of_the_cache(lib, field, value):  # noqa: F811
    from paper_2602_08722_b200 import api
    p, mx = good_params(), good_mx(api)
    setattr(mx, field, value)
    before = api.quoka_launch_count()
    n = C.c_size_t(0)
    assert lib.quoka_workspace_size_mx(C.byref(p), C.byref(mx), C.byref(n)) == api.ERR_INVALID_ARG
    for call in calls(lib, p, mx):
        assert call() == api.ERR_INVALID_ARG
    for call in calls(lib, p, None):
        assert call() == api.ERR_INVALID_ARG
    assert api.quoka_launch_count() == before


def test_pointers_workspace_and_rows(lib):  # noqa: F811
    from paper_2602_08722_b200 import api
    p, mx = good_params(), good_mx(api)
    before = api.quoka_launch_count()
    pp, pm = C.byref(p), C.byref(mx)
    need = api.quoka_workspace_size_mx(p, mx)
    assert need >= 256
    for ptr in (None, 0x1008):
        for call in calls(lib, p, mx, ptr=ptr):
            assert call() == api.ERR_INVALID_ARG
    for ws, n in ((None, 1 << 33), (0x4010, 1 << 33), (0x4000, 255)):
        for call in calls(lib, p, mx, ws=ws, ws_bytes=n):
            assert call() == api.ERR_WORKSPACE
    for first, n in ((-2, 5), (0, -1)):
        assert lib.quoka_read_kv_mx(pp, pm, 0x1000, 0x2000, first, n, 0x3000, 0x5000, 0x4000, 1 << 33, None) == api.ERR_INVALID_ARG
    # values come with their output and the other way round; no rows is nothing to do
    assert lib.quoka_read_kv_mx(pp, pm, 0x1000, 0x2000, 0, 5, 0x3000, None, 0x4000, 1 << 33, None) == api.ERR_INVALID_ARG
    assert lib.quoka_read_kv_mx(pp, pm, 0x1000, None, 0, 5, 0x3000, 0x5000, 0x4000, 1 << 33, None) == api.ERR_INVALID_ARG
    assert lib.quoka_read_kv_mx(pp, pm, 0x1000, None, 0, 0, 0x3000, None, 0x4000, 1 << 33, None) == api.OK
    assert lib.quoka_workspace_size_mx(pp, pm, None) == api.ERR_INVALID_ARG
    assert api.quoka_launch_count() == before


def test_scale_tensors_are_dense():
    import torch
    from paper_2602_08722_b200 import api
    scale = torch.zeros(2, 3, 8, 4, dtype=torch.uint8)
    assert api.make_mx_cache(api.KV_MXFP4, scale, scale).format == api.KV_MXFP4
    with pytest.raises(ValueError):
        api.make_mx_cache(api.KV_MXFP4, scale.transpose(1, 2), scale)
    k, v, ks, vs = api.alloc_mx_cache((2, 3, 8), 128, api.KV_MXFP4, device="cpu")
    assert k.shape == (2, 3, 8, 64) and vs.shape == (2, 3, 8, 4)
