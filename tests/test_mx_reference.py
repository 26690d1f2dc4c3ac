"""The quantiser that the kernels of the microscaled cache are compared with, against the definition by brute force (CPU)."""
import numpy as np
import pytest

from paper_2602_08722_b200 import api
from tests import mx_reference as R

FORMATS = [api.KV_MXFP8, api.KV_MXFP4]


@pytest.mark.parametrize("fmt", FORMATS)
def test_nearest_element_of_the_smallest_scale_that_reaches(fmt):
    r = np.random.default_rng(3)
    x = r.normal(size=(40, 32)) * 2.0 ** r.integers(-70, 20, (40, 1))
    x[0] = 0
    x[1, 1:] = 0
    codes, scale = R.quantise(x, fmt)
    vals = R.values(codes, scale, fmt)
    el = R.element_values(fmt)
    el = el[np.isfinite(el)]
    most = el.max()
    for i in range(len(x)):
        amax = np.abs(x[i]).max()
        e = int(scale[i, 0]) - 127
        assert R.E_MIN <= e <= R.E_MAX
        assert amax <= most * 2.0 ** e or e == R.E_MAX
        assert e == R.E_MIN or amax > most * 2.0 ** (e - 1)
        for j in range(32):
            want = np.clip(x[i, j], -most * 2.0 ** e, most * 2.0 ** e)
            best = np.abs(el * 2.0 ** e - want).min()
            assert abs(vals[i, j] - want) == best


@pytest.mark.parametrize("fmt,ties", [(api.KV_MXFP4, {0.25: 0.0, 0.75: 1.0, 1.25: 1.0, 1.75: 2.0, 2.5: 2.0, 3.5: 4.0, 5.0: 4.0}),
                                      (api.KV_MXFP8, {2.0 ** -10: 0.0, 3 * 2.0 ** -10: 2.0 ** -8, 17.0: 16.0, 19.0: 20.0, 248.0: 256.0})])
def test_ties_go_to_the_even_fraction(fmt, ties):
    x = np.zeros((1, 32))
    x[0, 0] = 6.0 if fmt == api.KV_MXFP4 else 448.0          # scale 1
    for i, t in enumerate(ties):
        x[0, 1 + 2 * i], x[0, 2 + 2 * i] = t, -t
    v = R.values(*R.quantise(x, fmt), fmt)
    for i, want in enumerate(ties.values()):
        assert v[0, 1 + 2 * i] == want and v[0, 2 + 2 * i] == -want


@pytest.mark.parametrize("fmt", FORMATS)
def test_blocks_that_are_not_finite_read_as_nan(fmt):
    x = np.ones((3, 64))
    x[0, 5], x[1, 40] = np.nan, -np.inf
    codes, scale = R.quantise(x, fmt)
    assert scale[0].tolist() == [255, scale[2, 1]] and scale[1].tolist() == [scale[2, 0], 255]
    v = R.values(codes, scale, fmt)
    assert np.isnan(v[0, :32]).all() and np.isnan(v[1, 32:]).all() and (v[0, 32:] == 1).all() and (v[2] == 1).all()


@pytest.mark.parametrize("fmt", FORMATS)
def test_values_are_bf16_numbers(fmt):
    import torch
    codes = (np.arange(256 if fmt == api.KV_MXFP8 else 32) % (256 if fmt == api.KV_MXFP8 else 16)).reshape(1, -1)
    for b in (63, 100, 127, 142):
        v = R.values(codes, np.full((1, codes.shape[1] // 32), b, dtype=np.uint8), fmt)
        t = torch.from_numpy(v)
        assert torch.equal(torch.nan_to_num(t.to(torch.bfloat16).double(), nan=1e9), torch.nan_to_num(t, nan=1e9))
