"""Stores of the 4-bit cache from strides that the other tests do not have: one row of any stride, and negative ones."""

import numpy as np
import pytest
import torch

from gpu_util import archer, dev_i32, say
from oracle import cache4 as oc
from test_gpu_cache4 import F16, F32, dev, new_cache, random_bytes

pytestmark = pytest.mark.gpu


def _finite(rng, H, n, hd, dtype):
    x = rng.standard_normal((H, n, hd)) * 2.0 ** rng.integers(-6, 6, (H, n, 1))
    return x.astype(np.float16 if dtype == F16 else np.float32)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("step", [1, 2, 3, -1])
def test_one_row_of_any_stride(dtype, hd, step):
    """A single row's values need no unit stride: along the rows there is nothing to step over."""
    say(f"one row {dtype} hd={hd} step={step}")
    a, H, page = archer(), 3, 32
    rng = np.random.default_rng(hd + step)
    K, V = _finite(rng, H, 1, hd, dtype), _finite(rng, H, 1, hd, dtype)
    data = random_bytes(rng, 2, H, page, hd)
    c = new_cache(data, page, hd)
    s = abs(step)
    src = torch.full((H, hd * s + 1), float("nan"), dtype=dtype, device="cuda")
    src[:, :hd * s:s] = dev(V[:, 0] if step > 0 else V[:, 0, ::-1], dtype)
    slots = dev_i32([37])
    if step > 0:
        v = src.as_strided((H, 1, hd), (hd * s + 1, 5, s))
        a.cache4_write(c, dev(K, dtype), v, slots)
    else:      # torch has no negative strides
        esz = src.element_size()
        k = dev(K, dtype)
        a._check(a.lib.archer_cache4_write(a.BF16 if dtype == F16 else a.FP32, c.ref, 1, k.data_ptr(), hd, hd,
                                           src.data_ptr() + (hd - 1) * esz, hd * s + 1, 5, -1, slots.data_ptr(),
                                           a._raw_stream(0)))
    np.testing.assert_array_equal(c.data.cpu().numpy(), oc.write(data, page, hd, K, V, [37]))


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("transposed", [False, True])
@pytest.mark.parametrize("n", [5, 300])
def test_negative_strides(dtype, hd, transposed, n):
    """Heads, rows and (transposed) dimensions from the last to the first: strides of any sign."""
    say(f"negative strides {dtype} hd={hd} transposed={transposed} n={n}")
    a, H, page = archer(), 3, 64
    rng = np.random.default_rng(hd + n)
    K, V = _finite(rng, H, n, hd, dtype), _finite(rng, H, n, hd, dtype)
    n_pages = -(-n // page) + 2
    data = random_bytes(rng, n_pages, H, page, hd)
    slots = np.arange(n) + 3
    k = dev(K[::-1, ::-1], dtype)                       # [heads][rows][dims], both from the last one
    # values: heads and rows from the last, or [heads][dims][rows], heads and dimensions from the last
    v = dev(V[::-1, :, ::-1].transpose(0, 2, 1) if transposed else V[::-1, ::-1], dtype)
    c, s = new_cache(data, page, hd), dev_i32(slots)
    esz, last = k.element_size(), (H * n - 1) * hd
    at, vr, vd = ((H * hd - 1) * n, 1, -n) if transposed else (last, -hd, 1)
    a._check(a.lib.archer_cache4_write(a.BF16 if dtype == F16 else a.FP32, c.ref, n, k.data_ptr() + last * esz, -n * hd,
                                       -hd, v.data_ptr() + at * esz, -n * hd, vr, vd, s.data_ptr(), a._raw_stream(0)))
    np.testing.assert_array_equal(c.data.cpu().numpy(), oc.write(data, page, hd, K, V, slots))
