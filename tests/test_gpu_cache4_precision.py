"""Attention over the 4-bit cache within the bounds of the kernel that runs: the column kernel rounds no query,
the row kernel to 2^-18.9 of the largest of 32 elements (``oracle/cache4.py``)."""

import numpy as np
import pytest
import torch

from gpu_util import host, say
from oracle import cache4 as oc
from test_gpu_cache4 import F16, F32, SOME, Case

pytestmark = pytest.mark.gpu


def row_kernel(c):
    """Whether a call takes the row kernel: as many columns as the library's rule asks for."""
    ncol = c.G * c.hq // c.hkv
    full = (ncol + 31) // 32 >= 4 * ((ncol + 255) // 256)
    return c.dtype == F16 and c.hd == 128 and ncol > 16 and full and ncol * len(c.lens) * c.hkv >= 1 << 15


def check(c, O, rows_of=None):
    """As Case.check, every row against the bound of its own scores."""
    O = host(O).reshape(len(c.lens), c.G, c.hq, c.hd)
    worst = 0.0
    for b in range(len(c.lens)):
        pick = np.arange(c.rows[b]) if rows_of is None else rows_of[rows_of < c.rows[b]]
        for h in range(c.hq):
            k, v = c.keys(b, h // (c.hq // c.hkv))
            if len(k) == 0 or len(pick) == 0:
                continue
            q = c.Q[h, b * c.G + pick].astype(np.float64)
            ref, A = oc.attention(q, k, v)[:2]
            smax = np.abs(q @ k.T).max(-1, keepdims=True) / np.sqrt(c.hd)
            qk, block = oc.score_sums(q, k)
            tol = oc.attention_bound(ref, A, qk, smax, len(k), c.hd, np.abs(v).max(), c.dtype == F16,
                                     block if row_kernel(c) else 0.0)
            err = np.abs(O[b, pick, h] - ref)
            assert (err <= tol).all(), (b, h, float((err / tol).max()))
            worst = max(worst, float((err / tol).max()))
    return worst


WIDE_LENS = [300, 41, 0, 90, 64, 128, 7, 200]


@pytest.mark.parametrize("dtype,lens,G,hq,hkv,hd,fresh", [
    (F16, [300, 41], 1, 4, 2, 128, True),
    (F16, [300, 41], 1, 4, 2, 64, False),
    (F16, [300, 41], 80, 4, 2, 128, True),
    (F16, [300, 41], 80, 4, 2, 64, True),
    (F32, [300, 41], 3, 4, 2, 128, True),
    (F32, [300, 41], 3, 4, 2, 64, True),
    (F16, [3001, 5, 0, 1500], 1, 7, 1, 128, True),        # cut along the keys
    (F16, [5000], 1, 8, 2, 64, False),
    (F16, WIDE_LENS, 512, 8, 4, 128, True),
    (F16, WIDE_LENS, 512, 16, 8, 64, True),
])
@pytest.mark.parametrize("q_scale", [0.1, 2.0, 30.0])
def test_bound_of_the_kernel_that_runs(dtype, lens, G, hq, hkv, hd, fresh, q_scale):
    say(f"attention {dtype} lens={lens} G={G} hq={hq} hkv={hkv} hd={hd} q_scale={q_scale}")
    c = Case(dtype, lens, G, hq, hkv, hd, 64, fresh, seed=70, q_scale=q_scale)
    say(f"  worst error / bound {check(c, c.run(), rows_of=SOME):.3f}")


@pytest.mark.parametrize("lens,G,hq,hkv", [([300, 41], 1, 4, 2), ([300, 41], 80, 4, 2), (WIDE_LENS, 512, 8, 4)])
def test_queries_with_one_large_element_per_block(lens, G, hq, hkv):
    """One element of each 32 a thousand times the others, which all point one way along keys that have nothing there:
    what a query rounded relative to its largest element is off by adds up over the dimensions."""
    hd, page = 128, 64
    c = Case(F16, lens, G, hq, hkv, hd, page, False, seed=71)
    rng = np.random.default_rng(72)
    # of the fp16 numbers next to one, that which times the softmax's factor is farthest from the multiples of 2^-12
    # of the terms' scale (32 here: the largest element times the factor is 127.5)
    near = np.arange(1.0, 1.25, 2.0**-10)
    off = near * 1.4426950408889634 / np.sqrt(hd) / 2.0**-7 % 1.0
    small = near[np.argmin(np.abs(off - 0.5))]
    large = np.arange(hd) % 32 == 5
    q = np.where(large, 1000.0, small) * rng.choice([-1.0, 1.0], (hq, len(lens) * G, 1))
    c.Q = q.astype(np.float16)
    for b, n in enumerate(lens):
        slots = [c.table[b, p // page] * page + p % page for p in range(n)]
        k = np.where(large, 0.0, rng.choice([-1.0, -0.5, 0.5, 1.0], (hkv, n, 1)))
        c.data = oc.write(c.data, page, hd, k, c.V[b], slots)
        c.K[b], c.V[b] = oc.read(c.data, page, hd, slots)
        np.testing.assert_array_equal(c.K[b], k)
    say(f"G={G} hq={hq}: worst error / bound {check(c, c.run(), rows_of=SOME):.3f}")
