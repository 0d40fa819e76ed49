"""Attention over the 4-bit cache with infinite scores: a key of score -infinity takes nothing, and a row whose keys
all have it is NaN, as its softmax is, in every kernel; a row without keys is zeros."""

import numpy as np
import pytest

from gpu_util import host, say
from oracle import cache4 as oc
from test_gpu_cache4 import F16, F32, SOME, Case

pytestmark = pytest.mark.gpu

WIDE_LENS = [300, 41, 0, 90, 64, 128, 7, 200]
# dtype, lens, G, hq, hkv, hd, fresh: one and two blocks, cut along the keys, four blocks, the row kernel, fp32
CALLS = [(F16, [100, 0, 41], 1, 4, 2, 128, False), (F16, [100, 0, 41], 1, 4, 2, 64, True),
         (F16, [100, 0, 41], 80, 4, 2, 128, True), (F32, [100, 0, 41], 3, 4, 2, 128, True),
         (F16, [5000], 1, 8, 2, 128, False), (F16, [3300, 0], 16, 32, 8, 64, True), (F16, [4100], 100, 2, 2, 128, True),
         (F16, WIDE_LENS, 512, 16, 8, 64, True), (F16, WIDE_LENS, 512, 8, 4, 128, True),
         (F16, WIDE_LENS, 512, 8, 4, 128, False)]
D = 9       # the dimension that is infinite


@pytest.mark.parametrize("dtype,lens,G,hq,hkv,hd,fresh", CALLS)
def test_rows_of_infinite_scores(dtype, lens, G, hq, hkv, hd, fresh):
    """Query rows with -infinity where every key of theirs has 1, beside finite rows of the same call."""
    say(f"{dtype} lens={lens} G={G} hq={hq} hkv={hkv} hd={hd} fresh={fresh}")
    c = Case(dtype, lens, G, hq, hkv, hd, 64, fresh, seed=80)
    for b, n in enumerate(lens):
        slots = [c.table[b, p // 64] * 64 + p % 64 for p in range(n)]
        k = c.K[b].copy()
        k[..., D] = 1.0
        c.data = oc.write(c.data, 64, hd, k, c.V[b], slots)
        c.K[b], c.V[b] = oc.read(c.data, 64, hd, slots)
        assert (c.K[b][..., D] > 0).all()
    if fresh:
        c.K2[..., D] = 1.0
    plain = host(c.run())
    bad = np.zeros((len(lens), G, hq), bool)
    bad[:, G // 2, 1] = bad[0, 0, hq - 1] = bad[-1, G - 1, 0] = True
    q = c.Q.reshape(hq, len(lens), G, hd)
    q.transpose(1, 2, 0, 3)[bad, D] = -np.inf
    got = host(c.run()).reshape(len(lens), G, hq, hd)
    none = np.array([n == 0 and not fresh for n in lens])[:, None, None] & np.ones_like(bad)
    assert (got[none] == 0).all()
    assert np.isnan(got[bad & ~none]).all()
    np.testing.assert_array_equal(got[~bad], plain.reshape(got.shape)[~bad])


@pytest.mark.parametrize("dtype,lens,G,hq,hkv,hd,fresh", [x for x in CALLS if x[6]])
@pytest.mark.parametrize("every", [False, True])
def test_keys_of_infinite_scores(dtype, lens, G, hq, hkv, hd, fresh, every):
    """Fresh keys, some or all of a sequence, that no row may attend to: they are as if they were not there, and
    where there are no others the rows are NaN."""
    say(f"{dtype} lens={lens} G={G} hq={hq} hkv={hkv} hd={hd} every={every}")
    c = Case(dtype, lens, G, hq, hkv, hd, 64, fresh, seed=81)
    c.Q[..., D] = np.abs(c.Q[..., D]) + np.float16(0.1)
    hide = np.ones(G, bool) if every else np.arange(G) % 3 > 0
    for b in range(len(lens)):
        c.K2[:, b * c.stride + np.flatnonzero(hide), D] = -np.inf
    O = host(c.run()).reshape(len(lens), G, hq, hd)
    worst = 0.0
    pick = SOME[SOME < G]
    for b, n in enumerate(lens):
        for h in range(hq):
            k, v = c.keys(b, h // (hq // hkv))
            keep = np.r_[np.ones(n, bool), ~hide]
            k, v = k[keep], v[keep]
            if len(k) == 0:
                assert np.isnan(O[b, :, h]).all()
                continue
            ref, A, qk, smax = oc.attention(c.Q[h, b * G + pick].astype(np.float64), k, v)
            tol = oc.attention_bound(ref, A, qk, smax, n + G, hd, np.abs(v).max(), dtype == F16)
            err = np.abs(O[b, pick, h] - ref)
            assert (err <= tol).all(), (b, h)
            worst = max(worst, float((err / tol).max()))
    say(f"  worst error / bound {worst:.3f}")
