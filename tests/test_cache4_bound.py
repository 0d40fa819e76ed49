"""The error bound of the 4-bit cache's attention rejects what it is meant to (no GPU)."""

import numpy as np
import pytest

from oracle import cache4 as oc


def _case(q_scale, hd=128, n=300):
    rng = np.random.default_rng(3)
    q = (rng.standard_normal((4, hd)) * q_scale).astype(np.float16).astype(np.float64)
    k, v = oc.stored(rng.standard_normal((n, hd))), oc.stored(rng.standard_normal((n, hd)))
    ref, A, _, _ = oc.attention(q, k, v)
    qk, block = oc.score_sums(q, k)
    return q, k, v, ref, A, qk, block, np.abs(q @ k.T).max(-1, keepdims=True) / np.sqrt(hd)


def test_score_sums():
    q, k, _, _, _, qk, block, smax = _case(2.0, n=9)
    s = np.array([[sum(abs(a * b) for a, b in zip(x, y)) for y in k] for x in q]).max(-1) / np.sqrt(128)
    np.testing.assert_allclose(qk[:, 0], s, rtol=1e-12)
    assert (block >= qk).all() and (qk >= smax).all()
    assert float(block.max()) == pytest.approx(oc.attention(q, k, k)[2], rel=1e-12)


@pytest.mark.parametrize("q_scale", [2.0, 30.0])
@pytest.mark.parametrize("rows_kernel", [False, True])
def test_a_score_scale_off_by_one_percent_is_outside(q_scale, rows_kernel):
    q, k, v, ref, A, qk, block, smax = _case(q_scale)
    tol = oc.attention_bound(ref, A, qk, smax, len(k), 128, np.abs(v).max(), True, block if rows_kernel else 0.0)
    assert (np.abs(oc.attention(1.01 * q, k, v)[0] - ref) > tol).any()
    # the output's own rounding and fp16 probabilities are inside
    p = np.exp(q @ k.T / np.sqrt(128))
    p = (p / p.max(-1, keepdims=True)).astype(np.float16).astype(np.float64)
    got = p @ v / p.sum(-1, keepdims=True)
    got += np.sign(got - ref) * np.abs(got) * 2.0**-9
    assert (np.abs(got - ref) <= tol).all()


def _e2m3(x, scale):
    """The nearest e2m3 values of x / scale, times the scale: steps of 1/8 below 2, 1/4 below 4, 1/2 up to 7.5."""
    y = np.abs(x) / scale
    step = np.where(y < 2, 0.125, np.where(y < 4, 0.25, 0.5))
    return np.copysign(np.minimum(np.round(y / step) * step, 7.5), x) * scale


@pytest.mark.parametrize("terms", [3, 4])
def test_terms_of_a_query(terms):
    """Four e2m3 terms leave 2^-17 of the first one's scale, three 2^-12; magnitudes add up as the bound says."""
    rng = np.random.default_rng(5)
    x = rng.standard_normal((4000, 32)) * 2.0 ** rng.integers(-12, 1, (4000, 32))
    x = np.concatenate([x, np.linspace(-7.5, 7.5, 32 * 4001).reshape(-1, 32)])
    top = np.abs(x).max(-1, keepdims=True)
    s1 = 2.0 ** np.ceil(np.log2(top / 7.5))
    assert (top <= 7.5 * s1).all() and (top > 3.75 * s1 * (1 - 1e-12)).all()
    r, total = x.copy(), np.zeros_like(x)
    for below in (0, 4, 9, 14)[:terms]:
        t = _e2m3(r, s1 * 2.0**-below)
        r -= t
        total += np.abs(t)
    assert (np.abs(r) <= 2.0 ** (-17 if terms == 4 else -12) * s1).all()
    assert (total <= 3.5 * np.abs(x) + 1e-30).all() and (total <= np.abs(x) + 0.52 * s1).all()
    assert terms == 4 or (np.abs(r) > 2.0**-14 * s1).any()
