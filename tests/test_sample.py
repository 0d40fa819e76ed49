"""Sampling without a GPU: the oracle against first principles, and the library's refusals."""

import itertools

import numpy as np
import pytest
import torch

from oracle import sample as osm


def _brute(l, u, t, k, p, m):
    """The definition with sets, of a few tokens of distinct weights."""
    order = sorted(range(len(l)), key=lambda i: (-l[i], i))
    w = {i: np.exp((l[i] - max(l)) / t) for i in order}
    s1 = order[:k] if k > 0 else order
    if p < 1:
        n = next(n for n in range(1, len(s1) + 1) if sum(w[i] for i in s1[:n]) >= p * sum(w[i] for i in s1))
        s1 = s1[:n]
    keep = {i for i in s1 if w[i] >= m} | {order[0]}
    total, run = sum(w[i] for i in keep), 0.0
    for i in sorted(keep):
        run += w[i]
        if run > u * total:
            return i, np.log(w[i] / total)


@pytest.mark.parametrize("t,k,p,m", list(itertools.product([0.5, 1.0, 3.0], [0, 1, 3, 9], [0.3, 0.8, 1.0], [0.0, 0.05, 0.4])))
def test_oracle_is_the_definition(t, k, p, m):
    rng = np.random.default_rng(int(t * 10) + k)
    for _ in range(20):
        l, u = rng.standard_normal(7) * 2, rng.random()
        got, want = osm.sample(l, u, temperature=t, top_k=k, top_p=p, min_p=m), _brute(l, u, t, k, p, m)
        assert got[0] == want[0] and abs(got[1] - want[1]) < 1e-12


def test_oracle_edges():
    inf = np.inf
    assert osm.sample([1, 5, 5, 2], 0.9, temperature=0.0) == (1, 0.0)
    assert osm.sample([1, 5, 5, 2], 0.9, temperature=0.0, exclude=1) == (2, 0.0)
    assert osm.sample([-inf, -inf], 0.5) == (-1, -inf) and osm.sample([3.0], 0.5, exclude=0) == (-1, -inf)
    assert osm.sample([1, np.nan], 0.5)[0] == -1 and np.isnan(osm.sample([1, np.nan], 0.5)[1])
    assert osm.sample([1, np.nan], 0.5, exclude=1) == (0, 0.0)
    assert osm.sample([9, inf, 3, inf], 0.6) == (3, np.log(0.5)) and osm.sample([9, inf, 3, inf], 0.4) == (1, np.log(0.5))
    assert osm.sample([0, 0, 0, 0], 0.5) == (2, np.log(0.25)) and osm.sample([0, 0, 0, 0], 0.5, top_k=2) == (1, np.log(0.5))
    assert osm.sample([0, 0, 0, 0], 0.99, top_p=0.0) == (0, 0.0) and osm.sample([0, 1, 1, 0], 0.99, min_p=2.0) == (1, 0.0)
    assert osm.sample([0, -inf, 0], 1.0) == (2, np.log(0.5))


def test_frequencies():
    """Over an even grid of u each token comes as often as its weight says."""
    l, n = np.array([0.3, -1, 2, 0.5, -4]), 20000
    w = np.exp(l / 0.7)
    got = np.bincount([osm.sample(l, (i + 0.5) / n, temperature=0.7)[0] for i in range(n)], minlength=5) / n
    assert np.abs(got - w / w.sum()).max() <= 1 / n


# -- the library's refusals: every one before a launch ------------------------------------------------
X = 1 << 20


@pytest.mark.parametrize("change,code", [
    (dict(dtype=3), "E_ARG"), (dict(dtype=-1), "E_ARG"), (dict(rows=-1), "E_SHAPE"), (dict(vocab=0), "E_SHAPE"),
    (dict(vocab=524289), "E_SHAPE"), (dict(exclude=-2), "E_ARG"), (dict(exclude=100), "E_ARG"), (dict(logits=None), "E_ARG"),
    (dict(u=None), "E_ARG"), (dict(token=None), "E_ARG"), (dict(logits=X + 2), "E_ARG"), (dict(dtype=0, logits=X + 1), "E_ARG"),
    (dict(ws=None), "E_WORKSPACE"), (dict(ws=X + 128), "E_WORKSPACE"), (dict(ws_bytes=1000), "E_WORKSPACE"),
])
def test_arguments(change, code):
    from paper_2608_08086_amd import archer as a
    v = dict(dtype=a.FP32, rows=2, vocab=100, logits=X, stride=100, exclude=-1, u=X, t=None, k=None, p=None, m=None, token=X, logp=None, ws=X,
             ws_bytes=a.lib.archer_op_sample_ws_bytes(a.FP32, 2, 100))
    v.update(change)
    assert a.lib.archer_op_sample(*v.values(), None) == getattr(a, code)
    assert a.lib.archer_last_error()


def test_no_rows():
    from paper_2608_08086_amd import archer as a
    assert a.lib.archer_op_sample(a.FP32, 0, 100, None, 100, -1, *[None] * 8, 0, None) == a.OK


def test_workspace():
    from paper_2608_08086_amd import archer as a
    ws = a.lib.archer_op_sample_ws_bytes
    assert ws(a.FP32, 1, 1) > 0 and ws(a.FP32, 1, 1) % 256 == 0
    assert ws(3, 1, 1) == ws(a.FP32, 0, 1) == ws(a.FP32, 1, 0) == ws(a.FP32, 1, 524289) == 0
    assert ws(a.BF16, 2**31 - 1, 152064) == ws(a.BF16, 1024, 152064) < 2**29      # many rows: in groups


def test_binding_refusals(monkeypatch):
    from paper_2608_08086_amd import archer as a
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    monkeypatch.setattr(a.lib, "archer_op_sample", lambda *x: pytest.fail("the library was called"))
    l, u, i = torch.zeros(2, 10), torch.zeros(2), torch.zeros(2, dtype=torch.int32)
    for f in (lambda: a.op_sample(l[0], u), lambda: a.op_sample(l.double(), u.double()), lambda: a.op_sample(l.T, torch.zeros(10)),
              lambda: a.op_sample(l, torch.zeros(3)), lambda: a.op_sample(l, u.double()), lambda: a.op_sample(l, u, temperature=i),
              lambda: a.op_sample(l, u, top_k=u), lambda: a.op_sample(l, u, top_p=torch.zeros(1)), lambda: a.op_sample(l, u, min_p=u.half()),
              lambda: a.op_sample(l, u, exclude=2**32), lambda: a.op_sample(l, torch.zeros(4)[::2])):
        with pytest.raises(a.ArcherError):
            f()
