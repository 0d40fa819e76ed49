"""GPU parity of sampling where a rule meets the ends of a type or of its own sums: rows of the lowest finite value,
temperatures at which every finite logit weighs the same, filters that cut nothing, and a top_p whose border lies
between two partial sums.  Tolerances as in ``test_gpu_sample``."""

import math

import numpy as np
import pytest
import torch

from gpu_util import say
from test_gpu_sample import T, check, run

pytestmark = pytest.mark.gpu

LOWEST = {"fp32": torch.finfo(torch.float32).min, "bf16": torch.finfo(torch.bfloat16).min, "fp16": torch.finfo(torch.float16).min}


# -- the lowest finite value ------------------------------------------------------------------------
@pytest.mark.parametrize("vocab", [3, 257, 1025, 4096, 30001])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("kw", [{}, dict(top_k=10**6), dict(top_k=29999), dict(min_p=0.5), dict(top_k=1300), dict(top_p=0.37),
                                dict(top_k=2901, top_p=0.41)])
def test_rows_of_the_lowest_value(vocab, dtype, kw):
    """Every token is alike, whatever value they share: only -infinity has no weight."""
    say(f"lowest {vocab} {dtype} {kw}")
    rng = np.random.default_rng(vocab)
    n = 12
    z = torch.full((n, vocab), LOWEST[dtype], dtype=T[dtype], device="cuda")
    if vocab > 256:
        z[1::3, 5:vocab // 2] = -torch.inf
        z[2::3, rng.integers(0, vocab, vocab // 3)] = -torch.inf
    # (a row is left out where p or u times its tokens is a whole number of them: rarely, and not 0.41 * 2901)
    for exclude in (-1, vocab // 3):
        check(z, rng.random(n), {k: [v] * n for k, v in kw.items()}, exclude=exclude, most_unsafe=0.2)


@pytest.mark.parametrize("kw", [{}, dict(top_k=10**6), dict(min_p=1e-3), dict(top_p=0.9)])
def test_lowest_values_beside_others(kw):
    """A mask of the lowest value: without weight beside others, unless the temperature is as large as they are apart."""
    rng = np.random.default_rng(1)
    n = 6
    z = torch.from_numpy(rng.standard_normal((n, 9000)).astype(np.float32)).cuda()
    z[:, 100:4300] = LOWEST["fp32"]
    z[3:, :100] = LOWEST["fp32"]
    z[:, 8999] = -torch.inf
    kw = dict({k: [v] * n for k, v in kw.items()}, temperature=[1.0, 1e38, 3e38, 0.7, 2e38, np.inf])
    check(z, rng.random(n), kw, exclude=17, most_unsafe=0.2)


# -- temperatures as large as the type's values -----------------------------------------------------
@pytest.mark.parametrize("t", [1e36, 1.1e37, 1e38, 3e38, np.inf])
@pytest.mark.parametrize("k", [1501, 2000, 10**6])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_masked_tokens_at_large_temperatures(t, k, dtype):
    """More finite tokens than a list of all of them takes and a top_k beyond their number: nothing is cut, and masked
    tokens weigh nothing, the excluded one and those past the row's end neither."""
    say(f"temperature {t} top_k {k} {dtype}")
    rng = np.random.default_rng(k)
    n = 16
    z = torch.from_numpy(rng.standard_normal((n, 3001)).astype(np.float32)).to(T[dtype]).cuda()
    z[:, 1:3000:2] = -torch.inf                    # 1501 finite ones, with the last
    z[8:, 1024:2048] = -torch.inf                  # a piece without any
    for exclude in (-1, 40):
        check(z, rng.random(n), dict(temperature=[t] * n, top_k=[k] * n), exclude=exclude, most_unsafe=0.2)


@pytest.mark.parametrize("kw", [dict(top_k=1200), dict(top_p=0.37), dict(min_p=0.5), dict(top_k=1401, top_p=0.41)])
def test_cuts_among_masked_tokens_at_large_temperatures(kw):
    """A cut within the one value that they weigh, beside masked tokens."""
    rng = np.random.default_rng(3)
    n = 8
    z = torch.from_numpy(rng.standard_normal((n, 30000)).astype(np.float32)).cuda()
    z[:, ::3] = -torch.inf
    z[4:] = -torch.inf
    z[4:, 7::13] = 1.5
    check(z, rng.random(n), dict({k: [v] * n for k, v in kw.items()}, temperature=[np.inf, 1e38] * 4), exclude=1, most_unsafe=0.3)


# -- top_k and top_p together where one value is there too often ------------------------------------
@pytest.mark.parametrize("k,p,n", [(100, 0.505, 51), (101, 0.5, 51), (100, 0.995, 100), (7, 0.01, 1)])
def test_top_p_of_top_k_in_a_value_that_many_tokens_share(k, p, n):
    """p of the k tokens' weight lies half a token from a border: n tokens are left, the first ones."""
    say(f"shared k={k} p={p}")
    rng = np.random.default_rng(5)
    rows = 24
    z = torch.from_numpy(np.where(rng.random((rows, 60000)) < 0.5, 0.0, -1.0)).float().cuda()
    u = (np.arange(rows) + 0.31) / rows
    tok = check(z, u, dict(top_k=[k] * rows, top_p=[p] * rows, temperature=[1 / math.log(4.0)] * rows), most_unsafe=0.0)
    for r in range(rows):
        first = np.flatnonzero(z[r].cpu().numpy() == 0)
        assert tok[r] == first[int(u[r] * n)]


# -- a border between two partial sums --------------------------------------------------------------
def _row_at_a_border(rng, over):
    """A token of weight 1, and others of 2^15 - 1 + `over` together, each of about e^(-1/16) and by themselves."""
    total = 2.0**15 - 1 + over
    l = rng.uniform(-0.075, -0.069, 35300).astype(np.float32)
    w = np.cumsum(np.exp(l.astype(np.float64)))
    l = l[:int(np.searchsorted(w, total - 0.93)) + 1]
    # what lacks is shared out among 3000 of them, and one takes what is left: its logits are 2^-27 apart
    share = l[:3000].astype(np.float64)
    l[:3000] = share + np.log1p((total - 0.93 - w[len(l) - 1]) / np.exp(share).sum())
    last = total - math.fsum(np.exp(l.astype(np.float64)))
    l = np.append(l, np.float32(math.log(last)))
    assert abs(math.fsum(np.exp(l.astype(np.float64))) - total) < over / 2
    return np.concatenate([[np.float32(0)], l])


def test_top_p_at_a_border_between_two_partial_sums():
    """A first token of weight 1, the others with 2^15 - 1 and 2^-24 more: top_p = 2^-15 asks for the first one and a little
    more than none of the next.  The sum up to the second one and that without it lie 2^-38 apart in 64 bits, which may
    be more than the border is from either: one token is kept or two, whichever rounding, never all of them."""
    rng = np.random.default_rng(11)
    rows = [_row_at_a_border(rng, 2.0**-24) for _ in range(32)]
    V = max(len(r) for r in rows)
    z = np.full((len(rows), V), -np.inf, np.float32)
    for i, r in enumerate(rows):
        z[i, :len(r)] = r
    tok, logp = (x.cpu().numpy() for x in run(torch.from_numpy(z).cuda(), [0.75] * len(rows), dict(top_p=[2.0**-15] * len(rows))))
    for i, row in enumerate(z):
        order = np.argsort(-row, kind="stable")
        assert tok[i] in order[:2], (i, tok[i], order[:2])
        assert logp[i] >= math.log(0.25)
