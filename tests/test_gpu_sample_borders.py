"""GPU parity of sampling where a rule meets the ends of a type: rows of the lowest finite value, temperatures at which
every finite logit weighs the same, filters that cut nothing.  Tolerances as in ``test_gpu_sample``."""

import numpy as np
import pytest
import torch

from gpu_util import say
from test_gpu_sample import T, check

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
