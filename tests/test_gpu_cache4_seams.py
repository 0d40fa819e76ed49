"""Stores of the 4-bit cache whose rows do not begin where its 8-token blocks do: the eights are cut (row-major) or
regrouped (transposed) at the workgroups' seams, of STEP and of ALL rows."""

import numpy as np
import pytest
import torch

from gpu_util import archer, dev_i32, say
from oracle import cache4 as oc
from test_gpu_cache4 import F16, F32, dev, new_cache, random_bytes
from test_gpu_cache4_strides import _finite

pytestmark = pytest.mark.gpu

ALL = {64: 256, 128: 128}        # rows that a workgroup's threads own
FORMS = ["rows", "transposed", "transposed odd"]


def _values(V, form, dtype):
    H, n, hd = V.shape
    if form == "rows":
        return dev(V, dtype)
    ld, off = ((n + 7) // 8 * 8, 0) if form == "transposed" else (n + 5, 3)
    t = torch.full((H, hd, ld), float("nan"), dtype=dtype, device="cuda")
    t[:, :, off:off + n] = dev(V.transpose(0, 2, 1), dtype)
    return t[:, :, off:off + n].transpose(1, 2)


def _check(rng, slots, n_pages, page, hd, form, dtype, H=2):
    n = len(slots)
    K, V = _finite(rng, H, n, hd, dtype), _finite(rng, H, n, hd, dtype)
    data = random_bytes(rng, n_pages, H, page, hd)
    c = new_cache(data, page, hd)
    archer().cache4_write(c, dev(K, dtype), _values(V, form, dtype), dev_i32(slots))
    np.testing.assert_array_equal(c.data.cpu().numpy(), oc.write(data, page, hd, K, V, slots))


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("form", FORMS)
@pytest.mark.parametrize("n", [300, 600])
def test_shifted_runs(dtype, hd, form, n):
    """One run over several workgroups, from each position of an 8-token block."""
    say(f"shifted runs {dtype} hd={hd} {form} n={n}")
    rng = np.random.default_rng(n + hd)
    for first in range(1, 8):
        _check(rng, np.arange(n) + first + 32, -(-n // 32) + 3, 32, hd, form, dtype)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_run_ends_at_a_workgroups_seam(dtype, hd, form):
    say(f"seam {dtype} hd={hd} {form}")
    rng = np.random.default_rng(hd)
    for n in list(range(ALL[hd] - 9, ALL[hd] + 2)) + [2 * ALL[hd] - 3, 2 * ALL[hd] + 1]:
        for lead in (1, 4, 7):
            _check(rng, np.arange(n) + lead, -(-n // 64) + 2, 64, hd, form, dtype, H=1)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("hd", [64, 128])
@pytest.mark.parametrize("form", FORMS)
def test_ragged_prompts_with_rows_left_out(dtype, hd, form):
    """Prompts of odd lengths that begin inside a page, over pages in random order, rows without a slot around the
    workgroups' seams."""
    say(f"ragged {dtype} hd={hd} {form}")
    rng = np.random.default_rng(7 + hd)
    page = 32
    for turn in range(3):
        lens, starts = [37, 131, 1, 250, 8, 119, 77], [3, 7, 31, 13, 1, 6, 0]
        need = [-(-(n + s) // page) for n, s in zip(lens, starts)]
        order = rng.permutation(sum(need) + 2)
        slots, at = [], 0
        for n, s, k in zip(lens, starts, need):
            p = np.arange(s, s + n)
            slots.append(order[at + p // page] * page + p % page)
            at += k
        slots = np.concatenate(slots)
        out = [x for r in range(0, len(slots), 8) for x in (r - turn, r) if rng.random() < 0.15]
        for step in (ALL[hd], ALL[hd] - 8):
            out += [r + d for r in range(step, len(slots), step) for d in ([0], [-1, 0, 1], range(-9, 9))[turn]]
        slots[[r for r in out if 0 <= r < len(slots)]] = -1
        _check(rng, slots, len(order), page, hd, form, dtype)
