"""Attention over the 4-bit cache where one sequence is far longer than the others: it is cut along its keys, however
many sequences there are."""

import numpy as np
import pytest

from gpu_util import archer, say
from test_gpu_cache4 import F16, F32, SOME, Case
from test_gpu_cache4_precision import check

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,B,G,hq,hkv,hd,fresh", [
    (F16, 40, 1, 28, 4, 64, False),       # more chunks than sequences in any case
    (F16, 200, 1, 8, 8, 128, True),       # fewer: one to a sequence on average
    (F16, 256, 3, 2, 2, 128, False),
    (F16, 60, 40, 8, 4, 64, True),        # two blocks of columns
    (F32, 130, 2, 4, 4, 64, True),
])
def test_one_long_sequence(dtype, B, G, hq, hkv, hd, fresh):
    lens = [(53 * b) % 131 for b in range(B)]
    lens[B // 3] = 33001
    say(f"{dtype} B={B} G={G} hq={hq} hkv={hkv} hd={hd} fresh={fresh}")
    a = archer()
    n = a.lib.archer_op_attention_cache4_ws_bytes(0 if dtype == F16 else 1, B, G, hq, hkv, hd, max(lens), int(fresh))
    assert n > 0, "a sequence of 33001 keys is cut"
    c = Case(dtype, lens, G, hq, hkv, hd, 256, fresh, seed=100 + B)
    say(f"  worst error / bound {check(c, c.run(), rows_of=None if G < 10 else SOME):.3f}")
