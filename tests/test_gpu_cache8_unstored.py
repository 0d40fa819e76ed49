"""Attention over an 8-bit cache where blocks without a token of the sequence hold anything, their scale bytes too.

A block of 32 tokens that no sequence has a token of was never stored: its scale byte may be any, and 255 stands for
an infinite scale.  The keys and values there have no weight, so nothing of them may reach a result.  Bounds as in
``test_gpu_cache8``, which this does not change: the same tokens count."""

import numpy as np
import pytest

from gpu_util import say
from oracle import cache4 as oc
from test_gpu_cache8 import F16, F32, SOME, Case

pytestmark = pytest.mark.gpu

# last tiles of 64 keys whose second half has no key, and lengths around; `page` 32 or 64 (a block or two)
LENS = [32, 1, 0, 31, 64, 65, 96, 300]
# every kernel: one and two blocks of columns, 64 dimensions, fp32, the one for many columns, split sequences
KINDS = [(F16, LENS, 1, 4, 2, 128), (F16, LENS, 20, 4, 2, 128), (F16, LENS, 80, 4, 2, 64), (F32, LENS, 3, 4, 2, 128), (F32, LENS, 3, 2, 2, 64),
         (F16, LENS, 512, 8, 8, 128), (F16, [3001, 5, 0, 33], 1, 7, 1, 128)]


def unstored(c, byte):
    """A cache with a page more, the first one, that nobody lists, and `byte` for the scales of every block without a
    token of any sequence; the tables of it."""
    page, hd = c.page, c.hd
    data = np.concatenate([np.full_like(c.data[:1], 255), c.data])
    data[0, :, 2 * page * hd:] = byte
    table = c.table.astype(np.int64) + 1
    table[(c.table < 0) | (c.table >= len(c.data))] = -1
    stored = np.zeros((len(data), page // 32), bool)
    for b, n in enumerate(c.lens):
        for p in range(0, n, 32):
            stored[table[b, p // page], p % page // 32] = True
    for p, k in zip(*np.nonzero(~stored)):
        data[p, :, 2 * page * hd + 2 * k:2 * page * hd + 2 * k + 2] = byte
    return data, table


@pytest.mark.parametrize("dtype,lens,G,hq,hkv,hd", KINDS)
@pytest.mark.parametrize("page,fresh", [(64, False), (32, True)])
@pytest.mark.parametrize("byte", [255, 254, 0])
def test_scales_of_blocks_that_were_never_stored(dtype, lens, G, hq, hkv, hd, page, fresh, byte):
    say(f"unstored blocks {dtype} lens={lens} G={G} heads={hq}/{hkv} hd={hd} page={page} byte={byte}")
    c = Case(dtype, lens, G, hq, hkv, hd, page, fresh, seed=60 + G)
    data, table = unstored(c, byte)
    c.check(c.run(data=data, table=table), rows_of=SOME)


@pytest.mark.parametrize("dtype,lens,G,hq,hkv,hd", KINDS)
@pytest.mark.parametrize("byte", [255, 0])
def test_pages_that_the_cache_has_not(dtype, lens, G, hq, hkv, hd, byte):
    """Entries outside the pool are left out, whatever the pool's first page holds."""
    say(f"missing pages {dtype} lens={lens} G={G} heads={hq}/{hkv} hd={hd} byte={byte}")
    c = Case(dtype, lens, G, hq, hkv, hd, 64, False, seed=70 + G)
    data, table = unstored(c, byte)
    gone = {0: [0], len(lens) - 1: [0], int(np.argmax(lens)): [1, oc.pages(max(lens), 64) - 1]}
    for b, pages in gone.items():
        keep = np.ones(lens[b], bool)
        for i, p in enumerate(pages):
            if p * 64 >= lens[b]:
                continue
            table[b, p] = (-1, len(data), 2**31 - 1)[(b + i) % 3]
            keep[p * 64:(p + 1) * 64] = False
        c.K[b], c.V[b] = c.K[b][:, keep], c.V[b][:, keep]
    c.check(c.run(data=data, table=table), rows_of=SOME)
    # no page at all
    c.K, c.V = [k[:, :0] for k in c.K], [v[:, :0] for v in c.V]
    c.check(c.run(data=data, table=np.full_like(table, -1)), rows_of=SOME)
