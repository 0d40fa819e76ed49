"""Pages of the 4-bit cache that several rows of a table list."""

import numpy as np
import pytest
import torch

from gpu_util import archer, dev_i32
from oracle import cache4 as oc
from test_gpu_cache4 import random_bytes

pytestmark = pytest.mark.gpu


def test_pages_shared_by_rows_outside_the_plan():
    """A prompt's pages belong to one planned request; other rows of an attention's table list them as well.  While the
    owner keeps them, the plans of other requests take none of them, and the sharers' results stay."""
    a = archer()
    rng = np.random.default_rng(90)
    page, hkv, hd, hq, n_pages = 32, 2, 128, 4, 12
    cache = a.Cache4(torch.from_numpy(random_bytes(rng, n_pages, hkv, page, hd)).cuda(), page, hd)
    table, ring, pool = dev_i32(np.full((2, 6), -1)), dev_i32(rng.permutation(n_pages)), dev_i32([0, n_pages])
    # request 0 is the prompt, request 1 another one
    old = [0, 0]

    def plan(new):
        nonlocal old, pool
        pool, off, slots, st = a.cache4_plan(dev_i32(old), dev_i32(new), page, table, ring, pool, 200)
        assert st.item() == 0
        g = torch.Generator(device="cuda").manual_seed(sum(new))
        k, v = (torch.randn(hkv, 200, hd, generator=g, device="cuda").half() for _ in range(2))
        a.cache4_write(cache, k, v, slots)
        old = new

    plan([70, 40])
    shared = table[0, :3].tolist()
    q = torch.randn(hq, 3, hd, device="cuda").half()
    sharers = dev_i32([shared, shared[:2] + [-1], shared])
    lens = dev_i32([70, 64, 5])
    first = a.op_attention_cache4(q, cache, sharers, lens, 70)
    for new in ([70, 150], [70, 20], [70, 180], [70, 0]):
        plan(new)
        assert table[0, :3].tolist() == shared
        assert not set(shared) & set(table[1, :oc.pages(new[1], page)].tolist())
        assert torch.equal(a.op_attention_cache4(q, cache, sharers, lens, 70), first)
    plan([0, 0])                                  # the sharers are done: now the owner gives them back, each once
    head, count = pool.tolist()
    assert count == n_pages
    assert sorted(int(ring[(head + i) % n_pages]) for i in range(count)) == list(range(n_pages))
