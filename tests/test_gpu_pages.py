"""GPU parity of the pages that several sequences share against their oracle: every output exactly."""

import numpy as np
import pytest
import torch

from gpu_util import archer, dev_i32, say
from oracle import pages as op
from test_pages import turns

pytestmark = pytest.mark.gpu


def same(got, want):
    np.testing.assert_array_equal(got.cpu().numpy(), want)


def gpu_call(name, args, want, in_place):
    """The call on the device, twice (once where it works in place), against the oracle's outputs."""
    a = archer()
    d = lambda x: dev_i32(x)  # noqa: E731
    for again in range(1 if in_place else 2):
        if name == "fork":
            src, dst, keep, page, table, refs = args
            t, r = d(table), d(refs)
            for _ in range(again + 1):
                out, st = a.pages_fork(d(src), d(dst), d(keep), page, t, r, refs_out=r if in_place else None)
            for g, w in ((t, want[0]), (out, want[1])):
                same(g, w)
            assert st.item() == want[2]
            if not in_place:
                same(r, refs)
        elif name == "plan":
            old, new, page, table, ring, pool, refs, rows = args
            t, f, r = d(table), d(ring), d(refs)
            for _ in range(again + 1):
                p = a.pages_plan(d(old), d(new), page, t, f, d(pool), r, rows, table_out=t if in_place else None,
                                 refs_out=r if in_place else None)
            for g, w in ((p.table, want[0]), (f, want[1]), (p.pool, want[2]), (p.refs, want[3]), (p.row_off, want[4]),
                         (p.slots, want[5]), (p.copy_src, want[6]), (p.copy_dst, want[7]), (p.status, [want[8]])):
                same(g, w)
            if not in_place:
                same(t, table)
                same(r, refs)
        else:
            length, page, table, refs = args
            t, r = d(table), d(refs)
            for _ in range(again + 1):
                m = a.pages_compact(d(length), page, t, r, table_out=t if in_place else None, refs_out=r if in_place else None)
            for g, w in zip(m, want[:6]):
                same(g, w)
            assert m.moves.item() == want[6]
            if not in_place:
                same(t, table)
                same(r, refs)


@pytest.mark.parametrize("in_place", [False, True])
@pytest.mark.parametrize("n_pages,rows,width,page,seed", [(1, 1, 1, 32, 0), (9, 3, 6, 32, 1), (64, 12, 6, 64, 2), (300, 40, 9, 32, 3),
                                                          (50, 70, 70, 256, 4)])
def test_turns_match_oracle(n_pages, rows, width, page, seed, in_place):
    say(f"turns pages={n_pages} rows={rows} in_place={in_place}")
    turns(n_pages, rows, width, page, seed, 8, lambda *c: gpu_call(*c, in_place))


def _large(B, page, n_pages, seed, samples):
    """A pool whose B rows share prompts in groups of `samples`: inputs of a plan that drops, writes and grows."""
    rng = np.random.default_rng(seed)
    width = 12
    table, refs, order, at = np.full((B, width), -1), np.zeros(n_pages, dtype=int), rng.permutation(n_pages), 0
    old = np.zeros(B, dtype=int)
    for b in range(0, B, samples):
        n = int(rng.integers(1, 9 * page))
        k = op.pages(n, page)
        for i in range(b, min(b + samples, B)):
            table[i, :k], old[i] = order[at:at + k], n
            refs[order[at:at + k]] += 1
        at += k
    new = np.where(rng.random(B) < 0.2, 0, np.where(rng.random(B) < 0.2, old // 2, old + rng.integers(0, 2 * page, B)))
    head, rest = int(rng.integers(0, n_pages)), n_pages - at
    ring = rng.integers(-9, 10**6, n_pages)
    ring[(head + np.arange(rest)) % n_pages] = order[at:]
    return old, new, page, table, ring, [head, rest], refs, int(np.maximum(new - old, 0).sum()) + 5


@pytest.mark.parametrize("B,page,samples", [(4096, 32, 7), (1000, 64, 64), (65, 256, 65), (2, 32, 2)])
def test_large_plan(B, page, samples):
    say(f"plan B={B} samples={samples}")
    args = _large(B, page, 60000, B, samples)
    want = op.plan(*args)
    assert want[8] == 0 and ((want[6] >= 0).any() or B == 2)
    gpu_call("plan", args, want, False)
    gpu_call("plan", args, want, True)


@pytest.mark.parametrize("change,want", [
    (dict(old=[-1, 3, 40]), 2), (dict(new=[0, 3, 97]), 2), (dict(new=[96, 96, 96], pool=[0, 3]), 1), (dict(rows=0), 3),
    (dict(pool=[9, 1]), 4), (dict(pool=[0, 10]), 4), (dict(pool=[-1, 1]), 4), (dict(table=[[0, 1, 2], [99, 3, 4], [5, 6, 7]]), 4),
    (dict(table=[[0, 1, 2], [3, 3, 4], [5, -6, 7]], new=[5, 3, 0]), 4), (dict(pool=[0, 9]), 4),
])
def test_plan_refusals_change_nothing(change, want):
    v = dict(old=[5, 3, 40], new=[6, 4, 0], page=32, table=[[0, 1, 2], [3, 1, 2], [4, 5, 7]], ring=[6, 7, 8, 0, 0, 0, 0, 0, 0],
             pool=[0, 3], refs=[1, 0, 0, 1, 1, 1, 0, 0, 0], rows=9)
    v.update(change)
    args = tuple(np.array(x) if isinstance(x, list) else x for x in v.values())
    out = op.plan(*args)
    assert out[8] == want
    for in_place in (False, True):
        gpu_call("plan", args, out, in_place)


@pytest.mark.parametrize("src,dst,keep", [([0], [4], [5]), ([0], [-1], [5]), ([4], [1], [5]), ([0, 0], [2, 2], [5, 5]),
                                          ([0, 2], [2, 3], [5, 5]), ([0], [1], [-1]), ([0], [1], [97]), ([0], [0], [5])])
def test_fork_refusals_change_nothing(src, dst, keep):
    args = (src, dst, keep, 32, np.arange(12).reshape(4, 3), np.arange(12))
    want = op.fork(*args)
    assert want[2] == 2
    for in_place in (False, True):
        gpu_call("fork", args, want, in_place)


def test_fork_of_nothing_and_of_foreign_entries():
    """No token: no page.  Entries of no page of the pool are listed and not counted."""
    args = ([0, 0, 1], [2, 3, 4], [0, 65, 64], 32, np.array([[3, -1, 77], [1, 2, 0]] + [[9, 9, 9]] * 3), np.ones(4, dtype=int))
    want = op.fork(*args)
    assert want[2] == 0
    gpu_call("fork", args, want, False)


@pytest.mark.parametrize("n_pages,used", [(1, 0), (1, 1), (2, 1), (2047, 0.5), (2048, 0.0), (2049, 1.0), (5000, 0.3), (100001, 0.7)])
def test_compact_of_many_pages(n_pages, used):
    say(f"compact {n_pages} {used}")
    rng = np.random.default_rng(n_pages)
    refs = np.where(rng.random(n_pages) < used, rng.integers(1, 4, n_pages), 0)
    pages = np.flatnonzero(refs)[:60]
    table = np.full((3, 61), -1)
    table[0, :len(pages)] = table[2, :len(pages)] = rng.permutation(pages)
    table[1, :2] = [-5, n_pages]         # no pages of the pool: left as they are
    args = ([len(pages) * 32, 64, max(len(pages) * 32 - 40, -3)], 32, table, refs)
    want = op.compact(*args)
    for in_place in (False, True):
        gpu_call("compact", args, want, in_place)


@pytest.mark.parametrize("shape", [(5, 1, 16), (3, 7, 2, 48), (2, 9, 3, 16400), (1, 4, 1, 65552), (40, 6, 4, 8208)])
@pytest.mark.parametrize("counted", [None, 2, 0, 99, -1])
def test_copy(shape, counted):
    say(f"copy {shape} {counted}")
    a = archer()
    g = torch.Generator().manual_seed(shape[-1])
    data = torch.randint(0, 256, shape, generator=g, dtype=torch.uint8)
    n_pages = shape[-3]
    src, dst = [0, -1, 1, n_pages, 0, 0], [2, 3, -1, 3, 3, n_pages]
    want = data.clone()
    for s, d in list(zip(src, dst))[:len(src) if counted is None else max(counted, 0)]:
        if 0 <= s < n_pages and 0 <= d < n_pages:
            want[..., d, :, :] = data[..., s, :, :]
    got = data.cuda()
    a.pages_copy(got, dev_i32(src), dev_i32(dst), count=None if counted is None else dev_i32([counted]))
    assert torch.equal(got.cpu(), want)


def test_copy_into_far_pages():
    """Offsets beyond 32 bits: pages of 64 MiB, the far ones past 4 GiB."""
    a = archer()
    data = torch.zeros(70, 1, 1 << 26, dtype=torch.uint8, device="cuda")
    data[3] = 7
    data[69, 0, -5:] = 9
    a.pages_copy(data, dev_i32([3, 69]), dev_i32([66, 1]))
    assert (data[66] == 7).all() and (data[1, 0, -5:] == 9).all() and not data[1, 0, :-5].any() and not data[67].any()


@pytest.mark.parametrize("B,n_pages,width,slots", [(16, 4096, 12, 0), (17, 4096, 12, 0), (16, 4097, 12, 0), (16, 4096, 1024, 0), (16, 4096, 1025, 0),
                                                   (15, 4000, 12, 16384), (15, 4000, 12, 16385)])
def test_plans_at_the_end_of_small_ones(B, n_pages, width, slots):
    """The largest plan that one workgroup makes and the first ones that it does not: rows, pages, table entries, slots."""
    say(f"small plan B={B} pages={n_pages} width={width} slots={slots}")
    old, new, page, table, ring, pool, refs, rows = _large(B, 32, n_pages, B + width, 3)
    table = np.pad(table, ((0, 0), (0, width - table.shape[1])), constant_values=-1)
    args = old, new, page, table, ring, pool, refs, max(rows, slots)
    want = op.plan(*args)
    assert want[8] == 0 and (want[6] >= 0).any()
    gpu_call("plan", args, want, False)
    gpu_call("plan", args, want, True)
