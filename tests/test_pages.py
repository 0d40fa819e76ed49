"""Pages that several sequences share, without a GPU: the oracle against first principles, and the
library's refusals (every one before a launch)."""

import numpy as np
import pytest
import torch

from oracle import pages as op


class Server:
    """A pool as a program would keep it by hand: sequences as lists of pages, for comparison with the oracle."""

    def __init__(self, n_pages, rows, width, page, seed):
        self.rng = np.random.default_rng(seed)
        self.page, self.width = page, width
        self.table = np.full((rows, width), -1)
        self.refs = np.zeros(n_pages, dtype=np.int64)
        self.ring = self.rng.permutation(n_pages)
        self.pool = np.array([0, n_pages])
        self.len = np.zeros(rows, dtype=np.int64)

    def check(self):
        held = [self.table[b, :op.pages(n, self.page)] for b, n in enumerate(self.len)]
        count = np.zeros_like(self.refs)
        for r in held:
            assert len(set(r)) == len(r)
            np.add.at(count, r, 1)
        np.testing.assert_array_equal(count, self.refs)
        free = self.ring[(self.pool[0] + np.arange(self.pool[1])) % len(self.refs)]
        assert sorted(free) == sorted(np.flatnonzero(count == 0))

    def random_fork(self):
        empty, live = np.flatnonzero(self.len == 0), np.flatnonzero(self.len > 0)
        k = min(len(empty), int(self.rng.integers(0, 4)))
        if not len(live):
            k = 0
        dst = self.rng.permutation(empty)[:k]
        src = self.rng.choice(live, k) if k else np.zeros(0, dtype=np.int64)
        return src, dst, np.array([int(self.rng.integers(1, self.len[s] + 1)) for s in src], dtype=np.int64)

    def random_lengths(self):
        new = self.len.copy()
        for b in range(len(new)):
            u = self.rng.random()
            if u < 0.4:
                new[b] = min(new[b] + int(self.rng.integers(1, 2 * self.page)), self.width * self.page)
            elif u < 0.6:
                new[b] = int(self.rng.integers(0, new[b] + 1))
            elif u < 0.7:
                new[b] = 0
        return new

    def takes(self, new):
        return sum(op.pages(n, self.page) + 1 for n in new)


def turns(n_pages, rows, width, page, seed, n, each):
    """n turns of forks, plans and compactions; each(name, inputs, outputs) sees every call."""
    s = Server(n_pages, rows, width, page, seed)
    for i in range(n):
        src, dst, keep = s.random_fork()
        if len(src):
            args = (src, dst, keep, page, s.table, s.refs)
            out = op.fork(*args)
            each("fork", args, out)
            s.table, s.refs, st = out
            assert st == 0
            s.len[dst] = keep
            s.check()
        new = s.random_lengths()
        grown = int(np.maximum(new - s.len, 0).sum())
        args = (s.len.copy(), new, page, s.table, s.ring, s.pool, s.refs, grown + 3)
        out = op.plan(*args)
        each("plan", args, out)
        if out[-1] == 0:
            before = {b: [int(x) for x in s.table[b, :op.pages(s.len[b], page)]] for b in range(rows)}
            s.table, s.ring, s.pool, s.refs = out[:4]
            # nobody's earlier tokens changed their page but for the copies, and no new token is on a shared page
            for b in range(rows):
                kept = op.pages(min(s.len[b], new[b]), page)
                for j in range(kept):
                    assert s.table[b, j] == before[b][j] or (out[6][b] == before[b][j] and out[7][b] == s.table[b, j])
                if new[b] > s.len[b]:
                    assert all(s.refs[s.table[b, j]] == 1 for j in range(s.len[b] // page, op.pages(new[b], page)))
            s.len = new
        else:
            assert out[-1] == 1
        s.check()
        if i % 3 == 2:
            args = (s.len.copy(), page, s.table, s.refs)
            out = op.compact(*args)
            each("compact", args, out)
            s.table, s.refs, s.ring, s.pool = out[:4]
            s.check()
            assert (s.refs[:int((s.refs > 0).sum())] > 0).all()


@pytest.mark.parametrize("seed", range(6))
def test_turns_keep_the_pool(seed):
    turns([9, 40, 64, 7, 200, 64][seed], [3, 9, 12, 2, 30, 5][seed], 6, 32, seed, 30, lambda *a: None)


def test_the_last_holder_keeps_the_page():
    """Three rows share a page of 5 tokens; where all grow, two copy; where one holds still, all that grow copy."""
    table, refs = np.array([[7, -1]] * 3), np.zeros(10, dtype=int)
    refs[7] = 3
    ring = np.array([0, 1, 2, 3, 4, 5, 6, 8, 9, 0])
    for new, src, dst, left in (([6, 6, 6], [7, 7, -1], [0, 1, -1], 1), ([6, 5, 6], [7, -1, 7], [0, -1, 1], 1),
                                ([6, 0, 6], [7, -1, -1], [0, -1, -1], 1), ([0, 6, 0], [-1] * 3, [-1] * 3, 1),
                                ([0, 0, 0], [-1] * 3, [-1] * 3, 0)):
        out = op.plan([5] * 3, new, 32, table, ring, [0, 9], refs, 9)
        assert out[8] == 0
        assert list(out[6]) == src and list(out[7]) == dst and out[3][7] == left
        if left == 0:        # given back once
            assert list(out[1]) == [0, 1, 2, 3, 4, 5, 6, 8, 9, 7] and list(out[2]) == [0, 10]


# -- refusals of the library: every one before a launch, so any aligned address will do ------------
A = 1 << 20


@pytest.fixture
def lib():
    from paper_2608_08086_amd import archer
    return archer


def _refused(a, status, code, text):
    assert status == code
    assert text in a.lib.archer_last_error().decode()


@pytest.mark.parametrize("change,code,text", [
    (dict(n=0), "E_SHAPE", "n must"), (dict(n=4097), "E_SHAPE", "n must"), (dict(rows=65537), "E_SHAPE", "n_rows"),
    (dict(page=48), "E_SHAPE", "page_size"), (dict(pages=0), "E_SHAPE", "n_pages"), (dict(pages=1 << 26), "E_SHAPE", "n_pages"),
    (dict(width=0), "E_SHAPE", "max_pages"), (dict(width=1 << 27), "E_SHAPE", "max_pages"), (dict(src=0), "E_ARG", "null"),
    (dict(out=4 * A + 4), "E_ARG", "overlap"),
])
def test_fork_refusals(lib, change, code, text):
    v = dict(n=2, src=A, dst=2 * A, len=3 * A, page=32, pages=9, rows=4, width=5, table=5 * A, refs=4 * A, out=4 * A, status=6 * A)
    v.update(change)
    _refused(lib, lib.lib.archer_pages_fork(*v.values(), None), getattr(lib, code), text)


@pytest.mark.parametrize("change,code,text", [
    (dict(batch=0), "E_SHAPE", "batch"), (dict(batch=4097), "E_SHAPE", "batch"), (dict(page=16), "E_SHAPE", "page_size"),
    (dict(pages=-1), "E_SHAPE", "n_pages"), (dict(width=0), "E_SHAPE", "max_pages"), (dict(rows=-1), "E_SHAPE", "slot_rows"),
    (dict(slots=0), "E_ARG", "null"), (dict(pool_out=7 * A + 4), "E_ARG", "pool_out"), (dict(t_out=4 * A + 4), "E_ARG", "overlap"),
    (dict(r_out=9 * A - 4), "E_ARG", "overlap"), (dict(ws=0), "E_WORKSPACE", "workspace"), (dict(ws=16 * A + 4), "E_WORKSPACE", "workspace"),
    (dict(bytes=255), "E_WORKSPACE", "workspace"),
])
def test_plan_refusals(lib, change, code, text):
    v = dict(batch=2, old=A, new=2 * A, page=32, pages=9, width=5, t_in=4 * A, t_out=4 * A, free=6 * A, pool_in=7 * A,
             pool_out=8 * A, r_in=9 * A, r_out=9 * A, off=10 * A, slots=11 * A, rows=4, src=12 * A, dst=13 * A, status=14 * A,
             ws=16 * A, bytes=256)
    v.update(change)
    _refused(lib, lib.lib.archer_pages_plan(*v.values(), None), getattr(lib, code), text)


@pytest.mark.parametrize("change,code,text", [
    (dict(batch=0), "E_SHAPE", "batch"), (dict(page=0), "E_SHAPE", "page_size"), (dict(pages=0), "E_SHAPE", "n_pages"),
    (dict(width=-1), "E_SHAPE", "max_pages"), (dict(src=0), "E_ARG", "null"), (dict(t_out=3 * A + 8), "E_ARG", "overlap"),
    (dict(r_out=5 * A + 4), "E_ARG", "overlap"), (dict(bytes=0), "E_WORKSPACE", "workspace"),
])
def test_compact_refusals(lib, change, code, text):
    v = dict(batch=2, len=A, page=32, pages=9, width=5, t_in=3 * A, t_out=3 * A, r_in=5 * A, r_out=5 * A, free=6 * A,
             pool=7 * A, src=8 * A, dst=9 * A, moves=10 * A, ws=16 * A, bytes=256)
    v.update(change)
    _refused(lib, lib.lib.archer_pages_compact(*v.values(), None), getattr(lib, code), text)


@pytest.mark.parametrize("change,code,text", [
    (dict(bytes=24), "E_SHAPE", "page_bytes"), (dict(bytes=0), "E_SHAPE", "page_bytes"), (dict(bytes=2**62), "E_SHAPE", "2^63"),
    (dict(pages=0), "E_SHAPE", "n_pages"), (dict(planes=0), "E_SHAPE", "plane_stride"), (dict(stride=272), "E_SHAPE", "plane_stride"),
    (dict(stride=4 * 256 + 8), "E_SHAPE", "plane_stride"), (dict(n=-1), "E_SHAPE", "n must"), (dict(data=A + 8), "E_ARG", "aligned"),
    (dict(src=0), "E_ARG", "null"),
])
def test_copy_refusals(lib, change, code, text):
    v = dict(bytes=256, pages=4, planes=2, stride=1024, data=A, n=3, src=2 * A, dst=3 * A, count=0)
    v.update(change)
    _refused(lib, lib.lib.archer_pages_copy(*v.values(), None), getattr(lib, code), text)


def test_no_pairs_is_no_launch(lib):
    assert lib.lib.archer_pages_copy(256, 4, 1, 1024, None, 0, None, None, None, None) == lib.OK


def test_workspaces(lib):
    assert lib.lib.archer_pages_plan_ws_bytes(4, 100) >= 4 * (200 + 9)
    assert lib.lib.archer_pages_plan_ws_bytes(0, 100) == lib.lib.archer_pages_plan_ws_bytes(4, 0) == 0
    assert lib.lib.archer_pages_compact_ws_bytes(5000) >= 4 * 5003
    assert lib.lib.archer_pages_compact_ws_bytes(-1) == 0


def test_binding_refusals(lib, monkeypatch):
    """Host tensors in the place of the device's: every refusal comes before the library is called."""
    a = lib
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    for f in ("archer_pages_fork", "archer_pages_plan", "archer_pages_compact", "archer_pages_copy"):
        monkeypatch.setattr(a.lib, f, lambda *x: pytest.fail("the library was called"))
    i = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    t, refs = i(0, 1, 2, 3).view(2, 2), i(0, 0, 0, 0, 0)
    for f in (lambda: a.pages_fork(i(0), i(1, 1), i(3), 32, t, refs), lambda: a.pages_fork(i(0), i(1), i(3).long(), 32, t, refs),
              lambda: a.pages_fork(i(0), i(1), i(3), 2**32 + 32, t, refs), lambda: a.pages_fork(i(0), i(1), i(3), 32, t[0], refs),
              lambda: a.pages_fork(i(0), i(1), i(3), 32, t, refs, refs_out=refs[:3]),
              lambda: a.pages_plan(i(1, 1), i(2, 2), 32, t, refs, i(0, 1), refs, 2**31),
              lambda: a.pages_plan(i(1), i(2), 32, t, refs, i(0, 1), refs, 4),
              lambda: a.pages_plan(i(1, 1), i(2, 2), 32, t, refs[:4], i(0, 1), refs, 4),
              lambda: a.pages_plan(i(1, 1), i(2, 2), 32, t.T, refs, i(0, 1), refs, 4),
              lambda: a.pages_plan(i(1, 1), i(2, 2), 32, t, refs, i(0, 1), refs, 4, table_out=t[:1]),
              lambda: a.pages_compact(i(1), 32, t, refs), lambda: a.pages_compact(i(1, 1), -32, t, refs),
              lambda: a.pages_copy(torch.zeros(4, 32), i(0), i(1)), lambda: a.pages_copy(torch.zeros(4, 2, 32)[:, :1], i(0), i(1)),
              lambda: a.pages_copy(torch.zeros(4, 2, 32), i(0), i(1, 2)),
              lambda: a.pages_copy(torch.zeros(4, 2, 32), i(0), i(1), count=i(1, 1)),
              lambda: a.pages_copy(torch.zeros(0, 4, 2, 32), i(0), i(1))):
        with pytest.raises(a.ArcherError):
            f()
