"""The 4-bit cache's calls at the same time on several streams."""

import pytest
import torch

from gpu_util import archer, say

pytestmark = pytest.mark.gpu


class Work:
    """A stream's calls: attentions cut along the keys, each with the workspace of its own call, stores of the rows
    behind the cached ones and reads of them.  Everything is on the device before the first call."""

    def __init__(self, seed, turns):
        a = archer()
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.n, self.hq, hkv, hd, page, more = [9000, 300 + seed], 8, 2, 128, 64, 200
        width = -(-(max(self.n) + turns * more) // page)
        data = torch.randint(0, 256, (2 * width, hkv, page * (hd + hd // 16)), generator=g, device="cuda", dtype=torch.uint8)
        data[:, :, page * hd:] = 125
        self.data, self.page, self.hd = data, page, hd
        self.table = torch.randperm(2 * width, generator=g, device="cuda").int().view(2, width)
        self.q = torch.randn(turns, self.hq, 2, hd, generator=g, device="cuda").half()
        self.k = torch.randn(turns, hkv, 2 * more, hd, generator=g, device="cuda").half()
        self.v = torch.randn(turns, hkv, hd, 2 * more, generator=g, device="cuda").half()
        self.lens, self.slots = [], []
        for t in range(turns + 1):
            lens = torch.tensor([x + t * more for x in self.n], device="cuda")
            self.lens.append(lens.int())
            p = lens[:, None] + torch.arange(more, device="cuda")
            self.slots.append((torch.gather(self.table, 1, (p // page).clamp(max=width - 1)) * page + p % page).int().view(-1))
        self.most = max(self.n) + turns * more
        nb = a.lib.archer_op_attention_cache4_ws_bytes(0, 2, 1, self.hq, hkv, hd, self.most, 0)
        assert nb > 0, "the attention is meant to be cut"
        self.turns, self.more, self.hkv = turns, more, hkv

    def buffers(self):
        d = self.data.clone()
        return archer().Cache4(d, self.page, self.hd), torch.zeros(self.turns, 2, self.hq * self.hd, device="cuda",
                                                                   dtype=torch.bfloat16)

    def turn(self, cache, O, t):
        a = archer()
        a.op_attention_cache4(self.q[t], cache, self.table, self.lens[t], self.most, O=O[t])
        a.cache4_write(cache, self.k[t], self.v[t].transpose(1, 2), self.slots[t])
        return a.cache4_read(cache, self.slots[t])


def test_streams_at_the_same_time():
    turns = 25
    works = [Work(s, turns) for s in range(3)]
    want = []
    for w in works:                               # one after the other
        cache, O = w.buffers()
        rows = [w.turn(cache, O, t) for t in range(turns)]
        torch.cuda.synchronize()
        want.append((O, cache.data, rows))
    assert not torch.equal(want[0][0], want[1][0])
    streams = [torch.cuda.Stream() for _ in works]
    ev = [[torch.cuda.Event(enable_timing=True) for _ in range(2)] for _ in works]
    big = torch.randn(8192, 8192, device="cuda").half()
    # twice: the first pass leaves each stream's allocations behind; in the second the calls are queued while
    # large products hold all three streams, so that the host keeps ahead of them
    for gated in (False, True):
        bufs = [w.buffers() for w in works]
        got = [[] for _ in works]
        torch.cuda.synchronize()
        if gated:
            for _ in range(20):
                torch.mm(big, big)
        gate = torch.cuda.Event()
        gate.record()
        for t in range(turns):
            for i, (w, s) in enumerate(zip(works, streams)):
                with torch.cuda.stream(s):
                    if t == 0:
                        s.wait_event(gate)
                        ev[i][0].record()
                    got[i].append(w.turn(*bufs[i], t))
                    if t == turns - 1:
                        ev[i][1].record()
        torch.cuda.synchronize()
    for x in ev:                                  # they did run at the same time
        for y in ev:
            assert x[0].elapsed_time(y[1]) > 0
    say("us of the streams:", [round(1e3 * x[0].elapsed_time(x[1])) for x in ev])
    for (O, data, rows), (cache, O2), rows2 in zip(want, bufs, got):
        assert torch.equal(O, O2) and torch.equal(data, cache.data)
        for x, y in zip(rows, rows2):
            assert torch.equal(x[0], y[0]) and torch.equal(x[1], y[1])
