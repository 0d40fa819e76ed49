"""GPU parity of sampling against its oracle.

Tokens have to be the oracle's wherever no border is as near as the kernel's sums may be off: weights to 2^-44
of themselves, sums in 64 bits, and tokens more than 33 nats below the largest left out, which are at most
2^19 e^-33 = 2^-28.6 of the weight.  So `oracle.sample.safe` with 2^-28; what is nearer is rare, and counted.
A log-probability is then off by 2^-27 and its rounding, 2^-24 of it."""

import numpy as np
import pytest
import torch

from gpu_util import archer, dev_f32, dev_i32, say
from oracle import sample as osm

pytestmark = pytest.mark.gpu

T = {"fp32": torch.float32, "bf16": torch.bfloat16, "fp16": torch.float16}


def run(logits, u, kw, exclude=-1, view=None):
    a = archer()
    t = logits if view is None else view
    d = {k: (dev_i32(v) if k == "top_k" else dev_f32(v)) for k, v in kw.items()}
    return a.op_sample(t, dev_f32(u), exclude=exclude, **d)


def check(logits, u, kw, exclude=-1, view=None, most_unsafe=0.02):
    """logits: CUDA [rows][vocab]; u and the lists in kw: one value a row."""
    token, logp = (x.cpu().numpy() for x in run(logits, u, kw, exclude, view))
    host = logits.float().cpu().numpy()
    u = np.asarray(u, dtype=np.float32).astype(np.float64)
    unsafe = 0
    for r in range(len(host)):
        row = {k: (int(v[r]) if k == "top_k" else float(np.float32(v[r]))) for k, v in kw.items()}
        want = osm.sample(host[r], u[r], exclude=exclude, **row)
        if not osm.safe(host[r], u[r], exclude=exclude, **row):
            unsafe += 1
            continue
        assert token[r] == want[0], (r, row, u[r], token[r], want)
        if not np.isfinite(want[1]):
            np.testing.assert_equal(logp[r], want[1])
        else:
            assert abs(logp[r] - want[1]) <= 2.0**-24 * abs(want[1]) + 2.0**-27, (r, logp[r], want[1])
    assert unsafe <= most_unsafe * len(host)
    return token


def logits_of(rng, rows, vocab, spread, dtype="fp32", peaks=True):
    z = rng.standard_normal((rows, vocab)) * spread
    if peaks:
        for r in range(rows):
            z[r, rng.integers(0, vocab, 6)] += rng.random(6) * 10
    return torch.from_numpy(z).to(T[dtype]).cuda()


SETTINGS = [{}, dict(top_k=1), dict(top_k=7), dict(top_p=0.9), dict(top_p=0.3), dict(min_p=0.1), dict(top_k=40, top_p=0.95),
            dict(top_k=40, top_p=0.9, min_p=0.02), dict(top_p=0.8, min_p=0.3), dict(top_k=10**6), dict(top_p=0.0), dict(min_p=1.0)]


@pytest.mark.parametrize("vocab", [1, 2, 3, 4, 5, 7, 8, 9, 63, 64, 65, 255, 1000, 1024, 4095, 4096, 4097, 50257])
@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
def test_sizes(vocab, dtype):
    say(f"sizes {vocab} {dtype}")
    rng = np.random.default_rng(vocab)
    n = len(SETTINGS) * (3 if vocab < 10000 else 1)
    z = logits_of(rng, n, vocab, 2.0, dtype)
    kw = {k: [SETTINGS[i % len(SETTINGS)].get(k, d) for i in range(n)] for k, d in (("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))}
    kw["temperature"] = 0.3 + rng.random(n)
    check(z, rng.random(n), kw, most_unsafe=0.1)


@pytest.mark.parametrize("vocab", [126464, 152064])
@pytest.mark.parametrize("spread,temp", [(0.02, 1.0), (1.0, 1.3), (3.0, 0.7), (8.0, 0.2)])
def test_vocabularies(vocab, spread, temp):
    """From flat rows, of whose tokens most are kept, to sharp ones."""
    say(f"vocab {vocab} spread {spread}")
    rng = np.random.default_rng(int(spread * 100))
    n = len(SETTINGS)
    z = logits_of(rng, n, vocab, spread, peaks=spread > 0.5)
    kw = {k: [s.get(k, d) for s in SETTINGS] for k, d in (("top_k", 0), ("top_p", 1.0), ("min_p", 0.0))}
    kw["temperature"] = [temp] * n
    check(z, rng.random(n), kw, exclude=vocab - 1, most_unsafe=0.1)


@pytest.mark.parametrize("k,p,m", [(3000, 1.0, 0.0), (3000, 0.5, 0.0), (30000, 0.99, 0.0), (30000, 0.9, 0.3), (0, 0.99, 0.05), (0, 1.0, 0.05),
                                   (49999, 1.0, 0.0), (2048, 0.9, 0.0), (2049, 0.9, 0.0), (5000, 0.0001, 0.0), (0, 0.9999999, 0.0)])
@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
def test_many_kept(k, p, m, dtype):
    """More kept tokens than are sorted in one go; bf16: many equal logits at every cut."""
    say(f"many k={k} p={p} m={m} {dtype}")
    rng = np.random.default_rng(k + 1)
    z = logits_of(rng, 4, 50000, 1.0, dtype, peaks=False)
    check(z, rng.random(4), dict(top_k=[k] * 4, top_p=[p] * 4, min_p=[m] * 4, temperature=[1.0, 0.5, 2.0, 30.0]), most_unsafe=0.3)


@pytest.mark.parametrize("values", [[0.0], [0.0, -0.0], [1.5, 1.5, 1.25], [0.0, -3.0, -3.0, -3.0]])
@pytest.mark.parametrize("k,p", [(0, 1.0), (5000, 1.0), (0, 0.37), (7001, 0.41), (3, 1.0), (19999, 0.9)])
def test_equal_logits(values, k, p):
    """A few values, each more often than the list holds: ties go to the lower index."""
    rng = np.random.default_rng(k + len(values))
    z = torch.tensor(rng.choice(values, (5, 20000)), dtype=torch.float32, device="cuda")
    check(z, rng.random(5), dict(top_k=[k] * 5, top_p=[p] * 5), most_unsafe=0.0 if k == 0 and p == 1 else 0.2)


def test_the_draw_walks_through_the_row():
    """Equal weights, power of two many: u = i / n is token i, and just below it token i - 1."""
    n = 4096
    z = torch.zeros(1, n, device="cuda").expand(2 * n - 1, n)        # rows with stride 0
    i = np.arange(1, n)
    u = np.concatenate([np.arange(n) / n, np.nextafter((i / n).astype(np.float32), np.float32(0))])
    token, logp = run(None, u, {}, view=z)
    assert token.tolist() == list(range(n)) + list(range(n - 1))
    np.testing.assert_array_equal(logp.cpu().numpy(), np.float32(np.log(1 / n)))


@pytest.mark.parametrize("first", [-30.0, -np.inf, -1000.0])
@pytest.mark.parametrize("kw", [{}, dict(top_p=0.9), dict(top_k=5)])
def test_the_reference_is_far_off(first, kw):
    """The tokens that the reference is taken from are far below the row's others, or none at all; and the other way round."""
    rng = np.random.default_rng(3)
    z = rng.standard_normal((4, 9000))
    z[:2, :6000] = first + (0 if np.isinf(first) else rng.standard_normal((2, 6000)))
    z[2:, 6000:] = -500
    z[3] -= 900
    t = [1.0, 0.05, 1.0, 0.1]
    check(torch.from_numpy(z).float().cuda(), rng.random(4), dict({k: [v] * 4 for k, v in kw.items()}, temperature=t), most_unsafe=0.3)


@pytest.mark.parametrize("kw", [{}, dict(top_p=0.9), dict(top_k=5), dict(min_p=0.3), dict(top_k=3000, top_p=0.9)])
def test_infinite_and_nan_logits(kw):
    rng = np.random.default_rng(4)
    z = rng.standard_normal((8, 5000)).astype(np.float32)
    z[0] = -np.inf
    z[1] = -np.inf
    z[1, 77] = 3
    z[2, [5, 4000]] = np.inf
    z[3, 4999] = np.nan
    z[4, 17] = np.nan
    z[5, ::2] = -np.inf
    z[6, 17] = np.inf
    z[7, 4900] = np.inf
    z[7, 3] = np.nan
    d = {k: [v] * 8 for k, v in kw.items()}
    u = rng.random(8)
    tok = check(torch.from_numpy(z).cuda(), u, d, most_unsafe=0.3)
    assert tok[0] == tok[3] == tok[4] == tok[7] == -1 and tok[1] == 77 and tok[2] in (5, 4000) and tok[5] % 2 == 1 and tok[6] == 17
    tok = check(torch.from_numpy(z).cuda(), u, d, exclude=17, most_unsafe=0.3)     # what is excluded may be anything
    assert tok[4] >= 0 and tok[6] != 17
    one = torch.full((2, 3), -torch.inf, device="cuda")
    one[1, 1] = 0
    assert check(one, [0.5, 0.5], {}, exclude=1).tolist() == [-1, -1]


@pytest.mark.parametrize("t", [0.0, -1.0, np.nan, 1e-38, 1e-45, 1e-3, 50.0, 1e30, np.inf])
def test_temperatures(t):
    rng = np.random.default_rng(5)
    z = rng.standard_normal((6, 3000)).astype(np.float32)
    z[:, 2000] = z[:, 100] = 4.0                     # the maximum, twice
    kw = dict(temperature=[t] * 6, top_k=[0, 0, 2500, 5, 0, 0], top_p=[1, 0.9, 1, 1, 0.999, 1], min_p=[0, 0, 0, 0, 0, 1.0])
    u = [0.4999, 0.7, 0.2, 0.9, 0.3, 0.6]
    # at 1e30 and beyond every weight is 1: of six rows' borders, 0.2 * 2500 and 0.999 * 3000 are whole numbers of
    # tokens (to 2^-25, u's own rounding), and every weight is min_p = 1
    tok = check(torch.from_numpy(z).cuda(), u, kw, most_unsafe=0.5)
    if not t > 0:
        assert (tok == 100).all()


def test_u_at_its_ends():
    rng = np.random.default_rng(6)
    z = logits_of(rng, 6, 30000, 1.0)
    z[:, 0] = z[:, -1] = -torch.inf
    last = np.nextafter(np.float32(1), np.float32(0))
    kw = dict(top_p=[1, 1, 0.5, 0.5, 1, 1], top_k=[0, 0, 0, 0, 6, 6])
    tok, _ = (x.cpu().numpy() for x in run(z, [0, last, 0, last, 0, last], kw))
    for r in range(6):
        w, _ = osm.kept(z[r].cpu().numpy(), top_p=kw["top_p"][r], top_k=kw["top_k"][r])
        assert w[tok[r]] > 0
        pos = np.flatnonzero(w)
        share = w[:tok[r]].sum() / w.sum()
        assert tok[r] == pos[0] if r % 2 == 0 else share >= float(last) - w[tok[r]] / w.sum() - 2.0**-28
    # at one and beyond (outside the interval): a kept token all the same
    tok, _ = run(z, [1.0, 2.0, 1.0, np.inf, 1.0, -1.0], kw)
    assert all(osm.kept(z[r].cpu().numpy(), top_p=kw["top_p"][r], top_k=kw["top_k"][r])[0][int(tok[r])] > 0 for r in range(6))


@pytest.mark.parametrize("dtype", ["fp32", "bf16", "fp16"])
@pytest.mark.parametrize("off,pad", [(0, 1), (1, 0), (3, 5), (5, 64)])
def test_strides_and_alignment(dtype, off, pad):
    rng = np.random.default_rng(off)
    n, V = 4, 9001
    big = torch.full((n, V + off + pad), float("nan"), dtype=T[dtype], device="cuda")      # what lies around is not read
    view = big[:, off:off + V]
    view.copy_(logits_of(rng, n, V, 2.0, dtype))
    check(view, rng.random(n), dict(top_p=[0.9, 1, 0.5, 1], top_k=[0, 0, 9, 3000]), most_unsafe=0.3)


def test_far_rows():
    """Rows past 2^32 elements."""
    V, n = 400000, 11000
    base = torch.empty(V * n, dtype=torch.float16, device="cuda")
    rows = base.view(n, V)[[0, n - 1]].clone()
    z = logits_of(np.random.default_rng(7), 2, V, 2.0, "fp16")
    view = base.view(n, V)[::n - 1]
    view.copy_(z)
    assert view.stride(0) > 2**32
    del rows
    check(view, [0.3, 0.8], dict(top_p=[0.9, 1.0]), view=view, most_unsafe=0.5)


def test_same_bits_again_in_other_company_and_on_another_stream():
    rng = np.random.default_rng(8)
    z = logits_of(rng, 40, 20000, 1.0, "bf16")
    u = rng.random(40)
    kw = dict(top_p=[0.9] * 20 + [1.0] * 20, top_k=([0] * 10 + [50] * 10) * 2)
    a = run(z, u, kw)
    b = run(z[5:9], u[5:9], {k: v[5:9] for k, v in kw.items()})
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        c = run(z, u, kw)
    s.synchronize()
    for x, y, w in zip(a, b, c):
        assert torch.equal(x[5:9], y) and torch.equal(x, w)


def test_captured_and_replayed():
    rng = np.random.default_rng(9)
    a = archer()
    z = logits_of(rng, 8, 30000, 2.0)
    u, p = dev_f32(rng.random(8)), dev_f32([0.9] * 8)
    a.op_sample(z, u, top_p=p)
    torch.cuda.synchronize()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=torch.cuda.Stream()):
        got = a.op_sample(z, u, top_p=p)
    for i in range(3):
        z.copy_(logits_of(rng, 8, 30000, 0.5 + i))
        u.copy_(dev_f32(rng.random(8)))
        g.replay()
        torch.cuda.synchronize()
        for x, y in zip(got, a.op_sample(z, u, top_p=p)):
            assert torch.equal(x, y)


def test_no_temperature_is_the_decision_of_archer_decide():
    """Greedy rows: the decoder's argmax, MASK left out."""
    rng = np.random.default_rng(10)
    z = logits_of(rng, 16, 1024, 1.0)
    z[:, 1023] = 99
    tok, logp = run(z, [0.5] * 16, dict(temperature=[0.0] * 16), exclude=1023)
    assert torch.equal(tok.long(), z[:, :1023].argmax(-1)) and not logp.any()


@pytest.mark.parametrize("dtype", ["fp32", "bf16"])
@pytest.mark.parametrize("kw", [dict(top_k=3500, top_p=0.95), dict(top_k=3999, top_p=0.5, min_p=0.001), dict(top_p=0.7), dict(top_k=3900), dict(min_p=0.3)])
def test_long_lists_of_one_part(kw, dtype):
    """A vocabulary that one workgroup has, most of which is kept."""
    say(f"one part {kw} {dtype}")
    rng = np.random.default_rng(11)
    z = logits_of(rng, 3, 4000, 1.0, dtype, peaks=False)
    check(z, rng.random(3), dict({k: [v] * 3 for k, v in kw.items()}, temperature=[1.0, 0.4, 3.0]), most_unsafe=0.4)


@pytest.mark.parametrize("kw", [dict(top_p=0.4), dict(top_p=0.9), dict(top_k=30000), dict(top_k=60000, top_p=0.8), dict(top_k=100, top_p=0.5),
                                dict(min_p=0.2), dict(min_p=0.5, top_p=0.99), {}])
def test_values_that_many_tokens_share(kw):
    """Two values of 50000 tokens each: lists that are too long.  Weights 1 and 1/4 (in 64 bits to 2^-52)."""
    say(f"shared {kw}")
    rng = np.random.default_rng(12)
    z = torch.from_numpy(np.where(rng.random((2, 100000)) < 0.5, 0.0, -1.0)).float().cuda()
    # 100 tokens of one weight and half of them: the border of top_p is the sum of the first 50 exactly, so every row is at one
    at_border = kw.get("top_k") == 100
    check(z, [0.3, 0.9], dict({k: [v] * 2 for k, v in kw.items()}, temperature=[1 / np.log(4.0)] * 2), most_unsafe=1.0 if at_border else 0.5)


@pytest.mark.parametrize("kw", [dict(top_p=0.9), dict(top_k=20), dict(top_k=20, top_p=0.9), dict(min_p=0.1), {}])
def test_the_first_tokens_say_little(kw):
    """Rows that begin with thousands of masked tokens, or whose largest logits are hundreds of nats above the first ones."""
    say(f"first tokens {kw}")
    rng = np.random.default_rng(13)
    z = logits_of(rng, 5, 30000, 2.0)
    z[0, :4096] = -torch.inf
    z[1, :12000] = -torch.inf
    z[2] = -torch.inf
    z[2, 29990:] = torch.arange(10).float() / 4
    z[3, 20000:20050] += 300
    z[4, 29999] += 5000
    check(z, rng.random(5), {k: [v] * 5 for k, v in kw.items()}, most_unsafe=0.3)


def test_more_rows_than_go_together():
    rng = np.random.default_rng(14)
    R = 2100
    z = logits_of(rng, R, 260, 2.0)
    kw = dict(temperature=rng.choice([0.0, 0.5, 1.0], R), top_k=rng.choice([0, 1, 20], R), top_p=rng.choice([0.5, 0.9, 1.0], R),
              min_p=rng.choice([0.0, 0.02], R))
    check(z, rng.random(R), {k: list(v) for k, v in kw.items()})


@pytest.mark.parametrize("dtype", ["fp32", "fp16"])
def test_rows_alone_are_the_same_bits(dtype):
    """However a row is divided between workgroups."""
    rng = np.random.default_rng(15)
    R, V = 1024, 70000
    z = torch.randn(R, V, device="cuda", generator=torch.Generator(device="cuda").manual_seed(3)).to(T[dtype])
    u = rng.random(R)
    kw = dict(temperature=list(rng.choice([0.5, 1.0], R)), top_k=list(rng.choice([0, 40, 9000], R)),
              top_p=list(rng.choice([0.6, 1.0], R)), min_p=list(rng.choice([0.0, 0.01], R)))
    token, logp = run(z, u, kw)
    for r in range(0, R, 41):
        t, p = run(z[r:r + 1], u[r:r + 1], {k: v[r:r + 1] for k, v in kw.items()})
        assert t.item() == token[r].item() and p.item() == logp[r].item(), r


def test_two_calls_at_once_and_a_workspace_of_anything():
    """Two streams, and the C call with a workspace whose bytes are not zeros, twice."""
    rng = np.random.default_rng(16)
    a = archer()
    z = logits_of(rng, 64, 90000, 2.0)
    u, p = dev_f32(rng.random(64)), dev_f32([0.9] * 64)
    want = a.op_sample(z, u, top_p=p)
    streams = [torch.cuda.Stream() for _ in range(2)]
    torch.cuda.synchronize()
    got = []
    for s in streams * 3:
        with torch.cuda.stream(s):
            got.append(a.op_sample(z, u, top_p=p))
    torch.cuda.synchronize()
    for t, l in got:
        assert torch.equal(t, want[0]) and torch.equal(l, want[1])
    n = a.lib.archer_op_sample_ws_bytes(a.FP32, 64, 90000)
    ws = torch.randint(0, 256, (n + 256,), dtype=torch.uint8, device="cuda")
    guard = ws[n:].clone()
    for _ in range(2):
        token, logp = torch.zeros(64, dtype=torch.int32, device="cuda"), torch.zeros(64, device="cuda")
        assert a.lib.archer_op_sample(a.FP32, 64, 90000, z.data_ptr(), z.stride(0), -1, u.data_ptr(), None, None, p.data_ptr(), None,
                                      token.data_ptr(), logp.data_ptr(), ws.data_ptr(), n, a._raw_stream(torch.cuda.current_device())) == a.OK
        assert torch.equal(token, want[0]) and torch.equal(logp, want[1])
    assert torch.equal(ws[n:], guard)


def test_samples_of_a_prompt_are_drawn():
    """As they are used: four samples of one stored prompt; in each turn a token a sample is stored, attended from and the next
    one drawn.  Eagerly against the oracle's draw from the same logits, then the turns again as replays of one graph."""
    a = archer()
    B, hq, hkv, hd, page, n_pages, width, turns = 4, 8, 2, 128, 32, 40, 8, 6
    V, P = hq * hd, 70
    g = torch.Generator(device="cuda").manual_seed(4)
    rand = lambda *s: torch.randn(*s, device="cuda", generator=g)  # noqa: E731
    tk, tv, tq, tl = rand(V, hkv, hd).half(), rand(V, hkv, hd).half(), rand(V, hq, hd).half(), rand(V, V) * 2
    pk, pv = rand(hkv, P, hd).half(), rand(hkv, hd, P).half().transpose(1, 2)
    u = torch.rand(turns, B, device="cuda", generator=g)
    temp, top_p, top_k = dev_f32([1.0, 0.7, 1.0, 0.0]), dev_f32([0.9, 1.0, 0.8, 1.0]), dev_i32([0, 40, 100, 0])
    cache = a.Cache8.empty(n_pages, page, hkv, hd)
    ring, table = dev_i32(np.arange(n_pages)), dev_i32(np.full((B, width), -1))
    pool, refs, lens, tok, draw = dev_i32([0, n_pages]), dev_i32([0] * n_pages), dev_i32([0] * B), dev_i32([0] * B), u[0].clone()

    def begin():
        ring.copy_(dev_i32(np.arange(n_pages)))
        table.fill_(-1)
        refs.zero_()
        pool.copy_(dev_i32([0, n_pages]))
        p = a.pages_plan(dev_i32([0] * B), dev_i32([P] + [0] * (B - 1)), page, table, ring, pool, refs, P, table_out=table, refs_out=refs)
        pool.copy_(p.pool)
        a.cache8_write(cache, table, dev_i32([0] * B), p.row_off, pk, pv)
        _, st = a.pages_fork(dev_i32([0] * 3), dev_i32([1, 2, 3]), dev_i32([P] * 3), page, table, refs, refs_out=refs)
        assert p.status.item() == 0 and st.item() == 0
        lens.fill_(P)
        tok.copy_(dev_i32([5, 5, 5, 6]))

    def turn():
        new = lens + 1
        p = a.pages_plan(lens, new, page, table, ring, pool, refs, B, table_out=table, refs_out=refs)
        a.pages_copy(cache.data, p.copy_src, p.copy_dst)
        i = tok.long()
        a.cache8_write(cache, table, lens, p.row_off, tk[i].transpose(0, 1).contiguous(), tv[i].transpose(0, 1).contiguous())
        O = a.op_attention_cache8(tq[i].transpose(0, 1).contiguous(), cache, table, new, width * page)
        logits = O.float() * 4 + tl[i]
        t, lp = a.op_sample(logits, draw, temperature=temp, top_k=top_k, top_p=top_p, exclude=V - 1)
        pool.copy_(p.pool)
        lens.copy_(new)
        tok.copy_(t)
        return t, lp, logits, p.status

    begin()
    eager, unsafe = [], 0
    for n in range(turns):
        draw.copy_(u[n])
        t, lp, logits, st = turn()
        eager.append((t, lp, logits))
        assert st.item() == 0
        for b in range(B):
            kw = dict(temperature=float(temp[b]), top_k=int(top_k[b]), top_p=float(top_p[b]), exclude=V - 1)
            host, x = logits[b].cpu().numpy(), float(u[n, b])
            want = osm.sample(host, x, **kw)
            if not osm.safe(host, x, **kw):
                unsafe += 1
                continue
            assert t[b].item() == want[0] and abs(lp[b].item() - want[1]) <= 2.0**-24 * abs(want[1]) + 2.0**-27
    assert unsafe <= 1
    # the samples' own pages: the shared ones are held by all
    full = P // page
    assert (refs[table[:, :full].long()] == B).all() and len(set(table[:, full].tolist())) == B
    # and stored are the tokens that were drawn
    k, _ = a.cache8_read(cache, (table[:, P // page] * page + P % page + 1).int())
    want = tk[eager[0][0].long()].transpose(0, 1).float()
    assert ((k.float() - want).abs() <= 2.0**-4 * want.abs() + 2.0**-9).all()      # (a scale of 1 at most: half a step of the subnormals)

    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    begin()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        out = turn()
    for again in range(2):
        begin()
        for n in range(turns):
            draw.copy_(u[n])
            graph.replay()
            torch.cuda.synchronize()
            assert out[3].item() == 0
            for x, y in zip(out, eager[n]):
                assert torch.equal(x, y), (again, n)
