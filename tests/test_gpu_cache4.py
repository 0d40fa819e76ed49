"""GPU parity of the 4-bit paged prompt cache against its oracle: page plans and
stored bytes exactly, attention within bounds derived in ``oracle/cache4.py``."""

import numpy as np
import pytest
import torch

from gpu_util import archer, dev_i32, host, say
from oracle import cache4 as oc

pytestmark = pytest.mark.gpu


def dev(x, dtype):
    return torch.from_numpy(np.ascontiguousarray(x)).to(dtype).cuda()


def new_cache(data, page, hd):
    return archer().Cache4(torch.from_numpy(np.ascontiguousarray(data)).cuda(), page, hd)


def random_bytes(rng, n_pages, heads, page, hd):
    """Pages of anything: every code, scales from tiny to NaN."""
    return rng.integers(0, 256, (n_pages, heads, oc.page_bytes(page, hd)), dtype=np.uint8)


# -- plans ---------------------------------------------------------------------------------------
def _check_plan(old, new, page, table, ring, pool, rows):
    a = archer()
    t, r = dev_i32(table), dev_i32(ring)
    want = oc.plan(old, new, page, table, ring, pool, rows)
    for _ in range(2):        # the second call repeats the first
        got = a.cache4_plan(dev_i32(old), dev_i32(new), page, t, r, dev_i32(pool), rows)
        for g, w in zip((t, r, got[0], got[1], got[2]), want[:5]):
            np.testing.assert_array_equal(g.cpu().numpy(), w)
        assert got[3].item() == want[5]
    return want


@pytest.mark.parametrize("B,page,hi,rows_over,seed", [(1, 32, 100, 0, 0), (7, 64, 700, 3, 1), (64, 256, 900, 1, 2),
                                                      (300, 32, 400, 0, 3), (4096, 32, 70, 77, 4)])
def test_plan_matches_oracle(B, page, hi, rows_over, seed):
    say(f"plan B={B} page={page}")
    rng = np.random.default_rng(seed)
    old = rng.integers(0, hi, B)
    new = np.where(rng.random(B) < 0.3, old // 3, np.where(rng.random(B) < 0.3, 0, old + rng.integers(0, 2 * page, B)))
    if B > 2:
        old[1] = new[1] = 0
        new[2] = old[2]
    have = -(-old // page)
    more = np.maximum(-(-new // page) - have, 0).sum()
    n = int(have.sum() + more + 5)
    width = int(-(-max(old.max(), new.max(), 1) // page)) + 2
    order = rng.permutation(n)
    table = rng.integers(-9, 10**6, (B, width))
    at = 0
    for b in range(B):
        table[b, :have[b]] = order[at:at + have[b]]
        at += have[b]
    head, rest = int(rng.integers(0, n)), n - at
    ring = rng.integers(-9, 10**6, n)
    ring[(head + np.arange(rest)) % n] = order[at:]
    st = _check_plan(old, new, page, table, ring, [head, rest], int(np.maximum(new - old, 0).sum()) + rows_over)[5]
    assert st == 0


@pytest.mark.parametrize("old,new,pool,rows,want", [
    ([0], [129], [0, 5], 200, 2), ([-1], [3], [0, 5], 9, 2), ([2**31 - 1], [0], [0, 5], 9, 2), ([0], [97], [0, 3], 200, 1),
    ([0], [9], [0, 5], 8, 3), ([0], [9], [5, 1], 20, 4), ([0], [9], [-1, 1], 20, 4), ([0], [9], [0, 6], 20, 4),
    ([64], [0], [0, 4], 0, 4), ([0], [0], [0, 0], 0, 0), ([128], [128], [0, 0], 0, 0),
])
def test_plan_refusals_change_nothing(old, new, pool, rows, want):
    assert _check_plan(old, new, 32, np.arange(4)[None], np.arange(5), pool, rows)[5] == want


# -- stores --------------------------------------------------------------------------------------
def _rows(rng, H, n, hd, dtype):
    """Rows with ties, zeros, every magnitude, infinities and a NaN among them."""
    x = rng.standard_normal((H, n, hd)) * 2.0 ** rng.integers(-28, 18, (H, n, 1))
    x.flat[::7] = np.round(x.flat[::7] * 4) / 4
    ties = np.array([0.25, -0.75, 1.25, -1.75, 2.5, -3.5, 5, 7, 0, -0.0])
    x[:, ::3, :10] = ties
    x[:, ::3, 10:32] = 0.5
    if n > 1:
        x[:, 1, 32:64] = 0
        x[0, n - 1, 5], x[0, n - 1, 40] = np.inf, 1e-30
        x[-1, n // 2, hd - 1] = np.nan
    return x.astype(np.float16 if dtype == torch.float16 else np.float32)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("hd,page", [(64, 32), (128, 64), (128, 256)])
@pytest.mark.parametrize("n,order", [(1, "run"), (8, "run"), (9, "shifted"), (130, "run"), (77, "random")])
def test_write_matches_oracle(dtype, hd, page, n, order):
    say(f"write {dtype} hd={hd} page={page} n={n} {order}")
    a, H = archer(), 3
    rng = np.random.default_rng(n + hd + page)
    n_pages = -(-n // page) * 2 + 2
    with np.errstate(over="ignore"):
        K, V = _rows(rng, H, n, hd, dtype), _rows(rng, H, n, hd, dtype)
    if order == "random":
        slots = rng.permutation(n_pages * page)[:n]
        slots[3], slots[5], slots[8] = -1, n_pages * page, 2**31 - 1
    else:
        slots = np.arange(n) + (page * (n_pages - 1 - -(-n // page)) if order == "run" else 3)
    data = random_bytes(rng, n_pages, H, page, hd)
    want = oc.write(data, page, hd, K, V, slots)
    # keys and values as rows, as rows of tokens, transposed, and at odd offsets and strides
    def rows(x):
        return dev(x, dtype)

    def tokens(x):
        return dev(x.transpose(1, 0, 2), dtype).transpose(0, 1)

    def odd(x):
        t = torch.zeros(H, n + 1, hd + 3, dtype=dtype, device="cuda")
        t[:, 1:, 1:hd + 1] = dev(x, dtype)
        return t[:, 1:, 1:hd + 1]

    def transposed(x, ld, off):
        t = torch.full((H, hd, ld), float("nan"), dtype=dtype, device="cuda")
        t[:, :, off:off + n] = dev(x.transpose(0, 2, 1), dtype)
        return t[:, :, off:off + n].transpose(1, 2)
    ld = (n + 7) // 8 * 8
    for k, v in ((rows(K), rows(V)), (tokens(K), tokens(V)), (odd(K), odd(V)), (rows(K), transposed(V, ld, 0)),
                 (odd(K), transposed(V, ld + 5, 3))):
        c = new_cache(data, page, hd)
        a.cache4_write(c, k, v, dev_i32(slots))
        got = c.data.cpu().numpy()
        # by the values: the codes under a NaN scale are not specified
        k_ref, v_ref = oc.read(want, page, hd, slots)
        k_got, v_got = oc.read(got, page, hd, slots)
        np.testing.assert_array_equal(k_got, k_ref)
        np.testing.assert_array_equal(v_got, v_ref)
        # and nothing else was touched
        same = oc.write(got, page, hd, K, V, slots)
        np.testing.assert_array_equal(same, want)
        # what the library reads is what the bytes say
        kr, vr = a.cache4_read(c, dev_i32(slots), dtype)
        np.testing.assert_array_equal(host(kr), k_ref)
        np.testing.assert_array_equal(host(vr), v_ref)


@pytest.mark.parametrize("dtype", [torch.float16, torch.float32])
@pytest.mark.parametrize("hd", [64, 128])
def test_read_of_any_bytes(dtype, hd):
    """Every code and the scales a store makes, repeated slots, slots outside the cache."""
    rng = np.random.default_rng(5)
    page, H = 32, 2
    data = random_bytes(rng, 4, H, page, hd)
    sc = data[:, :, page * hd:]
    sc[...] = np.where(rng.random(sc.shape) < 0.05, 255, rng.integers(104, 141, sc.shape))
    slots = np.concatenate([rng.integers(0, 4 * page, 60), [-1, 4 * page, 5, 5, 2**31 - 1, -2**31], np.arange(24, 41)])
    k, v = archer().cache4_read(new_cache(data, page, hd), dev_i32(slots), dtype)
    k_ref, v_ref = oc.read(data, page, hd, slots)
    np.testing.assert_array_equal(host(k), k_ref)
    np.testing.assert_array_equal(host(v), v_ref)


def test_no_rows():
    a = archer()
    c = a.Cache4.empty(2, 32, 2, 64)
    none = dev_i32([])
    a.cache4_write(c, torch.zeros(2, 0, 64, dtype=torch.float16, device="cuda"),
                   torch.zeros(2, 0, 64, dtype=torch.float16, device="cuda"), none)
    k, v = a.cache4_read(c, none)
    assert k.shape == v.shape == (2, 0, 64) and not c.data.any()


# -- attention -----------------------------------------------------------------------------------
class Case:
    """A batch over a cache whose unused bytes are anything (NaN scales among them)."""

    def __init__(self, dtype, lens, G, hq, hkv, hd, page, fresh, resp=None, seed=0, q_scale=2.0, share=False,
                 k_scale=1.0):
        rng = np.random.default_rng(seed)
        self.dtype, self.lens, self.G, self.hq, self.hkv, self.hd, self.page = dtype, lens, G, hq, hkv, hd, page
        B = len(lens)
        np_t = np.float16 if dtype == torch.float16 else np.float32
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + 2
        order = rng.permutation(n_pages)
        width = max(need + [1]) + 1
        self.table = rng.integers(-5, 10**6, (B, width))      # what lies past a sequence's pages is not read
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        if share:                                             # two sequences with the same first page
            self.table[1, 0] = self.table[0, 0]
        self.data = random_bytes(rng, n_pages, hkv, page, hd)
        self.K, self.V = [], []
        for b, n in enumerate(lens):
            slots = [self.table[b, p // page] * page + p % page for p in range(n)]
            self.data = oc.write(self.data, page, hd, rng.standard_normal((hkv, n, hd)) * k_scale,
                                 rng.standard_normal((hkv, n, hd)), slots)
        for b, n in enumerate(lens):
            k, v = oc.read(self.data, page, hd, [self.table[b, p // page] * page + p % page for p in range(n)])
            self.K.append(k), self.V.append(v)
        self.Q = (rng.standard_normal((hq, B * G, hd)) * q_scale).astype(np_t)
        self.resp = resp
        self.stride, self.ld2, self.K2, self.V2 = (G + 7) // 8 * 8, 0, None, None
        rows = resp if resp is not None else [G] * B
        if fresh:
            self.ld2 = B * self.stride
            self.K2 = np.full((hkv, self.ld2, hd), np.nan, np_t)
            self.V2 = np.full((hkv, hd, self.ld2), np.nan, np_t)
            for b in range(B):
                s = slice(b * self.stride, b * self.stride + rows[b])
                self.K2[:, s] = rng.standard_normal((hkv, rows[b], hd)) * k_scale
                self.V2[:, :, s] = rng.standard_normal((hkv, hd, rows[b]))
        self.rows = rows

    def run(self, max_cached=None, data=None, table=None, fill=7.0):
        a = archer()
        O = torch.full((len(self.lens) * self.G, self.hq * self.hd), fill, device="cuda",
                       dtype=torch.bfloat16 if self.dtype == torch.float16 else torch.float32)
        d = lambda x: None if x is None else dev(x, self.dtype)  # noqa: E731
        return a.op_attention_cache4(
            d(self.Q), new_cache(self.data if data is None else data, self.page, self.hd),
            dev_i32(self.table if table is None else table), dev_i32(self.lens),
            max(self.lens) if max_cached is None else max_cached, K2=d(self.K2), Vt2=d(self.V2), fresh_stride=self.stride,
            resp_len=None if self.resp is None else dev_i32(self.resp), O=O)

    def keys(self, b, kh):
        k, v = self.K[b][kh], self.V[b][kh]
        if self.K2 is not None:
            s = slice(b * self.stride, b * self.stride + self.rows[b])
            k = np.concatenate([k, self.K2[kh, s].astype(np.float64)])
            v = np.concatenate([v, self.V2[kh, :, s].astype(np.float64).T])
        return k, v

    def check(self, O, fill=7.0, rows_of=None):
        O = host(O).reshape(len(self.lens), self.G, self.hq, self.hd)
        worst = 0.0
        for b in range(len(self.lens)):
            r = self.rows[b]
            assert (O[b, r:] == fill).all(), "rows past the response were written"
            pick = np.arange(r) if rows_of is None else rows_of[rows_of < r]
            if len(pick) == 0:
                continue
            for h in range(self.hq):
                k, v = self.keys(b, h // (self.hq // self.hkv))
                q = self.Q[h, b * self.G + pick].astype(np.float64)
                ref, A, qk, smax = oc.attention(q, k, v)
                if len(k) == 0:
                    assert (O[b, pick, h] == 0).all()
                    continue
                tol = oc.attention_bound(ref, A, qk, smax, len(k), self.hd, np.abs(v).max(), self.dtype == torch.float16)
                err = np.abs(O[b, pick, h] - ref)
                assert (err <= tol).all(), (b, h, float((err / tol).max()))
                worst = max(worst, float((err / tol).max()) if err.size else 0.0)
        return worst


F16, F32 = torch.float16, torch.float32
LENS = [0, 1, 31, 32, 33, 64, 65, 100, 257]


@pytest.mark.parametrize("dtype,lens,G,hq,hkv,hd,page,fresh,resp", [
    # single tokens: every remainder, an empty cache; with and without a fresh key
    (F16, LENS, 1, 4, 4, 128, 32, False, None),
    (F16, LENS, 1, 14, 2, 128, 64, True, None),
    (F16, LENS, 1, 4, 2, 64, 256, False, None),
    (F32, LENS, 1, 6, 2, 128, 32, True, None),
    (F32, LENS, 1, 4, 4, 64, 32, False, None),
    # short blocks: one and several column blocks, ragged responses, an empty response
    (F16, [40, 0, 130], 5, 7, 1, 128, 32, True, [5, 1, 3]),
    (F16, [40, 3, 130, 64], 9, 4, 2, 64, 64, True, [9, 0, 8, 1]),
    (F32, [40, 3, 130, 64], 9, 4, 2, 64, 64, True, [9, 0, 8, 1]),
    (F16, [0, 0], 16, 4, 1, 128, 32, True, [16, 11]),      # only fresh keys
    (F16, [0, 0], 3, 4, 1, 128, 32, False, None),          # no keys at all
    (F32, [0, 0], 3, 4, 1, 128, 32, False, None),
    (F16, [33, 70], 40, 2, 2, 128, 64, True, [40, 33]),
    # responses of a denoising step
    (F16, [100, 1, 0], 70, 2, 1, 128, 64, True, [70, 64, 65]),
    (F16, [513], 256, 2, 2, 128, 128, True, None),
    (F16, [300, 64], 130, 3, 1, 64, 32, True, [129, 130]),
    (F16, [700], 264, 1, 1, 128, 256, False, None),
    (F32, [100, 64], 70, 2, 1, 128, 64, True, [70, 3]),
])
def test_attention_matches_oracle(dtype, lens, G, hq, hkv, hd, page, fresh, resp):
    say(f"attention {dtype} lens={lens} G={G} hq={hq} hkv={hkv} hd={hd} page={page} fresh={fresh} resp={resp}")
    c = Case(dtype, lens, G, hq, hkv, hd, page, fresh, resp, seed=G + hd)
    say(f"  worst error / bound {c.check(c.run()):.3f}")


@pytest.mark.parametrize("dtype,lens,G,hq,hkv,hd,page,fresh", [
    (F16, [5000], 1, 8, 2, 128, 64, False),          # one sequence over many splits
    (F16, [3001, 5, 0, 1500], 1, 7, 1, 128, 32, True),   # splits of unequal sequences, some of one step
    (F32, [2500], 2, 4, 1, 64, 128, True),
    (F16, [4100], 100, 2, 2, 128, 64, True),
    (F16, [2047, 64, 0], 64, 2, 1, 64, 64, True),
    # 1024 rows and more, few chunks
    (F16, [3000], 32, 32, 16, 64, 32, False),
    (F16, [3300], 32, 32, 8, 128, 64, True),
    (F32, [4000], 32, 32, 32, 64, 32, True),
])
def test_split_attention_matches_oracle(dtype, lens, G, hq, hkv, hd, page, fresh):
    say(f"split attention {dtype} lens={lens} G={G} hq={hq} hkv={hkv}")
    c = Case(dtype, lens, G, hq, hkv, hd, page, fresh, seed=3)
    n = archer().lib.archer_op_attention_cache4_ws_bytes(0 if dtype == F16 else 1, len(lens), G, hq, hkv, hd, max(lens),
                                                         int(fresh))
    assert n > 0, "the case is meant to split"
    rows = None if G < 10 else np.arange(0, G, 7)
    say(f"  worst error / bound {c.check(c.run(), rows_of=rows):.3f}")


def test_split_of_more_sequences_than_lanes():
    """150 sequences of up to 1000 keys under a loose bound: chunks of 8 steps, found by a scan in three parts."""
    c = Case(F16, [(137 * b) % 1001 for b in range(150)], 1, 2, 1, 64, 32, True, seed=4)
    assert archer().lib.archer_op_attention_cache4_ws_bytes(0, 150, 1, 2, 1, 64, 10**6, 1) > 0
    say(f"  worst error / bound {c.check(c.run(max_cached=10**6)):.3f}")


@pytest.mark.parametrize("G", [1, 80])
def test_peaked_scores(G):
    """Score spread of about 30: one key takes nearly everything."""
    c = Case(F16, [300, 41], G, 4, 2, 128, 32, True, seed=9, q_scale=30.0)
    c.check(c.run())


@pytest.mark.parametrize("G", [1, 80])
def test_shared_pages_and_max_cached(G):
    c = Case(F16, [200, 90], G, 4, 2, 128, 64, False, seed=11, share=True)
    c.check(c.run())
    c.check(c.run(max_cached=1000))       # a looser bound on the lengths
    # a tighter one cuts the longer sequence
    c.K[0], c.V[0] = c.K[0][:, :150], c.V[0][:, :150]
    O = c.run(max_cached=150)
    c.check(O)


@pytest.mark.parametrize("G", [1, 80])
@pytest.mark.parametrize("page", [32, 128])
def test_pages_outside_the_cache_are_left_out(G, page):
    c = Case(F16, [page * 3 + 5], G, 2, 1, 128, page, True, seed=12)
    t = c.table.copy()
    t[0, 1] = len(c.data)
    t[0, 3] = -1
    keep = np.r_[0:page, 2 * page:3 * page]
    c.K[0], c.V[0] = c.K[0][:, keep], c.V[0][:, keep]
    c.check(c.run(table=t))
    # every page bad and no fresh keys: no key, zeros
    c.K2 = c.V2 = None
    c.K[0], c.V[0] = c.K[0][:, :0], c.V[0][:, :0]
    c.check(c.run(table=np.full_like(t, -1)))


@pytest.mark.parametrize("G", [1, 80])
def test_a_nan_key_stays_with_its_head(G):
    c = Case(F16, [100, 100], G, 4, 2, 128, 64, True, seed=13)
    ref = host(c.run())
    page, pos = divmod(77, 64)
    ks = oc.locate(64, 128)[3]
    data = c.data.copy()
    data[c.table[0, page], 1, ks[pos, 2]] = oc.NAN_SCALE
    got = host(c.run(data=data))
    O, R = got.reshape(2, G, 4, 128), ref.reshape(2, G, 4, 128)
    assert np.isnan(O[0, :, 2:]).all()
    np.testing.assert_array_equal(O[0, :, :2], R[0, :, :2])
    np.testing.assert_array_equal(O[1], R[1])


@pytest.mark.parametrize("dtype,G", [(F16, 1), (F16, 80), (F32, 3)])
def test_same_bits_again_and_on_another_stream(dtype, G):
    c = Case(dtype, [3000, 77], G, 4, 2, 128, 64, True, seed=14)
    a = c.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = c.run()
    s.synchronize()
    assert torch.equal(a, b)


# -- columns enough for the whole GPU: 2^15 of 128 dimensions, 2^16 of 64 -------------------------
SOME = np.r_[0, 1, 15:18, 31, 32, 63, 64, np.arange(97, 1024, 101), 127, 128, 255, 511]


@pytest.mark.parametrize("lens,G,hq,hkv,hd,page,fresh,resp", [
    # a workgroup's waves all in use, some, and in the second one few
    ([0, 1, 63, 64, 65, 130, 257, 700], 512, 8, 8, 128, 32, True, [512, 1, 0, 33, 300, 512, 257, 100]),
    ([191, 192, 193, 0] * 4, 160, 14, 2, 128, 64, False, None),
    (list(range(41)), 100, 8, 8, 128, 256, True, None),
    ([2100, 40, 0, 1], 1024, 8, 8, 128, 128, True, [1024, 1000, 1024, 7]),       # more than 32 tiles
    ([0] * 8, 512, 8, 8, 128, 32, False, None),
    ([(37 * b) % 150 for b in range(70)], 64, 8, 4, 128, 32, True, None),      # more sequences than a wave has lanes
    ([0, 31, 33, 70, 200, 1, 64, 9] * 2, 256, 16, 4, 64, 32, True, [256, 255, 0, 1, 17, 128, 200, 64] * 2),
    ([500, 20, 0, 300] * 4, 512, 8, 8, 64, 256, False, None),
])
def test_wide_attention_matches_oracle(lens, G, hq, hkv, hd, page, fresh, resp):
    say(f"wide attention lens={lens} G={G} hq={hq} hkv={hkv} hd={hd} page={page} fresh={fresh}")
    c = Case(F16, lens, G, hq, hkv, hd, page, fresh, resp, seed=30 + hd)
    say(f"  worst error / bound {c.check(c.run(), rows_of=SOME):.3f}")


WIDE = [(8, 4, 128), (16, 8, 64)]       # hq, hkv, hd; of 8 sequences and 512 rows
WIDE_LENS = [300, 41, 0, 90, 64, 128, 7, 200]


@pytest.mark.parametrize("hq,hkv,hd", WIDE)
def test_wide_peaked_scores(hq, hkv, hd):
    c = Case(F16, WIDE_LENS, 512, hq, hkv, hd, 32, True, seed=31, q_scale=30.0)
    c.check(c.run(), rows_of=SOME)


@pytest.mark.parametrize("hq,hkv,hd", WIDE)
@pytest.mark.parametrize("q_scale,k_scale", [(2.0**-17, 2.0**12), (2.0**11, 2.0**-10)])
def test_wide_small_and_large_queries(hq, hkv, hd, q_scale, k_scale):
    c = Case(F16, WIDE_LENS, 512, hq, hkv, hd, 64, True, seed=35, q_scale=q_scale, k_scale=k_scale)
    c.check(c.run(), rows_of=SOME)


@pytest.mark.parametrize("hq,hkv,hd", WIDE)
def test_wide_bad_pages_and_max_cached(hq, hkv, hd):
    c = Case(F16, WIDE_LENS, 512, hq, hkv, hd, 64, False, seed=32, share=True)
    c.check(c.run(max_cached=5000), rows_of=SOME)
    t = c.table.copy()
    t[0, 1], t[0, 4], t[1, 0] = len(c.data), -1, 2**31 - 1
    K, V = list(c.K), list(c.V)
    keep = np.r_[0:64, 128:256]
    c.K[0], c.V[0], c.K[1], c.V[1] = K[0][:, keep], V[0][:, keep], K[1][:, :0], V[1][:, :0]
    c.check(c.run(table=t), rows_of=SOME)
    # a bound below some lengths
    c.K, c.V = [k[:, :100] for k in K], [v[:, :100] for v in V]
    c.check(c.run(max_cached=100), rows_of=SOME)


@pytest.mark.parametrize("hq,hkv,hd", WIDE)
def test_wide_nan_and_infinity_stay_in_place(hq, hkv, hd):
    c = Case(F16, WIDE_LENS, 512, hq, hkv, hd, 64, True, seed=33)
    ref = host(c.run()).reshape(8, 512, hq, hd)
    page, pos = divmod(77, 64)
    data = c.data.copy()
    data[c.table[0, page], 1, oc.locate(64, hd)[3][pos, 1]] = oc.NAN_SCALE
    c.Q[1, 3 * 512 + 5, 9] = np.inf                # sequence 3, row 5, head 1
    c.Q[0, 3 * 512 + 6, 0] = np.nan
    got = host(c.run(data=data)).reshape(8, 512, hq, hd)
    want = np.zeros(got.shape[:3], bool)
    want[0, :, 2:4] = want[3, 5, 1] = want[3, 6, 0] = True
    assert np.isnan(got[want]).all()
    np.testing.assert_array_equal(got[~want], ref[~want])


@pytest.mark.parametrize("hq,hkv,hd", WIDE)
def test_wide_same_bits_again_and_on_another_stream(hq, hkv, hd):
    c = Case(F16, WIDE_LENS, 512, hq, hkv, hd, 64, True, seed=34)
    a = c.run()
    torch.cuda.synchronize()
    s = torch.cuda.Stream()
    with torch.cuda.stream(s):
        b = c.run()
    s.synchronize()
    assert torch.equal(a, b)


# -- far pages, other lengths than the table's, several calls at once ------------------------------
@pytest.mark.parametrize("G", [1, 20, 1040])
def test_pages_beyond_4_gib(G):
    """The same tokens in the first pages and in the last ones of a cache of 5 GB: the same bits."""
    a = archer()
    page, hkv, hd, n = 256, 8, 128, 700
    n_pages = 5 * 10**9 // (hkv * page * (hd + hd // 16))
    data = torch.empty(n_pages, hkv, page * (hd + hd // 16), dtype=torch.uint8, device="cuda")
    data[:8] = 255
    data[-8:] = 255
    c = a.Cache4(data, page, hd)
    g = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.randn(hkv, n, hd, generator=g, device="cuda").half() for _ in range(2))
    Q = torch.randn(hkv, 4 * G, hd, generator=g, device="cuda").half()
    res = []
    for pages in ([4, 1, 2], [n_pages - 1, n_pages - 6, n_pages - 3]):
        t = torch.tensor(pages, device="cuda")
        p = torch.arange(n, device="cuda")
        slots = (t[p // page] * page + p % page).int()
        a.cache4_write(c, K, V, slots)
        k, v = a.cache4_read(c, slots)
        assert torch.isfinite(k.float()).all() and torch.isfinite(v.float()).all()
        table = t.int().repeat(4, 1).contiguous()
        res.append((k, v, a.op_attention_cache4(Q, c, table, dev_i32([n, 1, 0, 511]), n)))
    for x, y in zip(*res):
        assert torch.equal(x, y)


@pytest.mark.parametrize("G", [1, 80])
def test_lengths_beyond_the_table_are_cut(G):
    """A cached length (and max_cached) past the table's last page reads what the table has."""
    c = Case(F16, [128, 96], G, 4, 2, 128, 32, True, seed=40)
    c.table = c.table[:, :4].copy()
    c.table[1, 3] = -1                             # sequence 1 has three pages
    c.lens = [10**6, 2**31 - 1]
    c.check(c.run(max_cached=2**31 - 1))


def test_several_calls_at_once():
    """Split attentions (each with its own workspace) and stores on three streams."""
    cases = [Case(F16, [5000, 60], 1, 8, 2, 128, 64, False, seed=50 + i) for i in range(3)]
    alone = [c.run() for c in cases]
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in cases]
    for _ in range(3):
        out = []
        for c, s in zip(cases, streams):
            with torch.cuda.stream(s):
                out.append(c.run())
        torch.cuda.synchronize()
        for x, y in zip(alone, out):
            assert torch.equal(x, y)


# -- as they are used ----------------------------------------------------------------------------
@pytest.mark.parametrize("dtype,hq,hkv,hd,page", [(F16, 4, 2, 128, 32), (F32, 2, 2, 64, 64)])
def test_plan_store_attend_rollback(dtype, hq, hkv, hd, page):
    """A batch lives: prompts arrive, tokens follow, one request rolls back, one finishes, another takes its pages."""
    a = archer()
    rng = np.random.default_rng(21)
    np_t = np.float16 if dtype == F16 else np.float32
    B, n_pages, width = 3, 12, 8
    cache = a.Cache4.empty(n_pages, page, hkv, hd)
    table, ring, pool = dev_i32(np.full((B, width), -1)), dev_i32(np.arange(n_pages)), dev_i32([0, n_pages])
    old = np.zeros(B, int)
    K = [np.zeros((hkv, 0, hd)) for _ in range(B)]
    V = [np.zeros((hkv, 0, hd)) for _ in range(B)]
    for turn, new in enumerate(([70, 33, 0], [71, 34, 0], [40, 35, 5], [41, 0, 6], [100, 64, 7])):
        rows = int(np.maximum(np.array(new) - old, 0).sum())
        pool, off, slots, st = a.cache4_plan(dev_i32(old), dev_i32(new), page, table, ring, pool, rows + 3)
        k = rng.standard_normal((hkv, rows + 3, hd)).astype(np_t)
        v = rng.standard_normal((hkv, rows + 3, hd)).astype(np_t)
        vt = dev(v.transpose(0, 2, 1), dtype).transpose(1, 2)
        a.cache4_write(cache, dev(k, dtype), vt, slots)
        at = off.cpu().numpy()
        assert st.item() == 0
        for b in range(B):
            K[b] = np.concatenate([K[b][:, :new[b]], oc.stored(k[:, at[b]:at[b + 1]])], 1)
            V[b] = np.concatenate([V[b][:, :new[b]], oc.stored(v[:, at[b]:at[b + 1]])], 1)
            assert K[b].shape[1] == new[b]
        old = np.array(new)
        q = (rng.standard_normal((hq, B, hd)) * 2).astype(np_t)
        O = host(a.op_attention_cache4(dev(q, dtype), cache, table, dev_i32(new), max(new))).reshape(B, hq, hd)
        for b in range(B):
            for h in range(hq):
                kk, vv = K[b][h // (hq // hkv)], V[b][h // (hq // hkv)]
                ref, A, qk, smax = oc.attention(q[h, b:b + 1].astype(np.float64), kk, vv)
                vmax = np.abs(vv).max() if len(vv) else 0.0
                tol = oc.attention_bound(ref, A, qk, smax, len(kk), hd, vmax, dtype == F16)
                assert (np.abs(O[b, h] - ref[0]) <= tol[0]).all(), (turn, b, h)
    free = pool.cpu().numpy()
    held = sum(oc.pages(n, page) for n in new)
    assert free[1] == n_pages - held
    ids = [int(x) for b in range(B) for x in table[b, :oc.pages(new[b], page)]]
    ids += [int(ring[(free[0] + i) % n_pages]) for i in range(free[1])]
    assert sorted(ids) == list(range(n_pages))            # every page is somewhere, once


def test_captured_turn_replays():
    """Plan, store and attention of one token per sequence in one graph, replayed with other lengths and
    inputs, with eager work between the replays."""
    a = archer()
    rng = np.random.default_rng(22)
    B, hq, hkv, hd, page, n_pages, width = 4, 8, 2, 128, 32, 40, 20
    lens = dev_i32([0, 31, 32, 200])
    data = torch.from_numpy(random_bytes(rng, n_pages, hkv, page, hd)).cuda()
    data[:, :, page * hd:] = 125
    cache = a.Cache4(data, page, hd)
    table = dev_i32(np.arange(B * width).reshape(B, width) % n_pages)
    ring, pool = dev_i32(np.arange(n_pages)[::-1]), dev_i32([3, 20])
    k = torch.randn(hkv, B, hd, device="cuda").half()
    v = torch.randn(hkv, B, hd, device="cuda").half()
    q = torch.randn(hq, B, hd, device="cuda").half()
    O = torch.zeros(B, hq * hd, device="cuda", dtype=torch.bfloat16)

    def turn():
        new = lens + 1
        _, _, slots, st = a.cache4_plan(lens, new, page, table, ring, pool, B)
        a.cache4_write(cache, k, v, slots)
        a.op_attention_cache4(q, cache, table, new, 600, O=O)
        return slots, st

    turn()
    torch.cuda.synchronize()
    side = torch.cuda.Stream()
    g = torch.cuda.CUDAGraph()
    with torch.cuda.graph(g, stream=side):
        got = turn()
    for i in range(4):
        lens.copy_(dev_i32([i, 31 + i, 64 - i, 500 + i]))
        for t in (k, v, q):
            t.copy_(torch.randn_like(t))
        before = data.clone(), table.clone()
        g.replay()
        torch.cuda.synchronize()
        res = O.clone(), data.clone(), table.clone(), got[0].clone(), got[1].clone()
        data.copy_(before[0])
        table.copy_(before[1])
        O.zero_()
        s, st = turn()
        for x, y in zip(res, (O, data, table, s, st)):
            assert torch.equal(x, y)
        assert res[4].item() == 0 and torch.isfinite(res[0].float()).all()


def test_two_graphs_of_one_pool():
    """Two captured attentions that share their memory pool, replayed in turn with other lengths, with eager calls
    between: one whose sequences are cut (it needs a workspace), one of the row kernel."""
    a = archer()
    cases = [Case(F16, [5000, 60], 1, 8, 2, 128, 64, False, seed=60), Case(F16, WIDE_LENS, 512, 8, 4, 128, 64, True, seed=61)]
    args, outs, graphs = [], [], []
    for c in cases:
        d = lambda x: None if x is None else dev(x, F16)  # noqa: E731
        kw = dict(K2=d(c.K2), Vt2=d(c.V2), fresh_stride=c.stride)
        args.append(((d(c.Q), new_cache(c.data, c.page, c.hd), dev_i32(c.table)), dev_i32(c.lens), max(c.lens), kw))
        outs.append(torch.zeros(len(c.lens) * c.G, c.hq * c.hd, device="cuda", dtype=torch.bfloat16))

    def call(i, O):
        first, lens, most, kw = args[i]
        a.op_attention_cache4(*first, lens, most, O=O, **kw)

    for i in range(2):
        call(i, outs[i])
    torch.cuda.synchronize()
    for i in range(2):
        g = torch.cuda.CUDAGraph()
        with torch.cuda.graph(g, pool=graphs[0].pool() if graphs else None):
            call(i, outs[i])
        graphs.append(g)
    for turn in range(3):
        for c, x in zip(cases, args):
            x[1].copy_(dev_i32([max(0, n - 7 * turn) for n in c.lens]))
        for g in graphs:
            g.replay()
        got = [O.clone() for O in outs]
        for i in range(2):
            outs[i].zero_()
            call(i, outs[i])
            assert torch.equal(got[i], outs[i])


# -- the binding's refusals ----------------------------------------------------------------------
def test_binding_refusals():
    a = archer()
    c = a.Cache4.empty(4, 32, 2, 64)
    h = lambda *s: torch.zeros(*s, dtype=torch.float16, device="cuda")  # noqa: E731
    i = dev_i32
    bad = [
        lambda: a.Cache4(torch.zeros(4, 2, 100, dtype=torch.uint8, device="cuda"), 32, 64),
        lambda: a.Cache4(torch.zeros(4, 2, 32 * 68, dtype=torch.uint8), 32, 64),
        lambda: a.Cache4(torch.zeros(4, 2, 32 * 68, dtype=torch.int8, device="cuda"), 32, 64),
        lambda: a.Cache4(torch.zeros(4, 2, 16 * 68, dtype=torch.uint8, device="cuda"), 16, 64),
        lambda: a.cache4_write(c, h(2, 3, 64), h(2, 3, 64), i([0, 1])),
        lambda: a.cache4_write(c, h(2, 3, 64), h(2, 3, 64).float(), i([0, 1, 2])),
        lambda: a.cache4_write(c, h(2, 64, 3).transpose(1, 2), h(2, 3, 64), i([0, 1, 2])),
        lambda: a.cache4_write(c, h(2, 3, 64), h(2, 3, 128)[:, :, ::2], i([0, 1, 2])),
        lambda: a.cache4_write(c, h(2, 3, 64), h(2, 3, 64), i([0, 1, 2]).long()),
        lambda: a.cache4_write(c, h(2, 3, 64).bfloat16(), h(2, 3, 64).bfloat16(), i([0, 1, 2])),
        lambda: a.cache4_read(c, i([0, 1, 2]).cpu()),
        lambda: a.cache4_read(c, i([0, 1]), torch.bfloat16),
        lambda: a.cache4_plan(i([0]), i([1, 2]), 32, i([[0, 0]]), i([0]), i([0, 1]), 4),
        lambda: a.cache4_plan(i([0]), i([1]), 32, i([0, 0]), i([0]), i([0, 1]), 4),
        lambda: a.cache4_plan(i([0]), i([1]), 32, i([[0, 0, 0]])[:, ::2], i([0]), i([0, 1]), 4),
        lambda: a.cache4_plan(i([0]), i([1]), 32, i([[0, 0]]), i([0]), i([0, 1, 2]), 4),
        lambda: a.cache4_plan(i([0]), i([1]), 32, i([[0, 0]]), i([0]), i([0, 1]), -1),
        lambda: a.op_attention_cache4(h(2, 3, 64), c, i([[0], [1]]), i([1, 1]), 9),
        lambda: a.op_attention_cache4(h(3, 2, 64), c, i([[0], [1]]), i([1, 1]), 9),
        lambda: a.op_attention_cache4(h(2, 2, 128), c, i([[0], [1]]), i([1, 1]), 9),
        lambda: a.op_attention_cache4(h(2, 2, 64), c, i([[0], [1]]), i([1, 1, 1]), 9),
        lambda: a.op_attention_cache4(h(2, 2, 64), c, i([[0], [1]]), i([1, 1]), 9, K2=h(2, 16, 64)),
        lambda: a.op_attention_cache4(h(2, 2, 64), c, i([[0], [1]]), i([1, 1]), 9, K2=h(2, 16, 64), Vt2=h(2, 64, 16),
                                      fresh_stride=16),
        lambda: a.op_attention_cache4(h(2, 2, 64), c, i([[0], [1]]), i([1, 1]), 9, O=h(2, 128)),
        lambda: a.op_attention_cache4(h(2, 2, 64).cpu(), c, i([[0], [1]]), i([1, 1]), 9),
    ]
    for n, f in enumerate(bad):
        with pytest.raises(a.ArcherError):
            f()
            say(f"call {n} was not refused")
