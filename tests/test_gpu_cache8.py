"""GPU parity of the 8-bit paged prompt cache against its oracle: stored bytes exactly, attention within the
bounds derived in ``oracle/cache4.py`` (without the row kernel's query terms, which these kernels have not)."""

import numpy as np
import pytest
import torch

import test_gpu_cache4 as c4
from gpu_util import archer, dev_i32, host, say
from oracle import cache4 as oc
from oracle import cache8 as o8
from test_gpu_cache4 import F16, F32, LENS, SOME, WIDE_LENS, dev

pytestmark = pytest.mark.gpu


def new_cache(data, page, hd):
    return archer().Cache8(torch.from_numpy(np.ascontiguousarray(data)).cuda(), page, hd)


def random_bytes(rng, n_pages, heads, page, hd):
    """Pages of anything: every code, NaN among them; scales from tiny to huge."""
    return rng.integers(0, 256, (n_pages, heads, o8.page_bytes(page, hd)), dtype=np.uint8)


# -- stores --------------------------------------------------------------------------------------
def _rows(rng, H, n, hd, dtype):
    """Rows with ties, zeros, subnormal codes, saturation, infinities and a NaN among them."""
    x = rng.standard_normal((H, n, hd)) * 2.0 ** rng.integers(-26, 20, (H, n, 1))
    x[:, ::2] = rng.standard_normal((H, (n + 1) // 2, hd)) * 4
    x.flat[::7] = np.round(x.flat[::7] * 4) / 4
    ties = np.array([17, 19, 0.53125, -0.59375, 2.0**-9, 3 * 2.0**-10, 2.0**-10, 5 * 2.0**-11, 0, -0.0, 448, 432, 416, -440])
    x[:, n // 2, :14] = ties
    if n > 40:
        x[0, n - 1, 5], x[-1, 33, hd - 1] = np.inf, np.nan
        x[:, 36:38] = 0
    return x.astype(np.float16 if dtype == F16 else np.float32)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("hd,page", [(64, 32), (128, 64), (128, 256)])
@pytest.mark.parametrize("start,count", [([0], [1]), ([0], [64]), ([31], [1]), ([5], [130]), ([64, 0, 3, 33], [70, 0, 1, 200]),
                                         ([0, 1, 2, 3, 96], [31, 32, 33, 1, 5])])
def test_write_matches_oracle(dtype, hd, page, start, count):
    say(f"write {dtype} hd={hd} page={page} {start} {count}")
    a, H, B = archer(), 3, len(start)
    rng = np.random.default_rng(sum(count) + hd + page)
    need = [-(-(s + n) // page) for s, n in zip(start, count)]
    n_pages = sum(need) + 2
    width = max(need) + 1
    order = rng.permutation(n_pages)
    table, at = rng.integers(-5, 10**6, (B, width)), 0
    for b, k in enumerate(need):
        table[b, :k] = order[at:at + k]
        at += k
    off = np.concatenate([[0], np.cumsum(count)])
    n = int(off[-1]) + 3                       # three rows of no sequence
    with np.errstate(over="ignore"):
        K, V = _rows(rng, H, n, hd, dtype), _rows(rng, H, n, hd, dtype)
    # earlier tokens: any codes, scales that a store makes
    data = random_bytes(rng, n_pages, H, page, hd)
    data[:, :, 2 * page * hd:] = rng.integers(112, 135, data[:, :, 2 * page * hd:].shape)
    want = o8.write(data, page, hd, table, start, off, K, V)

    def rows(x):
        return dev(x, dtype)

    def tokens(x):
        return dev(x.transpose(1, 0, 2), dtype).transpose(0, 1)

    def odd(x):
        t = torch.zeros(H, n + 1, hd + 3, dtype=dtype, device="cuda")
        t[:, 1:, 1:hd + 1] = dev(x, dtype)
        return t[:, 1:, 1:hd + 1]

    def transposed(x, ld, o):
        t = torch.full((H, hd, ld), float("nan"), dtype=dtype, device="cuda")
        t[:, :, o:o + n] = dev(x.transpose(0, 2, 1), dtype)
        return t[:, :, o:o + n].transpose(1, 2)
    ld = (n + 7) // 8 * 8
    nan = lambda x: np.where(x & 127 == 127, 127, x)  # noqa: E731  (a NaN has either sign)
    codes = 2 * page * hd
    for k, v in ((rows(K), rows(V)), (tokens(K), tokens(V)), (odd(K), odd(V)), (rows(K), transposed(V, ld, 0)),
                 (odd(K), transposed(V, ld + 5, 3))):
        c = new_cache(data, page, hd)
        a.cache8_write(c, dev_i32(table), dev_i32(start), dev_i32(off), k, v)
        got = c.data.cpu().numpy()
        np.testing.assert_array_equal(got[..., codes:], want[..., codes:])
        np.testing.assert_array_equal(nan(got[..., :codes]), nan(want[..., :codes]))
        # what the library reads is what the bytes say
        slots = [s for b in range(B) for s in o8.slots_of(table, page, b, range(start[b] + count[b]))] + [-1]
        kr, vr = a.cache8_read(c, dev_i32(slots), F32)
        k_ref, v_ref = o8.read(got, page, hd, slots)
        np.testing.assert_array_equal(host(kr), k_ref)
        np.testing.assert_array_equal(host(vr), v_ref)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("hd", [64, 128])
def test_read_of_any_bytes(dtype, hd):
    rng = np.random.default_rng(5)
    page, H = 32, 2
    data = random_bytes(rng, 4, H, page, hd)
    data[:, :, 2 * page * hd:] = rng.integers(112, 135, data[:, :, 2 * page * hd:].shape)
    slots = np.concatenate([rng.integers(0, 4 * page, 60), [-1, 4 * page, 5, 5, 2**31 - 1, -2**31], np.arange(24, 41)])
    k, v = archer().cache8_read(new_cache(data, page, hd), dev_i32(slots), dtype)
    for got, ref in zip((k, v), o8.read(data, page, hd, slots)):
        np.testing.assert_array_equal(host(got), ref)


@pytest.mark.parametrize("dtype", [F16, F32])
@pytest.mark.parametrize("hd,page", [(64, 32), (128, 64)])
def test_read_of_runs(dtype, hd, page):
    """Slots that follow each other from every place in a block, over pages' ends and out of the cache, and some that do not quite."""
    rng = np.random.default_rng(7)
    H, n_pages = 3, 5
    data = random_bytes(rng, n_pages, H, page, hd)
    data[:, :, 2 * page * hd:] = rng.integers(112, 135, data[:, :, 2 * page * hd:].shape)
    n = n_pages * page
    runs = [np.arange(o, o + 57) for o in range(8)] + [np.arange(n - 50, n + 9), np.arange(-9, 20), np.arange(40)[::-1], np.repeat(3, 16)]
    odd = np.arange(64)
    odd[[5, 17, 29, 63]] = [6, 16, -1, n]
    slots = np.concatenate(runs + [odd, np.arange(2 * page - 3, 2 * page + 2)])
    k, v = archer().cache8_read(new_cache(data, page, hd), dev_i32(slots), dtype)
    for got, ref in zip((k, v), o8.read(data, page, hd, slots)):
        np.testing.assert_array_equal(host(got), ref)


def test_every_fp32_rounding_of_a_scale():
    """All codes, all midpoints and their neighbours, at every scale, through a store."""
    m = o8.MAGNITUDES
    mid = (m[1:] + m[:-1]) / 2
    x = np.concatenate([m, mid, np.nextafter(mid.astype(np.float32), np.float32(np.inf)), np.nextafter(mid.astype(np.float32), np.float32(0))])
    x = np.concatenate([x, -x])
    x = np.concatenate([x, np.zeros(-len(x) % 64)])
    a = archer()
    for e in range(-15, 8):
        rows = (x * 2.0**e).astype(np.float32).reshape(1, -1, 64)
        rows = np.concatenate([rows, np.full_like(rows[:, :1], 448 * 2.0**e)], 1)[:, -32:]
        c = a.Cache8.empty(1, 32, 1, 64)
        n = rows.shape[1]
        t = dev(rows, F32)
        a.cache8_write(c, dev_i32([[0]]), dev_i32([0]), dev_i32([0, n]), t, t)
        for got in a.cache8_read(c, dev_i32(np.arange(n)), F32):
            np.testing.assert_array_equal(host(got)[0], o8.stored(rows.astype(np.float64))[0])


def test_rows_that_have_no_place_are_not_stored():
    """Pages of no cache, tokens beyond the table, a negative start, offsets beyond the rows, falling offsets."""
    a, rng, page, hd, H = archer(), np.random.default_rng(6), 32, 64, 2
    data = random_bytes(rng, 4, H, page, hd)
    with np.errstate(over="ignore"):
        K = _rows(rng, H, 100, hd, F16)
    for table, start, off, put in (
            ([[9, 1, -1]], [0], [0, 96], [(1, 32, 64)]), ([[0, 1]], [40], [0, 60], [(1, 0, 24)]), ([[0, 1]], [-1], [0, 20], []),
            ([[0, 1]], [64], [0, 20], []), ([[0], [1], [2]], [0, 0, 0], [0, 10, 300, 400], [(0, 0, 10), (1, 10, 42)]),
            ([[0], [1]], [0, 0], [0, 20, 5], [(0, 0, 20)]), ([[0, 1, 2]], [2**31 - 1], [0, 9], [])):
        c = new_cache(data, page, hd)
        k = dev(K, F16)
        a.cache8_write(c, dev_i32(table), dev_i32(start), dev_i32(off), k, k.transpose(1, 2).contiguous().transpose(1, 2))
        want = data
        for p, lo, hi in put:
            first = 8 if start == [40] else 0
            want = o8.write(want, page, hd, [[p]], [first], [0, hi - lo], K[:, lo:hi], K[:, lo:hi])
        got = c.data.cpu().numpy()
        np.testing.assert_array_equal(np.where(got & 127 == 127, 127, got), np.where(want & 127 == 127, 127, want))


def test_no_rows():
    a = archer()
    c = a.Cache8.empty(2, 32, 2, 64)
    z = torch.zeros(2, 0, 64, dtype=F16, device="cuda")
    a.cache8_write(c, dev_i32([[0]]), dev_i32([0]), dev_i32([0, 0]), z, z)
    k, v = a.cache8_read(c, dev_i32([]))
    assert k.shape == v.shape == (2, 0, 64) and not c.data.any()


@pytest.mark.parametrize("B", [64, 65, 300])
def test_write_of_many_sequences(B):
    rng = np.random.default_rng(B)
    page, hd, H = 32, 64, 1
    start, count = rng.integers(0, 40, B), rng.integers(0, 9, B)
    table = rng.permutation(2 * B).reshape(B, 2)
    off = np.concatenate([[0], np.cumsum(count)])
    K, V = (rng.standard_normal((H, off[-1], hd)).astype(np.float16) for _ in range(2))
    data = random_bytes(rng, 2 * B, H, page, hd) & 0x77          # no NaN code, so that signs are compared too
    data[:, :, 2 * page * hd:] = 120
    c = new_cache(data, page, hd)
    archer().cache8_write(c, dev_i32(table), dev_i32(start), dev_i32(off), dev(K, F16), dev(V, F16))
    np.testing.assert_array_equal(c.data.cpu().numpy(), o8.write(data, page, hd, table, start, off, K, V))


# -- attention -----------------------------------------------------------------------------------
class Case(c4.Case):
    """A batch over a cache whose unused bytes are anything (NaN codes among them)."""

    def __init__(self, dtype, lens, G, hq, hkv, hd, page, fresh, resp=None, seed=0, q_scale=2.0, share=False, k_scale=1.0):
        rng = np.random.default_rng(seed)
        self.dtype, self.lens, self.G, self.hq, self.hkv, self.hd, self.page = dtype, lens, G, hq, hkv, hd, page
        B = len(lens)
        np_t = np.float16 if dtype == F16 else np.float32
        need = [-(-n // page) for n in lens]
        n_pages = sum(need) + 2
        order = rng.permutation(n_pages)
        self.table = rng.integers(-5, 10**6, (B, max(need + [1]) + 1))
        at = 0
        for b, n in enumerate(need):
            self.table[b, :n] = order[at:at + n]
            at += n
        self.data = self._pages(rng, n_pages, k_scale)
        if share:
            self.table[1, 0] = self.table[0, 0]
        self.K, self.V = [], []
        for b, n in enumerate(lens):
            k, v = o8.read(self.data, page, hd, o8.slots_of(self.table, page, b, range(n)))
            self.K.append(k), self.V.append(v)
        # behind the last token of every sequence: anything
        keep = np.zeros((n_pages, page), bool)
        for b, n in enumerate(lens):
            for p in range(n):
                keep[self.table[b, p // page], p % page] = True
        key, value, _ = o8.locate(page, hd)
        for p, t in zip(*np.nonzero(~keep)):
            for bytes_ in (key[t], value[t]):
                self.data[p][:, bytes_] = rng.choice(np.array([127, 255, 126, 3], np.uint8), (hkv, hd))
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

    def _pages(self, rng, n_pages, k_scale):
        """Every page full of stored normal rows (in bytes at once: codes of torch, scales of the definition)."""
        page, hd, hkv = self.page, self.hd, self.hkv
        data = np.zeros((n_pages, hkv, o8.page_bytes(page, hd)), np.uint8)
        data[:, :, 2 * page * hd:] = rng.integers(0, 256, (n_pages, hkv, 16))
        at = o8.locate(page, hd)
        for i, scale in enumerate((k_scale, 1.0)):
            x = rng.standard_normal((n_pages, hkv, page // 32, 32, hd)) * scale
            top = np.abs(x).max((-1, -2))
            e = np.clip(np.ceil(np.log2(top / 448)), -15, 7)
            y = torch.from_numpy(x * 2.0 ** -e[..., None, None]).float().clamp(-448, 448).to(torch.float8_e4m3fn)
            data[:, :, at[i]] = y.view(torch.uint8).numpy().reshape(n_pages, hkv, page, hd)
            data[:, :, at[2][::32, i]] = (e + 127).astype(np.uint8)
        return data

    def run(self, max_cached=None, data=None, table=None, fill=7.0):
        O = torch.full((len(self.lens) * self.G, self.hq * self.hd), fill, device="cuda",
                       dtype=torch.bfloat16 if self.dtype == F16 else torch.float32)
        d = lambda x: None if x is None else dev(x, self.dtype)  # noqa: E731
        return archer().op_attention_cache8(
            d(self.Q), new_cache(self.data if data is None else data, self.page, self.hd),
            dev_i32(self.table if table is None else table), dev_i32(self.lens),
            max(self.lens) if max_cached is None else max_cached, K2=d(self.K2), Vt2=d(self.V2), fresh_stride=self.stride,
            resp_len=None if self.resp is None else dev_i32(self.resp), O=O)

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
                ref, A, _, smax = oc.attention(q, k, v)
                if len(k) == 0:
                    assert (O[b, pick, h] == 0).all()
                    continue
                tol = oc.attention_bound(ref, A, oc.score_sums(q, k)[0], smax, len(k), self.hd, np.abs(v).max(),
                                         self.dtype == F16, block=0)
                err = np.abs(O[b, pick, h] - ref)
                assert (err <= tol).all(), (b, h, float((err / tol).max()))
                worst = max(worst, float((err / tol).max()) if err.size else 0.0)
        return worst


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
    (F16, [3300], 32, 32, 8, 128, 64, True),         # 1024 rows and more, few chunks
])
def test_split_attention_matches_oracle(dtype, lens, G, hq, hkv, hd, page, fresh):
    say(f"split attention {dtype} lens={lens} G={G} hq={hq} hkv={hkv}")
    c = Case(dtype, lens, G, hq, hkv, hd, page, fresh, seed=3)
    n = archer().lib.archer_op_attention_cache8_ws_bytes(0 if dtype == F16 else 1, len(lens), G, hq, hkv, hd, max(lens),
                                                         int(fresh))
    assert n > 0, "the case is meant to split"
    rows = None if G < 10 else np.arange(0, G, 7)
    say(f"  worst error / bound {c.check(c.run(), rows_of=rows):.3f}")


@pytest.mark.parametrize("lens,G,hq,hkv,hd,page,fresh,resp", [
    # columns enough for the row kernel (and for four blocks a wave of 64 dimensions): all waves in use, some, few
    ([0, 1, 63, 64, 65, 130, 257, 700], 512, 8, 8, 128, 32, True, [512, 1, 0, 33, 300, 512, 257, 100]),
    ([191, 192, 193, 0] * 4, 160, 14, 2, 128, 64, False, None),
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


KINDS = [([300, 41], 1, 4, 2, 128), ([300, 41], 80, 4, 2, 128), (WIDE_LENS, 512, 8, 4, 128), (WIDE_LENS, 512, 16, 8, 64)]


@pytest.mark.parametrize("lens,G,hq,hkv,hd", KINDS)
@pytest.mark.parametrize("q_scale,k_scale", [(30.0, 1.0), (2.0**-17, 2.0**12), (2.0**11, 2.0**-10)])
def test_peaked_small_and_large(lens, G, hq, hkv, hd, q_scale, k_scale):
    c = Case(F16, lens, G, hq, hkv, hd, 32, True, seed=9, q_scale=q_scale, k_scale=k_scale)
    c.check(c.run(), rows_of=SOME)


@pytest.mark.parametrize("lens,G,hq,hkv,hd", KINDS)
def test_shared_and_bad_pages_and_max_cached(lens, G, hq, hkv, hd):
    c = Case(F16, [300, 100] + lens[2:], G, hq, hkv, hd, 64, False, seed=32, share=True)
    c.check(c.run(), rows_of=SOME)
    c.check(c.run(max_cached=5000), rows_of=SOME)
    t = c.table.copy()
    t[0, 1], t[0, 4], t[1, 0] = len(c.data), -1, 2**31 - 1
    K, V = list(c.K), list(c.V)
    keep0, keep1 = np.r_[0:64, 128:256], np.r_[64:100]
    c.K[0], c.V[0], c.K[1], c.V[1] = K[0][:, keep0], V[0][:, keep0], K[1][:, keep1], V[1][:, keep1]
    c.check(c.run(table=t), rows_of=SOME)
    # a bound below some lengths
    c.K, c.V = [k[:, :90] for k in K], [v[:, :90] for v in V]
    c.check(c.run(max_cached=90), rows_of=SOME)
    # no page at all
    c.K, c.V = [k[:, :0] for k in K], [v[:, :0] for v in V]
    c.check(c.run(table=np.full_like(t, -1)), rows_of=SOME)


@pytest.mark.parametrize("lens,G,hq,hkv,hd", KINDS)
def test_nan_and_infinity_stay_in_place(lens, G, hq, hkv, hd):
    """A NaN in a key takes its head's rows of one sequence, one in a value one dimension of these; an infinite or
    NaN query its own row."""
    c = Case(F16, lens, G, hq, hkv, hd, 64, True, seed=33)
    B = len(lens)
    ref = host(c.run()).reshape(B, G, hq, hd)
    page, pos = divmod(77, 64)
    at = o8.locate(64, hd)
    data = c.data.copy()
    data[c.table[0, page], 1, at[0][pos, 9]] = 127
    data[c.table[1, 0], 0, at[1][40, 11]] = 255
    c.Q[1, 1 * G + G - 1, 9] = np.inf
    c.Q[0, 1 * G, 0] = np.nan
    got = host(c.run(data=data)).reshape(B, G, hq, hd)
    want = np.zeros(got.shape, bool)
    grp = hq // hkv
    want[0, :, grp:2 * grp] = want[1, G - 1, 1] = want[1, 0, 0] = True
    want[1, :, :grp, 11] = True
    assert np.isnan(got[want]).all()
    np.testing.assert_array_equal(got[~want], ref[~want])


@pytest.mark.parametrize("G", [1, 20])
def test_a_row_of_infinite_scores_is_nan(G):
    """Every score -infinity: keys there are, but no probability can be made of them."""
    c = Case(F16, [70], G, 4, 2, 128, 64, False, seed=5)
    c.data[:, :, :64 * 128] = 0x38                           # every key element 1 times its scale
    c.Q[2, 0] = 0
    c.Q[2, 0, 3] = -np.inf
    got = host(c.run()).reshape(G, 4, 128)
    assert np.isnan(got[0, 2]).all() and np.isfinite(np.delete(got, 2, 1)).all()


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


@pytest.mark.parametrize("G", [1, 20, 1040])
def test_pages_beyond_4_gib(G):
    """The same tokens in the first pages and in the last ones of a cache of 6 GB: the same bits."""
    a = archer()
    page, hkv, hd, n = 256, 8, 128, 700
    n_pages = 6 * 10**9 // (hkv * o8.page_bytes(page, hd))
    data = torch.empty(n_pages, hkv, o8.page_bytes(page, hd), dtype=torch.uint8, device="cuda")
    data[:8] = 255
    data[-8:] = 255
    c = a.Cache8(data, page, hd)
    g = torch.Generator(device="cuda").manual_seed(1)
    K, V = (torch.randn(hkv, n, hd, generator=g, device="cuda").half() for _ in range(2))
    Q = torch.randn(hkv, 4 * G, hd, generator=g, device="cuda").half()
    res = []
    for pages in ([4, 1, 2], [n_pages - 1, n_pages - 6, n_pages - 3]):
        t = torch.tensor(pages, device="cuda")
        p = torch.arange(n, device="cuda")
        a.cache8_write(c, t.int()[None], dev_i32([0]), dev_i32([0, n]), K, V)
        k, v = a.cache8_read(c, (t[p // page] * page + p % page).int())
        assert torch.isfinite(k.float()).all() and torch.isfinite(v.float()).all()
        table = t.int().repeat(4, 1).contiguous()
        res.append((k, v, a.op_attention_cache8(Q, c, table, dev_i32([n, 1, 0, 511]), n)))
    for x, y in zip(*res):
        assert torch.equal(x, y)


def test_several_calls_at_once():
    """Split attentions (each with its own workspace) on three streams."""
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
def test_samples_of_a_prompt(dtype, hq, hkv, hd, page):
    """Two prompts are stored; three samples of the first and one of the second are forked and grow side by side, one
    rolls back into the shared prompt, the first prompt's own row ends, the pool is compacted, the others go on.
    Every sample's attention is that of its own tokens."""
    a = archer()
    rng = np.random.default_rng(21)
    np_t = np.float16 if dtype == F16 else np.float32
    B, n_pages, width = 6, 24, 6
    cache = a.Cache8.empty(n_pages, page, hkv, hd)
    table, ring, pool = dev_i32(np.full((B, width), -1)), dev_i32(rng.permutation(n_pages)), dev_i32([0, n_pages])
    refs = dev_i32(np.zeros(n_pages))
    old = np.zeros(B, int)
    kv = [np.zeros((2, hkv, 0, hd)) for _ in range(B)]

    def plan(new):
        nonlocal table, refs, pool, old
        new = np.array(new)
        count = np.maximum(new - old, 0)
        p = a.pages_plan(dev_i32(old), dev_i32(new), page, table, ring, pool, refs, int(count.sum()) + 2)
        assert p.status.item() == 0
        a.pages_copy(cache.data, p.copy_src, p.copy_dst)
        n = int(count.sum())
        x = rng.standard_normal((2, hkv, n, hd)).astype(np_t)
        # at the row's end where it grows; rows that do not have no rows
        a.cache8_write(cache, p.table, dev_i32(old), p.row_off, dev(x[0], dtype),
                       dev(x[1].transpose(0, 2, 1), dtype).transpose(1, 2))
        off = p.row_off.cpu().numpy()
        for b in range(B):
            kv[b] = np.concatenate([kv[b][:, :, :min(old[b], new[b])], x[:, :, off[b]:off[b + 1]].astype(np.float64)], 2)
        table, refs, pool, old = p.table, p.refs, p.pool, new
        return p

    def check():
        q = (rng.standard_normal((hq, B, hd)) * 2).astype(np_t)
        O = host(a.op_attention_cache8(dev(q, dtype), cache, table, dev_i32(old), int(old.max()))).reshape(B, hq, hd)
        data, t = cache.data.cpu().numpy(), table.cpu().numpy()
        for b in range(B):
            k, v = o8.read(data, page, hd, o8.slots_of(t, page, b, range(old[b])))
            # what is stored is the sample's own tokens, to the format's rounding
            for got, x, i in ((k, kv[b][0], 0), (v, kv[b][1], 1)):
                if old[b]:
                    # half a step of the subnormals, of rising scales; 224 2^e < max |x|, but a token that was rolled
                    # back may have been up to 3.5 times as large
                    sc = np.abs(x).max() / 64
                    assert (np.abs(got - x) <= 2.0**-4 * np.abs(x) + 2 * 2.0**-10 * sc).all(), (b, i)
            for h in range(hq):
                kk, vv = k[h // (hq // hkv)], v[h // (hq // hkv)]
                ref, A, _, smax = oc.attention(q[h, b:b + 1].astype(np.float64), kk, vv)
                if len(kk) == 0:
                    assert (O[b, h] == 0).all()
                    continue
                tol = oc.attention_bound(ref, A, oc.score_sums(q[h, b:b + 1].astype(np.float64), kk)[0], smax, len(kk), hd,
                                         np.abs(vv).max(), dtype == F16, block=0)
                assert (np.abs(O[b, h] - ref[0]) <= tol[0]).all(), (b, h)
        used = [int(x) for b in range(B) for x in t[b, :oc.pages(old[b], page)]]
        np.testing.assert_array_equal(np.bincount(used, minlength=n_pages), refs.cpu().numpy())

    plan([2 * page + 9, 40, 0, 0, 0, 0])
    check()
    refs, st = a.pages_fork(dev_i32([0, 0, 0, 1]), dev_i32([2, 3, 4, 5]), dev_i32([2 * page + 9] * 3 + [40]), page, table, refs,
                            refs_out=refs)
    assert st.item() == 0
    for src, dst in ((0, 2), (0, 3), (0, 4), (1, 5)):
        kv[dst], old[dst] = kv[src].copy(), old[src]
    check()
    p = plan([2 * page + 9, 40, 2 * page + 10, 2 * page + 30, 2 * page + 9, 41])     # three rows write: each copies
    assert (p.copy_src >= 0).sum() == 3
    check()
    plan([0, 40, 2 * page + 11, page + 5, 3 * page, 70])                             # the prompt's row ends, one rolls back
    check()
    p = plan([0, 40, 2 * page + 12, page + 20, 3 * page, 71])                        # which then writes inside a shared page
    assert p.copy_src[3] >= 0
    check()
    m = a.pages_compact(dev_i32(old), page, table, refs)
    a.pages_copy(cache.data, m.move_src, m.move_dst, count=m.moves)
    table, refs, ring, pool = m.table, m.refs, m.free, m.pool
    check()
    U = int((refs > 0).sum())
    assert (refs[:U] > 0).all() and pool.tolist() == [0, n_pages - U]
    plan([3, 0, 2 * page + 13, page + 21, 3 * page + 1, 0])
    check()


def test_captured_turn_replays():
    """Plan, page copies, store and attention of one token per sample in one graph, replayed with other lengths and
    inputs, with eager work between the replays."""
    a = archer()
    B, hq, hkv, hd, page, n_pages, width = 4, 8, 2, 128, 32, 60, 20
    g = torch.Generator(device="cuda").manual_seed(2)
    data = torch.zeros(n_pages, hkv, o8.page_bytes(page, hd), dtype=torch.uint8, device="cuda")
    data[:, :, :2 * page * hd] = torch.randint(0, 64, (n_pages, hkv, 2 * page * hd), generator=g, device="cuda").byte()
    data[:, :, 2 * page * hd:] = 125
    cache = a.Cache8(data, page, hd)
    lens = dev_i32([5, 31, 32, 200])
    # two pairs of rows that share their pages
    table = dev_i32(np.stack([np.arange(width) + width * (b // 2) for b in range(B)]))
    refs = dev_i32([2] * 2 * width + [0] * (n_pages - 2 * width))
    ring, pool = dev_i32(np.arange(n_pages)[::-1]), dev_i32([0, n_pages - 2 * width])
    k, v = (torch.randn(hkv, B, hd, device="cuda").half() for _ in range(2))
    q = torch.randn(hq, B, hd, device="cuda").half()
    O = torch.zeros(B, hq * hd, device="cuda", dtype=torch.bfloat16)

    def turn():
        new = lens + 1
        p = a.pages_plan(lens, new, page, table, ring, pool, refs, B)
        a.pages_copy(data, p.copy_src, p.copy_dst)
        a.cache8_write(cache, p.table, lens, p.row_off, k, v)
        a.op_attention_cache8(q, cache, p.table, new, 600, O=O)
        return p

    turn()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph, stream=torch.cuda.Stream()):
        got = turn()
    for i in range(4):
        lens.copy_(dev_i32([5 + i, 31 + i, 64 - i, 500 + i]))
        for t in (k, v, q):
            t.copy_(torch.randn_like(t))
        before = data.clone()
        graph.replay()
        torch.cuda.synchronize()
        res = [O.clone(), data.clone()] + [x.clone() for x in got]
        data.copy_(before)
        O.zero_()
        p = turn()
        for x, y in zip(res, [O, data] + list(p)):
            assert torch.equal(x, y)
        assert res[-1].item() == 0 and torch.isfinite(res[0].float()).all()
