"""The 4-bit paged prompt cache without a GPU: the oracle's storage and plans,
and the library's host-side checks (no kernel runs here)."""

import ctypes as C

import numpy as np
import pytest

from oracle import cache4 as oc


def test_magnitudes_ties_and_saturation():
    # the block's largest element 4 sets the scale 1 (4 <= 7, 4 > 3.5)
    x = np.zeros(32)
    x[:14] = [4, 0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 0.2500001, 0.7499999, -0.75, -0.25, 3.4999999, -0.0, 0.1]
    code, scale = oc.quantise(x)
    assert scale.tolist() == [127]
    want = [4, 0, 1, 1, 2, 2, 4, 0.5, 0.5, -1, 0, 3, 0, 0]
    np.testing.assert_array_equal(oc.values(code, scale)[:14], want)
    assert code[9] == 10 and code[10] == 8 and code[12] == 8     # the sign stays with a zero


@pytest.mark.parametrize("top,e", [(7.0, 0), (np.nextafter(7.0, 8), 1), (3.5, -1), (6.0, 0), (0.0, oc.E_MIN),
                                   (2.0**-24, oc.E_MIN), (65504.0, oc.E_MAX), (np.inf, oc.E_MAX), (1e30, oc.E_MAX)])
def test_scale_is_the_least_that_reaches_the_largest_element(top, e):
    x = np.zeros(64)
    x[40] = -top
    code, scale = oc.quantise(x)
    assert scale.tolist() == [oc.E_MIN + 127, e + 127]
    v = oc.values(code, scale)[40]
    assert v == -6 * 2.0**e if top > 5 * 2.0**e else abs(v + top) <= 2.0**e


def test_stored_elements_are_exact_in_fp16_and_idempotent():
    rng = np.random.default_rng(0)
    x = (rng.standard_normal((300, 128)) * 2.0 ** rng.integers(-30, 20, (300, 1))).astype(np.float32)
    v = oc.stored(x)
    np.testing.assert_array_equal(v, v.astype(np.float16).astype(np.float64))
    np.testing.assert_array_equal(oc.stored(v), v)
    # no element moves by more than half a step of its block's largest binade, or to the saturated value
    err = np.abs(v - x).reshape(300, 4, 32)
    top = np.abs(x).reshape(300, 4, 32).max(-1)
    ok = top <= 7 * 2.0**oc.E_MAX
    assert (err.max(-1)[ok] <= np.maximum(top[ok] / 3.5, 2.0 ** (oc.E_MIN - 2))).all()


def test_a_nan_takes_its_block():
    x = np.ones(128)
    x[70] = np.nan
    v = oc.stored(x)
    assert np.isnan(v[64:96]).all() and (v[:64] == 1).all() and (v[96:] == 1).all()


@pytest.mark.parametrize("page,hd", [(32, 64), (64, 128), (256, 128)])
def test_layout_uses_every_nibble_once(page, hd):
    key, value, shift, ks, vs = oc.locate(page, hd)
    nib = np.concatenate([(2 * a + shift // 4).ravel() for a in (key, value)])
    sc = np.concatenate([ks.ravel(), vs.ravel()])
    assert len(set(nib.tolist())) == 2 * page * hd and len(set(sc.tolist())) == 2 * page * hd // 32
    assert nib.max() // 2 < sc.min() and sc.max() == oc.page_bytes(page, hd) - 1


def test_write_then_read():
    rng = np.random.default_rng(1)
    K, V = rng.standard_normal((2, 5, 64)), rng.standard_normal((2, 5, 64))
    slots = [33, -1, 64, 200, 2]
    data = oc.write(np.zeros((3, 2, oc.page_bytes(32, 64)), np.uint8), 32, 64, K, V, slots)
    k, v = oc.read(data, 32, 64, slots)
    for got, x in ((k, K), (v, V)):
        np.testing.assert_array_equal(got[:, [0, 2, 4]], oc.stored(x)[:, [0, 2, 4]])
        assert (got[:, [1, 3]] == 0).all()


def test_plan_grows_shrinks_and_rolls_back():
    T = 32
    table = np.full((3, 4), -7)
    ring = np.arange(100, 108)
    t, r, pool, off, slots, st = oc.plan([0, 0, 0], [33, 0, 64], T, table, ring, [6, 8], 100)
    assert st == 0 and pool.tolist() == [2, 4]
    assert t.tolist() == [[106, 107, -7, -7], [-7] * 4, [100, 101, -7, -7]]
    assert off.tolist() == [0, 33, 33, 97] and slots[32] == 107 * T and slots[33] == 100 * T and (slots[97:] == -1).all()
    # the first request rolls back to one page, the second starts, the third finishes
    t2, r2, pool2, off2, _, st = oc.plan([33, 0, 64], [20, 40, 0], T, t, r, pool, 40)
    assert st == 0 and t2[1, :2].tolist() == [102, 103] and off2.tolist() == [0, 0, 40, 40]
    assert pool2.tolist() == [4, 5] and [r2[(4 + i) % 8] for i in range(5)] == [104, 105, 107, 100, 101]


@pytest.mark.parametrize("old,new,pool,rows,want", [
    ([0], [129], [0, 5], 200, 2), ([-1], [3], [0, 5], 9, 2), ([0], [97], [0, 3], 200, 1), ([0], [9], [0, 5], 8, 3),
    ([0], [9], [5, 1], 20, 4), ([0], [9], [0, 6], 20, 4), ([64], [0], [0, 4], 0, 4),
])
def test_plan_refusals_change_nothing(old, new, pool, rows, want):
    table, ring = np.arange(4)[None], np.arange(5)
    t, r, p, off, slots, st = oc.plan(old, new, 32, table, ring, pool, rows)
    assert st == want and (t == table).all() and (r == ring).all() and p.tolist() == pool
    assert (off == 0).all() and (slots == -1).all()


# -- the library's host-side checks ----------------------------------------------------------------
X = 1 << 20   # a non-null, aligned address that no refused call reads


def _desc(a, **kw):
    d = dict(data=X, n_pages=4, page_size=64, n_kv_heads=2, head_dim=128)
    d.update(kw)
    return a.Cache4Desc(d["data"], d["n_pages"], d["page_size"], d["n_kv_heads"], d["head_dim"])


def test_cache_shapes():
    from paper_2608_08086_amd import archer as a
    assert a.lib.archer_cache4_bytes(C.byref(_desc(a, data=None))) == 4 * 2 * 64 * 136
    assert a.lib.archer_cache4_bytes(C.byref(_desc(a, head_dim=64, page_size=32))) == 4 * 2 * 32 * 68
    for kw in (dict(page_size=16), dict(page_size=48), dict(page_size=512), dict(head_dim=96), dict(n_pages=0),
               dict(n_kv_heads=0), dict(n_pages=1 << 25), dict(n_kv_heads=65536)):
        assert a.lib.archer_cache4_bytes(C.byref(_desc(a, **kw))) == 0, kw
        assert a.lib.archer_last_error()
    assert a.lib.archer_cache4_bytes(None) == 0


def test_plan_arguments():
    from paper_2608_08086_amd import archer as a
    base = dict(batch=2, old=X, new=X, page=64, n_pages=4, width=8, table=X, free=X, pin=X, pout=2 * X, off=X, slots=X,
                rows=8, status=X)

    def call(**kw):
        d = dict(base, **kw)
        return a.lib.archer_cache4_plan(d["batch"], d["old"], d["new"], d["page"], d["n_pages"], d["width"], d["table"],
                                        d["free"], d["pin"], d["pout"], d["off"], d["slots"], d["rows"], d["status"], None)
    for n in ("old", "new", "table", "free", "pin", "pout", "off", "slots", "status"):
        assert call(**{n: None}) == a.E_ARG, n
    for kw in (dict(batch=0), dict(batch=4097), dict(page=16), dict(page=65), dict(n_pages=0), dict(n_pages=1 << 25),
               dict(width=0), dict(width=1 << 25), dict(rows=-1)):
        assert call(**kw) == a.E_SHAPE, kw
    for out in (X, X + 4, X - 4):
        assert call(pout=out) == a.E_ARG       # pool_out aliases pool_in


def test_write_and_read_arguments():
    from paper_2608_08086_amd import archer as a

    def write(dtype=0, c=None, rows=3, K=X, V=X, vr=128, vd=1, slots=X, **kw):
        return a.lib.archer_cache4_write(dtype, C.byref(_desc(a, **kw)) if c is None else c, rows, K, 512, 128, V, 512, vr,
                                         vd, slots, None)

    def read(dtype=0, rows=3, K=X, V=X, slots=X, **kw):
        return a.lib.archer_cache4_read(dtype, C.byref(_desc(a, **kw)), rows, slots, K, V, None)
    for f in (write, read):
        assert f(dtype=a.FP16) == a.E_ARG and f(dtype=7) == a.E_ARG
        assert f(data=None) == a.E_ARG and f(data=X + 8) == a.E_ARG
        assert f(page_size=16) == a.E_SHAPE and f(head_dim=32) == a.E_SHAPE and f(rows=-1) == a.E_SHAPE
        assert f(K=None) == a.E_ARG and f(V=None) == a.E_ARG and f(slots=None) == a.E_ARG
        assert f(rows=0) == a.OK and f(rows=0, K=None, V=None, slots=None) == a.OK
    assert write(vr=2, vd=2) == a.E_UNSUPPORTED
    assert write(K=X + 1) == a.E_ARG and write(dtype=a.FP32, V=X + 2) == a.E_ARG
    assert read(K=X + 8) == a.E_ARG and read(V=X + 8) == a.E_ARG
    assert a.lib.archer_cache4_write(0, None, 3, X, 1, 1, X, 1, 1, 1, X, None) == a.E_ARG


def test_attention_arguments():
    from paper_2608_08086_amd import archer as a
    base = dict(dtype=0, B=2, G=4, Hq=4, Q=X, table=X, width=8, lens=X, cap=100, K2=X, V2=X, ld2=64, fs=8, resp=None, O=X)

    def call(desc=None, **kw):
        d = dict(base, **kw)
        return a.lib.archer_op_attention_cache4(d["dtype"], C.byref(desc or _desc(a)), d["B"], d["G"], d["Hq"], d["Q"],
                                                d["table"], d["width"], d["lens"], d["cap"], d["K2"], d["V2"], d["ld2"],
                                                d["fs"], d["resp"], d["O"], None, 0, None)
    for n in ("Q", "table", "lens", "O", "K2", "V2"):
        assert call(**{n: None}) == a.E_ARG, n
    for n in ("Q", "K2", "V2", "O"):
        assert call(**{n: X + 8}) == a.E_ARG, n
    assert call(dtype=a.FP16) == a.E_ARG and call(desc=_desc(a, data=None)) == a.E_ARG
    for kw in (dict(B=0), dict(G=0), dict(Hq=3), dict(Hq=0), dict(width=0), dict(width=1 << 26), dict(cap=-1),
               dict(fs=4), dict(G=9), dict(ld2=12), dict(ld2=8), dict(B=65536), dict(G=1 << 30, fs=1 << 30)):
        assert call(**kw) == a.E_SHAPE, kw
    assert call(desc=_desc(a, page_size=100)) == a.E_SHAPE
    # one sequence of many keys is split, and a split needs its workspace
    assert call(B=1, cap=100000) == a.E_WORKSPACE
    ws = a.lib.archer_op_attention_cache4_ws_bytes
    assert ws(0, 1, 4, 4, 2, 128, 100000, 1) > 0 and ws(0, 1, 4, 4, 2, 128, 0, 0) == 0
    assert ws(a.FP16, 1, 4, 4, 2, 128, 100, 1) == 0 and ws(0, 1, 4, 4, 3, 128, 100, 1) == 0
