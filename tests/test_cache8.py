"""The 8-bit paged prompt cache without a GPU: its oracle against first principles, and the library's refusals."""

import ctypes as C

import numpy as np
import pytest
import torch

from oracle import cache8 as o8


def test_every_value_is_itself_and_every_midpoint_goes_to_the_even_code():
    m = o8.MAGNITUDES
    assert len(m) == 127 and m[126] == 448 and (np.diff(m) > 0).all() and m[1] == 2.0**-9 and m[8] == 2.0**-6
    for e in (-15, 0, 7):
        np.testing.assert_array_equal(o8.codes(m * 2.0**e, e), np.arange(127))
        np.testing.assert_array_equal(o8.codes(-m * 2.0**e, e), np.arange(127) + 128)
        mid = (m[1:] + m[:-1]) / 2 * 2.0**e
        np.testing.assert_array_equal(o8.codes(mid, e), (np.arange(126) + 1) // 2 * 2)
        np.testing.assert_array_equal(o8.codes(np.nextafter(mid, np.inf), e), np.arange(126) + 1)
        np.testing.assert_array_equal(o8.codes(np.nextafter(mid, 0), e), np.arange(126))
    assert o8.codes(np.array([1e9, np.inf, -np.inf]), 7).tolist() == [126, 126, 254] and o8.codes(np.array([np.nan]), 0)[0] == 127
    # exact in fp16 over the whole range of scales
    for e in range(-15, 8):
        x = m * 2.0**e
        np.testing.assert_array_equal(x.astype(np.float16).astype(np.float64), x)


def test_codes_are_torch_s():
    x = torch.cat([torch.randn(20000) * 2.0**k for k in range(-10, 7)]).clamp(-448, 448)
    np.testing.assert_array_equal(o8.codes(x.numpy(), 0), x.to(torch.float8_e4m3fn).view(torch.uint8).numpy())


def test_exponents():
    for e in range(-14, 7):
        assert o8.exponent(448 * 2.0**e) == e and o8.exponent(np.nextafter(448 * 2.0**e, np.inf)) == e + 1
    assert o8.exponent(0) == -15 and o8.exponent(1e-9) == -15 and o8.exponent(np.inf) == 7


@pytest.mark.parametrize("page,hd", [(32, 64), (32, 128), (64, 128), (256, 64)])
def test_a_page_is_filled_once(page, hd):
    k, v, s = o8.locate(page, hd)
    at = np.concatenate([k.ravel(), v.ravel()])
    assert sorted(at) == list(range(2 * page * hd))
    assert sorted(set(s.ravel())) == list(range(2 * page * hd, 2 * page * hd + page // 16)) and s.max() < o8.page_bytes(page, hd)


def test_append_keeps_the_earlier_tokens():
    """Tokens one by one and all at once: the same scale at the end, and the earlier tokens no worse than by
    half a step of the last scale's smallest numbers."""
    rng = np.random.default_rng(0)
    hd, page, n = 64, 64, 45
    K, V = (rng.standard_normal((2, n, hd)) * 2.0 ** rng.integers(-6, 6, (2, n, 1)) for _ in range(2))
    table = [[3, 1]]
    once = o8.write(np.zeros((4, 2, o8.page_bytes(page, hd)), np.uint8), page, hd, table, [0], [0, n], K, V)
    step = np.zeros_like(once)
    for t in range(n):
        step = o8.write(step, page, hd, table, [t], [0, 1], K[:, t:t + 1], V[:, t:t + 1])
    at = o8.locate(page, hd)
    np.testing.assert_array_equal(step[3][:, at[2]], once[3][:, at[2]])
    slots = o8.slots_of(table, page, 0, range(n))
    for x, a, b, i in zip((K, V), o8.read(step, page, hd, slots), o8.read(once, page, hd, slots), range(2)):
        sc = 2.0 ** (once[3][:, at[2][:n, i]].astype(int) - 127.0)[..., None]
        # rounded relatively each time it is exact again; 2^-10 of the scale where it is subnormal, at most once a scale
        assert (np.abs(a - x) <= 2.0**-4 * np.abs(x) + 2 * 2.0**-10 * sc).all()
        assert (np.abs(b - x) <= 2.0**-4 * np.abs(x) + 2.0**-10 * sc).all()
    np.testing.assert_array_equal(o8.read(once, page, hd, slots[:32])[0], o8.stored(K[:, :32]))


# -- the library's host-side checks ----------------------------------------------------------------
X = 1 << 20


def _desc(a, **kw):
    d = dict(data=X, n_pages=4, page_size=64, n_kv_heads=2, head_dim=128)
    d.update(kw)
    return a.Cache8Desc(d["data"], d["n_pages"], d["page_size"], d["n_kv_heads"], d["head_dim"])


def test_cache_shapes():
    from paper_2608_08086_amd import archer as a
    for page, hd in ((32, 64), (64, 128), (256, 128)):
        n = a.lib.archer_cache8_bytes(C.byref(_desc(a, data=None, page_size=page, head_dim=hd)))
        assert n == 4 * 2 * o8.page_bytes(page, hd) and a.Cache8.page_bytes(page, hd) == o8.page_bytes(page, hd)
    for kw in (dict(page_size=16), dict(page_size=48), dict(page_size=512), dict(head_dim=96), dict(n_pages=0),
               dict(n_kv_heads=0), dict(n_pages=1 << 25), dict(n_kv_heads=65536)):
        assert a.lib.archer_cache8_bytes(C.byref(_desc(a, **kw))) == 0, kw
        assert a.lib.archer_last_error()
    assert a.lib.archer_cache8_bytes(None) == 0


def test_write_and_read_arguments():
    from paper_2608_08086_amd import archer as a

    def write(dtype=0, c=None, batch=2, table=X, width=4, start=X, off=X, rows=3, K=X, V=X, vr=128, vd=1, **kw):
        return a.lib.archer_cache8_write(dtype, C.byref(_desc(a, **kw)) if c is None else c, batch, table, width, start, off,
                                         rows, K, 512, 128, V, 512, vr, vd, None)

    def read(dtype=0, rows=3, K=X, V=X, slots=X, **kw):
        return a.lib.archer_cache8_read(dtype, C.byref(_desc(a, **kw)), rows, slots, K, V, None)
    for f in (write, read):
        assert f(dtype=a.FP16) == a.E_ARG and f(dtype=7) == a.E_ARG
        assert f(data=None) == a.E_ARG and f(data=X + 8) == a.E_ARG
        assert f(page_size=16) == a.E_SHAPE and f(head_dim=32) == a.E_SHAPE and f(rows=-1) == a.E_SHAPE
        assert f(K=None) == a.E_ARG and f(V=None) == a.E_ARG
        assert f(rows=0) == a.OK and f(rows=0, K=None, V=None) == a.OK
    for kw in (dict(batch=0), dict(batch=65536), dict(width=0), dict(width=1 << 26)):
        assert write(**kw) == a.E_SHAPE, kw
    for kw in (dict(table=None), dict(start=None), dict(off=None), dict(K=X + 1), dict(dtype=a.FP32, V=X + 2)):
        assert write(**kw) == a.E_ARG, kw
    assert write(vr=2, vd=2) == a.E_UNSUPPORTED
    assert read(slots=None) == a.E_ARG and read(K=X + 8) == a.E_ARG and read(V=X + 8) == a.E_ARG


def test_attention_arguments():
    from paper_2608_08086_amd import archer as a
    base = dict(dtype=0, B=2, G=4, Hq=4, Q=X, table=X, width=8, lens=X, cap=100, K2=X, V2=X, ld2=64, fs=8, resp=None, O=X)

    def call(desc=None, **kw):
        d = dict(base, **kw)
        return a.lib.archer_op_attention_cache8(d["dtype"], C.byref(desc or _desc(a)), d["B"], d["G"], d["Hq"], d["Q"],
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
    ws = a.lib.archer_op_attention_cache8_ws_bytes
    assert ws(0, 1, 4, 4, 2, 128, 100000, 1) > 0 and ws(0, 1, 4, 4, 2, 128, 0, 0) == 0
    assert ws(a.FP16, 1, 4, 4, 2, 128, 100, 1) == 0 and ws(0, 1, 4, 4, 3, 128, 100, 1) == 0


def test_binding_refusals(monkeypatch):
    """Host tensors in the place of the device's: every refusal comes before the library is called."""
    from paper_2608_08086_amd import archer as a
    monkeypatch.setattr(torch.cuda, "current_device", lambda: -1)
    for f in ("archer_cache8_write", "archer_cache8_read", "archer_op_attention_cache8", "archer_op_attention_cache4",
              "archer_cache4_write", "archer_cache4_read"):
        monkeypatch.setattr(a.lib, f, lambda *x: pytest.fail("the library was called"))
    i = lambda *x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    h = lambda *s: torch.zeros(*s, dtype=torch.float16)  # noqa: E731
    c = a.Cache8(torch.zeros(4, 2, o8.page_bytes(32, 64), dtype=torch.uint8), 32, 64)
    c4 = a.Cache4(torch.zeros(4, 2, 32 * 68, dtype=torch.uint8), 32, 64)
    t = i(0, 1)[None]
    bad = [
        lambda: a.Cache8(torch.zeros(4, 2, 32 * 128, dtype=torch.uint8), 32, 64),
        lambda: a.Cache8(torch.zeros(4, 2, o8.page_bytes(32, 64), dtype=torch.int8), 32, 64),
        lambda: a.Cache8(torch.zeros(4, 2, o8.page_bytes(32, 64), dtype=torch.uint8), 32, 2**32 + 64),
        lambda: a.cache8_write(c, t, i(0), i(0, 3), h(2, 3, 64), h(2, 4, 64)),
        lambda: a.cache8_write(c, t, i(0), i(0, 3), h(3, 3, 64), h(3, 3, 64)),
        lambda: a.cache8_write(c, t, i(0), i(0, 3), h(2, 3, 64), h(2, 3, 64).float()),
        lambda: a.cache8_write(c, t, i(0), i(0, 3), h(2, 64, 3).transpose(1, 2), h(2, 3, 64)),
        lambda: a.cache8_write(c, t, i(0), i(0, 1, 3), h(2, 3, 64), h(2, 3, 64)),
        lambda: a.cache8_write(c, t, i(0, 0), i(0, 3), h(2, 3, 64), h(2, 3, 64)),
        lambda: a.cache8_write(c, t[0], i(0), i(0, 3), h(2, 3, 64), h(2, 3, 64)),
        lambda: a.cache8_write(c, t.long(), i(0), i(0, 3), h(2, 3, 64), h(2, 3, 64)),
        lambda: a.cache8_write(c4, t, i(0), i(0, 3), h(2, 3, 64), h(2, 3, 64)),
        lambda: a.cache8_read(c, i(0, 1), torch.bfloat16),
        lambda: a.cache8_read(c4, i(0, 1)), lambda: a.cache4_read(c, i(0, 1)),
        lambda: a.cache4_write(c, h(2, 3, 64), h(2, 3, 64), i(0, 1, 2)),
        lambda: a.op_attention_cache4(h(2, 2, 64), c, i(0, 1)[:, None], i(1, 1), 9),
        lambda: a.op_attention_cache8(h(2, 2, 64), c4, i(0, 1)[:, None], i(1, 1), 9),
        lambda: a.op_attention_cache8(h(2, 2, 64), c, i(0, 1)[:, None], i(1, 1), 2**31),
        lambda: a.op_attention_cache8(h(2, 3, 64), c, i(0, 1)[:, None], i(1, 1), 9),
        lambda: a.op_attention_cache8(h(2, 2, 64), c, i(0, 1)[:, None], i(1, 1), 9, K2=h(2, 16, 64)),
    ]
    for f in bad:
        with pytest.raises(a.ArcherError):
            f()
