"""Oracle of the 8-bit paged prompt cache (float64 NumPy): stored elements and page bytes,
written from the definitions in ``include/archer_ops.h``.  Attention is `oracle.cache4.attention`."""

from __future__ import annotations

import numpy as np

from .cache4 import pages  # noqa: F401

BLOCK = 32
E_MIN, E_MAX = -15, 7
# the 127 finite magnitudes of e4m3, code 0 .. 126
MAGNITUDES = np.array([m * 2.0**-9 if e == 0 else (8 + m) * 2.0 ** (e - 10) for e in range(16) for m in range(8)])[:127]
VALUES = np.concatenate([MAGNITUDES, [np.nan], -MAGNITUDES, [np.nan]])


def page_bytes(page_size, hd):
    return 2 * page_size * hd + 16


def exponent(top):
    """Least e with top <= 448 * 2^e, clamped."""
    for e in range(E_MIN, E_MAX):
        if top <= 448 * 2.0**e:
            return e
    return E_MAX


def codes(x, e):
    """Nearest e4m3 codes of x / 2^e: of two, the even one; saturating; a NaN is a NaN."""
    y = np.minimum(np.abs(np.asarray(x, dtype=np.float64)) / 2.0**e, 448.0)
    hi = np.clip(np.searchsorted(MAGNITUDES, np.nan_to_num(y)), 1, 126)
    lo = hi - 1
    down, up = y - MAGNITUDES[lo], MAGNITUDES[hi] - y
    code = np.where((down < up) | ((down == up) & (lo % 2 == 0)), lo, hi)
    code = np.where(np.isnan(x), 127, code)
    return (code + 128 * np.signbit(x)).astype(np.uint8)


def stored(x, e=None):
    """x [heads][n <= 32][hd], one block's rows, as stored; e: [heads] scales of earlier tokens, or None."""
    out = np.empty(np.shape(x))
    for h in range(len(x)):
        a = np.abs(x[h])
        s = exponent(np.max(np.where(np.isnan(a), 0, a), initial=0.0))
        s = s if e is None else max(s, e[h])
        out[h] = VALUES[codes(x[h], s)] * 2.0**s
    return out


def locate(page_size, hd):
    """Byte offsets in a page: key[t][d], value[t][d], and scale[t][2] (of the keys, of the values)."""
    t, d = np.arange(page_size)[:, None], np.arange(hd)[None]
    unit, inside = d // (hd // 16), d % (hd // 16)
    value = page_size * hd + (t // 8 * (hd // 32) + inside // 2) * 256 + unit * 16 + inside % 2 * 8 + t % 8
    return t * hd + d, value, 2 * page_size * hd + t // BLOCK * 2 + np.arange(2)[None]


def write(data, page_size, hd, table, start, row_off, K, V):
    """Page bytes [n_pages][heads][...] after rows row_off[b] .. of K, V [heads][rows][hd] became the tokens from
    start[b] on of the sequence of row b of the table.  Bytes of later tokens of the last block: zeros."""
    data = np.array(data)
    at = locate(page_size, hd)
    H, rows, _ = np.shape(K)
    width = np.shape(table)[1]
    for b in range(len(start)):
        first = int(start[b])
        n = min(int(row_off[b + 1]), rows) - int(row_off[b])
        n = min(n, width * page_size - first)
        for blk in range(first // BLOCK, (first + n - 1) // BLOCK + 1 if n > 0 else 0):
            p0 = blk * BLOCK
            page, t0 = int(table[b][p0 // page_size]), p0 % page_size
            if not 0 <= page < len(data):
                continue
            lo, hi = max(first, p0), min(first + n, p0 + BLOCK)
            src = slice(int(row_off[b]) + lo - first, int(row_off[b]) + hi - first)
            for i, x in enumerate((K, V)):
                for h in range(H):
                    new = np.asarray(x[h, src], dtype=np.float64)
                    a = np.abs(new)
                    e = exponent(np.max(np.where(np.isnan(a), 0, a)))
                    byte = at[2][t0, i]
                    if first > p0:
                        was = min(max(int(data[page, h, byte]) - 127, E_MIN), E_MAX)
                        e = max(e, was)
                    for t in range(BLOCK):
                        bytes_ = at[i][t0 + t]
                        if p0 + t < lo:
                            data[page, h, bytes_] = codes(VALUES[data[page, h, bytes_]] * 2.0**was, e)
                        elif p0 + t < hi:
                            data[page, h, bytes_] = codes(new[p0 + t - lo], e)
                        else:
                            data[page, h, bytes_] = 0
                    data[page, h, byte] = e + 127
    return data


def read(data, page_size, hd, slots):
    """Stored K, V [heads][rows][hd] of the slots; rows without a slot are zero."""
    at = locate(page_size, hd)
    out = np.zeros((2, data.shape[1], len(slots), hd))
    for r, s in enumerate(slots):
        if not 0 <= s < data.shape[0] * page_size:
            continue
        p, t = divmod(int(s), page_size)
        for i in range(2):
            out[i, :, r] = VALUES[data[p][:, at[i][t]]] * 2.0 ** (data[p][:, at[2][t, i]].astype(np.int64) - 127.0)[:, None]
    return out[0], out[1]


def slots_of(table, page_size, b, positions):
    return [int(table[b][p // page_size]) * page_size + p % page_size for p in positions]
