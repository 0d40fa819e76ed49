"""Oracle of the 4-bit paged prompt cache (float64 NumPy): plans, stored
elements, page bytes and attention, written from the definitions in
``include/archer_ops.h``."""

from __future__ import annotations

import numpy as np

MAGNITUDES = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E_MIN, E_MAX, NAN_SCALE = -23, 13, 255
BLOCK = 32


def pages(n, page_size):
    return -(-int(n) // page_size)


def page_bytes(page_size, hd):
    return page_size * (hd + hd // 16)


# -- plan ----------------------------------------------------------------------------------------
def plan(len_old, len_new, page_size, table, free_pages, pool, slot_rows):
    """Returns (table, free_pages, pool, row_off, slot_map, status) after the plan; inputs unchanged."""
    table, ring = np.array(table), np.array(free_pages)
    n, width = len(ring), table.shape[1]
    head, count = int(pool[0]), int(pool[1])
    B = len(len_old)
    taken = sum(max(pages(b, page_size) - pages(a, page_size), 0) for a, b in zip(len_old, len_new))
    given = sum(max(pages(a, page_size) - pages(b, page_size), 0) for a, b in zip(len_old, len_new))
    rows = sum(max(int(b) - int(a), 0) for a, b in zip(len_old, len_new))
    status = 0
    if not (0 <= head < n and 0 <= count <= n):
        status = 4
    elif any(x < 0 or x > width * page_size for x in list(len_old) + list(len_new)):
        status = 2
    elif given > n - count:
        status = 4
    elif taken > count:
        status = 1
    elif rows > slot_rows:
        status = 3
    slots, off = np.full(slot_rows, -1, dtype=np.int64), np.zeros(B + 1, dtype=np.int64)
    if status:
        return table, ring, np.array([head, count]), off, slots, status
    front, back, at = head, head + count, 0
    for b in range(B):
        have, want = pages(len_old[b], page_size), pages(len_new[b], page_size)
        for j in range(have, want):
            table[b, j] = ring[front % n]
            front += 1
        for j in range(want, have):
            ring[back % n] = table[b, j]
            back += 1
        for p in range(int(len_old[b]), int(len_new[b])):
            slots[at] = table[b, p // page_size] * page_size + p % page_size
            at += 1
        off[b + 1] = at
    return table, ring, np.array([front % n, count - taken + given]), off, slots, 0


# -- storage -------------------------------------------------------------------------------------
def quantise(x):
    """x [..., D] -> codes (0..15) [..., D] and scale bytes [..., D / 32]."""
    x = np.asarray(x, dtype=np.float64)
    b = x.reshape(*x.shape[:-1], x.shape[-1] // BLOCK, BLOCK)
    with np.errstate(invalid="ignore"):
        top = np.max(np.abs(b), axis=-1)          # NaN if the block holds one
        e = np.full(top.shape, E_MIN)
        for k in range(E_MIN, E_MAX):
            e = np.where(top > 7.0 * 2.0**k, k + 1, e)
        y = np.abs(b) / 2.0 ** e[..., None]
        # nearest magnitude; between two, the one with the even code
        code = ((y > 0.25).astype(int) + (y >= 0.75) + (y > 1.25) + (y >= 1.75) + (y > 2.5) + (y >= 3.5) + (y > 5.0))
    code = code + 8 * np.signbit(b)
    scale = np.where(np.isnan(top), NAN_SCALE, e + 127)
    return code.reshape(x.shape).astype(np.uint8), scale.astype(np.uint8)


def values(code, scale):
    """The elements that codes [..., D] and scale bytes [..., D / 32] stand for."""
    v = np.where(code & 8, -1.0, 1.0) * MAGNITUDES[code & 7]
    s = np.repeat(scale.astype(np.int64), BLOCK, axis=-1)
    return np.where(s == NAN_SCALE, np.nan, v * 2.0 ** (s - 127.0))


def stored(x):
    return values(*quantise(x))


def locate(page_size, hd):
    """Where a token's nibbles and scales lie in a page: for the positions t of a page, arrays of byte
    offsets key[t][d], value[t][d] (with the nibble's shift, [d]) and key_scale[t][g], value_scale[t][g]."""
    t, d, g = np.arange(page_size)[:, None], np.arange(hd)[None], np.arange(hd // BLOCK)[None]
    unit, inside = d // (hd // 16), d % (hd // 16)
    key = t * (hd // 2) + d // 2
    value = page_size * hd // 2 + ((t // 8 * 16 + unit) * 8 + t % 8) * (hd // 32) + inside // 2
    ks = page_size * hd + (t // 8 * (hd // BLOCK) + g) * 8 + t % 8
    return key, value, 4 * (d[0] % 2), ks, ks + page_size * hd // BLOCK


def write(data, page_size, hd, K, V, slots):
    """Page bytes [n_pages][heads][...] after rows K, V [heads][rows][hd] went to their slots."""
    data = np.array(data)
    key, value, shift, ks, vs = locate(page_size, hd)
    kc, ke = quantise(K)
    vc, ve = quantise(V)
    for r, s in enumerate(slots):
        if not 0 <= s < data.shape[0] * page_size:
            continue
        p, t = divmod(int(s), page_size)
        for h in range(data.shape[1]):
            for code, at in ((kc[h, r], key[t]), (vc[h, r], value[t])):
                data[p, h, at[0::2]] = code[0::2] | code[1::2] << 4
            data[p, h, ks[t]], data[p, h, vs[t]] = ke[h, r], ve[h, r]
    return data


def read(data, page_size, hd, slots):
    """Stored K, V [heads][rows][hd] of the slots; rows without a slot are zero."""
    key, value, shift, ks, vs = locate(page_size, hd)
    H = data.shape[1]
    K, V = np.zeros((H, len(slots), hd)), np.zeros((H, len(slots), hd))
    for r, s in enumerate(slots):
        if not 0 <= s < data.shape[0] * page_size:
            continue
        p, t = divmod(int(s), page_size)
        K[:, r] = values((data[p][:, key[t]] >> shift) & 15, data[p][:, ks[t]])
        V[:, r] = values((data[p][:, value[t]] >> shift) & 15, data[p][:, vs[t]])
    return K, V


# -- attention -----------------------------------------------------------------------------------
def attention(Q, K, V):
    """Q [M][hd], K, V [n][hd] -> O [M][hd] and, for error bounds, A = sum p |v| / sum p, the largest
    sum |q k| / sqrt(hd) with each q taken as its 32 dimensions' largest, and the largest score magnitude
    (zeros without keys)."""
    M, hd = Q.shape
    if len(K) == 0:
        return np.zeros((M, hd)), np.zeros((M, hd)), 0.0, 0.0
    s = Q @ K.T / np.sqrt(hd)
    p = np.exp(s - s.max(-1, keepdims=True))
    p /= p.sum(-1, keepdims=True)
    top = np.repeat(np.abs(Q).reshape(M, hd // BLOCK, BLOCK).max(-1), BLOCK, axis=-1)
    return p @ V, p @ np.abs(V), float((top @ np.abs(K).T).max() / np.sqrt(hd)), float(np.abs(s).max())


def score_sums(Q, K):
    """Per query row, the largest sum |q k| / sqrt(hd) of its scores: as it is, and with each q taken as its 32
    dimensions' largest."""
    Q, K = np.abs(Q), np.abs(K)
    top = np.repeat(Q.reshape(len(Q), -1, BLOCK).max(-1), BLOCK, axis=-1)
    return tuple((x @ K.T).max(-1, keepdims=True) / np.sqrt(Q.shape[1]) for x in (Q, top))


def attention_bound(O, A, qk, smax, n, hd, vmax, half, block=None):
    """Largest error of the library's kernels.  half: fp16 queries (fp16 probabilities, bf16 output) or fp32.
    block None: qk is the second of `score_sums`, and any kernel may have run.  Else qk is the first, and block
    the second where the row kernel runs (fp16, 128 dimensions, many rows) and 0 for the others.

    A score is a sum of hd products in fp32, each rounding at most 2^-24 of the running sum of magnitudes,
    then scaled and rounded: (hd + 3) 2^-24 qk, and 2^-23 smax for the exponent's argument.  The exponential
    itself: 2^-22.  With fp16 queries the row kernel multiplies four e2m3 terms of each query element: the
    first is off by at most 2^-2 of its scale s1 (half the largest step), the second, of scale s1 / 16 and at
    most 4 of it, by 2^-3 s1 / 16, the third and the fourth, each of 2^-5 of the scale before and at most 4 of it, by
    2^-3 s1 / 512 and 2^-3 s1 / 2^14 = 2^-17 s1; s1 is the least power of two that has the block's largest element
    below 7.5 s1, which therefore exceeds 3.75 s1: 2^-18.9 of it, 2^-18.9 block in a score.  These are 4 hd
    products: a term that overshoots is taken back by the next ones, by at most |q| where it is the element's first
    (it is no more than twice |q|) and by at most s1 / 4 in all, so the terms' magnitudes add up to no more than 3.5 |q|
    and |q| + 0.52 s1; and the sum starts from the reference, at most smax:
    (4 hd + 4) 2^-24 (min(3.5 qk, qk + block / 7) + smax).
    These are relative errors of the probabilities, in the numerator and in the denominator.
    Sums over n keys in fp32, with one rescale per 32 keys: (n + n / 16 + 40) 2^-24 in both.  fp16 probabilities:
    half a step is 2^-11 relative, and 2^-25 absolute where they are subnormal (the largest is between 1 and
    2^8, so that the denominator is at least 1).  The output's own rounding: bf16 2^-8, fp32 2^-24."""
    rows = half if block is None else np.asarray(block) > 0
    block = qk if block is None else block
    rel = np.where(rows, (4 * hd + 4) * 2.0**-24 * (np.minimum(3.5 * qk, qk + block / 7) + smax) + 2.0**-18.9 * block, (hd + 3) * 2.0**-24 * qk)
    rel = 2 * (rel + 2.0**-23 * smax + 2.0**-22 + (n + n / 16 + 40) * 2.0**-24)
    if not half:
        return 2.0**-24 * np.abs(O) + A * rel + 1e-30
    return 2.0**-8 * np.abs(O) + A * (rel + 2.0**-11) + n * 2.0**-25 * vmax + 1e-30
