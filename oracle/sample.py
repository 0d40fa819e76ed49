"""Oracle of sampling (float64 NumPy), row by row from the definition in ``include/archer_ops.h``."""

from __future__ import annotations

import numpy as np


def kept(logits, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0, exclude=-1):
    """The kept tokens' weights [vocab] of one row (zeros of the others) and the order of its tokens; None for a row without any."""
    l = np.array(logits, dtype=np.float64)
    if exclude >= 0:
        l[exclude] = -np.inf
    if np.isnan(l).any() or l.max() == -np.inf:
        return None
    if l.max() == np.inf:
        l = np.where(l == np.inf, 0.0, -np.inf)
    order = np.argsort(-l, kind="stable")
    with np.errstate(over="ignore"):
        z = (l - l.max()) / np.float64(temperature) if temperature > 0 else np.where(np.arange(len(l)) == order[0], 0, -np.inf)
    z[l == -np.inf] = -np.inf
    w = np.exp(z)[order]
    keep = np.ones(len(l), bool)
    if top_k > 0:
        keep[top_k:] = False
    if top_p < 1:
        w1 = np.where(keep, w, 0)
        before = np.concatenate([[0.0], np.cumsum(w1)[:-1]])
        keep &= before < top_p * w1.sum()
    if min_p > 0:
        keep &= w >= min_p
    keep[0] = True
    out = np.zeros(len(l))
    out[order[keep]] = w[keep]
    return out, order


def sample(logits, u, **kw):
    """(token, logp) of one row."""
    k = kept(logits, **kw)
    if k is None:
        l = np.array(logits, dtype=np.float64)
        if kw.get("exclude", -1) >= 0:
            l[kw["exclude"]] = -np.inf
        return -1, np.nan if np.isnan(l).any() else -np.inf
    w = k[0]
    cum = np.cumsum(w)
    i = int(np.searchsorted(cum, u * cum[-1], side="right"))
    i = min(i, int(np.flatnonzero(w)[-1]))
    while w[i] == 0:
        i -= 1
    return i, float(np.log(w[i] / cum[-1]))


def safe(logits, u, tol=2.0**-28, **kw):
    """Whether the token of a row cannot change where weights and sums are off by tol of what they are: no border of the draw,
    of top_p or of min_p is as near."""
    k = kept(logits, **kw)
    if k is None or not kw.get("temperature", 1.0) > 0:
        return True
    w, order = k
    cum = np.cumsum(w)
    if np.abs(cum - u * cum[-1]).min() <= tol * cum[-1] and u > 0:
        return False
    if kw.get("min_p", 0) > 0 or kw.get("top_p", 1.0) < 1:
        kw2 = dict(kw, min_p=0.0, top_p=1.0)
        w1 = kept(logits, **kw2)[0][order]
        if kw.get("top_p", 1.0) < 1:
            c = np.cumsum(w1)
            if np.abs(c - kw["top_p"] * c[-1]).min() <= tol * c[-1]:
                return False
        if kw.get("min_p", 0) > 0 and np.abs(w1 / kw["min_p"] - 1).min() <= tol:
            return False
    return True
