"""Sampling rules and low-rank adapters in 64 bits (test infrastructure).

kept / draw follow the definition word by word: a row's ids in order of descending logit
(equal logits: ascending id), every part of the rule a prefix of that order, the shortest
one kept; the draw is the first id, ascending, at which the running sum of the kept
weights exp((z - max) / T) passes u times their sum.
"""
from __future__ import annotations

import numpy as np

LARGEST = float(np.finfo(np.float32).max)


def sane(z: np.ndarray) -> np.ndarray:
    """NaN as -inf, +inf as the largest finite float; float64."""
    z = np.asarray(z, dtype=np.float64)
    return np.where(np.isnan(z), -np.inf, np.minimum(z, LARGEST))


def counts_as(T: float) -> float:
    """A temperature above 0 and below 1e-30 is 1e-30."""
    return max(T, 1e-30) if T > 0 else T


def order_of(z: np.ndarray) -> np.ndarray:
    """The ids with a finite logit in the rule's order."""
    o = np.argsort(-z, kind="stable")
    return o[np.isfinite(z[o])]


def kept(z: np.ndarray, T: float, top_k: int = 0, top_p: float = 1.0, min_p: float = 0.0) -> np.ndarray:
    """Kept ids of one row, in the rule's order.  T, top_p, min_p as float32 holds them."""
    T, top_p, min_p = (float(np.float32(v)) for v in (counts_as(T), top_p, min_p))
    z = sane(z)
    o = order_of(z)
    if len(o) == 0 or not T > 0:
        return o[:1]
    w = np.exp((z[o] - z[o[0]]) / T)
    n = min(top_k, len(o)) if top_k > 0 else len(o)
    if top_p < 1:
        cum = np.cumsum(w[:n])
        n = min(n, 1 + int(np.sum(cum < top_p * cum[-1])))
    if min_p > 0:
        n = min(n, int(np.sum((z[o] - z[o[0]]) / T >= np.log(min(min_p, 1.0)))))
    return o[:n]


def mask(z: np.ndarray, *rule) -> np.ndarray:
    out = np.full(len(z), -np.inf)
    ids = kept(z, *rule)
    out[ids] = sane(z)[ids]
    return out


def draw(z: np.ndarray, u: float, T: float, *rule) -> int:
    ids = np.sort(kept(z, T, *rule))
    if len(ids) == 0:
        return -1
    z = sane(z)[ids]
    w = np.exp((z - z.max()) / float(np.float32(counts_as(T)))) if T > 0 else np.ones(1)
    cum = np.cumsum(w)
    return int(ids[np.argmax(cum > float(u) * cum[-1])])


def lora(x, a, b, ids, scales=None, ranks=None, base=None):
    """y = base + scale (x A^T) B^T row by row, and the sum of the absolute values of all
    products (what a rounding bound is a multiple of)."""
    x, a, b = (np.asarray(v, dtype=np.float64) for v in (x, a, b))
    y = np.zeros((len(x), b.shape[1])) if base is None else np.array(base, dtype=np.float64)
    size = np.abs(y)
    for r, i in enumerate(ids):
        if not 0 <= i < len(a):
            continue
        rk = a.shape[1] if ranks is None else min(max(int(ranks[i]), 0), a.shape[1])
        s = 1.0 if scales is None else float(scales[i])
        y[r] += s * (b[i, :, :rk] @ (a[i, :rk] @ x[r]))
        size[r] += abs(s) * (np.abs(b[i, :, :rk]) @ (np.abs(a[i, :rk]) @ np.abs(x[r])))
    return y, size
