"""CPU oracle for the pick of a token (``include/misample.h``).

TEST INFRASTRUCTURE ONLY, like the rest of this package: numpy, a row at a time, from the definition, in 80 bits where
the machine has them; no code shared with the HIP path.
"""
from __future__ import annotations

import math

import numpy as np

LD = np.longdouble


def pick(x, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, logprob, margin) of logits x (1-d, any float type holds them exactly).  margin: how near u's place is to a
    border of the token drawn, or top_p's to one that moves the end of what is kept, as a share of the sum."""
    x = np.asarray(x, dtype=np.float64)
    n = len(x)
    if np.isnan(x).any() or (x == np.inf).any() or (x == -np.inf).all():
        return -1, math.nan, 1.0
    order = np.lexsort((np.arange(n), -x))
    if not temperature > 0:
        return int(order[0]), 0.0, 1.0
    with np.errstate(all="ignore"):
        w = np.exp((x.astype(LD) - LD(x.max())) / LD(temperature))
    w[x == -np.inf] = 0
    w[x == x.max()] = 1
    share, grain = w, LD(2.0) ** -min(51, 62 - (n - 1).bit_length())
    w = np.rint(w / grain) * grain                  # held as multiples of a power of two
    kept = order[:top_k] if 0 < top_k < n else order
    margin = 1.0
    if top_p < 1:
        s = w[kept].cumsum()
        before = np.concatenate(([LD(0)], s[:-1]))
        most = LD(top_p) * s[-1]
        c = max(1, int((before < most).sum()))
        if top_p > 0:
            margin = min(margin, float(np.abs(before[max(0, c - 1):c + 1] - most).min() / s[-1]))
        kept = kept[:c]
    if min_p > 0:
        kept = np.concatenate((kept[:1], kept[1:][share[kept[1:]] >= min_p]))
    kept = np.sort(kept[w[kept] > 0])
    s = w[kept].cumsum()
    u = min(max(u, 0.0), 1 - 2.0 ** -24) if u == u else 0.0
    target = LD(u) * s[-1]
    i = int((s <= target).sum())
    edges = np.array([s[i - 1] if i else LD(-1), s[i]])
    margin = min(margin, float(np.abs(edges - target).min() / s[-1]))
    t = int(kept[i])
    return t, float((LD(x[t]) - LD(x.max())) / LD(temperature) - np.log(s[-1])), margin
