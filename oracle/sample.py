"""Oracle of drawing a token from a row of logits, written from the definition in include/eb.h: the
order, the prefix of it that is kept, the walk over the kept ids.  Sums in extended precision."""
from __future__ import annotations

import numpy as np


def kept_ids(z, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """Ids that are kept, rising, and the weight of every id.  z: a row whose largest is finite."""
    z = np.asarray(z, np.float64)
    order = np.lexsort((np.arange(len(z)), -z))
    if temperature <= 0:
        return order[:1], np.ones(len(z), np.longdouble)
    with np.errstate(over="ignore"):
        w = np.exp((z - z.max()) / np.float64(temperature)).astype(np.longdouble)
    n = top_k if 0 < top_k < len(z) else len(z)
    if top_p < 1:
        sums = np.cumsum(w[order[:n]])
        enough = sums >= np.longdouble(max(top_p, 0.0)) * sums[-1]
        n = max(int(np.argmax(enough)) + 1, 1)
    if min_p > 0:
        n = min(n, int(np.sum(w >= np.longdouble(min(min_p, 1.0)))))
    return np.sort(order[:n]), w


def sample(z, u, temperature=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(token, prob, conf) of one row."""
    z = np.asarray(z, np.float64)
    if np.isnan(z).any() or (z == np.inf).any():
        return -1, np.nan, np.nan
    if (z == -np.inf).all():
        return -1, 0.0, 0.0
    ids, w = kept_ids(z, temperature, top_k, top_p, min_p)
    sums = np.cumsum(w[ids])
    at = int(np.argmax(sums > np.longdouble(u) * sums[-1]))
    token = int(ids[at])
    soft = np.exp((z - z.max()).astype(np.longdouble))
    return token, float(w[token] / sums[-1]), float(soft[token] / soft.sum())
