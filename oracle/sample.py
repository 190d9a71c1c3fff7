"""The sampler in float64 (include/ssd.h, ssd_sample), one row at a time.
Test infrastructure only."""
from __future__ import annotations

import numpy as np

# Relative error of a float32 weight 2^(-(M - x) c): the exponent is at most 32
# and its three roundings (the difference, c, the product) are 2^-24 each, so
# 32 * 3 * 2^-24 * ln 2 = 4e-6, and exp2 adds 2^-22; doubled.
WEIGHT_ERR = 1e-5


def sample_row(x, temperature, top_k, top_p, min_p, u):
    """dict(tok, prob, kept, lo, hi, ids, cum): the token, its probability and
    the kept count; lo and hi bound the kept count where a cut is within the
    weights' error; ids the entries kept (of the upper bound), cum the running
    sums of their weights in vocabulary order (of the kept count)."""
    x = np.where(np.isnan(x), -np.inf, np.asarray(x, np.float64))
    V = len(x)
    top = x.max()
    if top == -np.inf:
        return dict(tok=-1, prob=0.0, kept=0, lo=0, hi=0, ids=np.zeros(0, int), cum=np.zeros(0))
    order = np.argsort(-x, kind="stable")
    if temperature == 0 or top_k == 1:
        return dict(tok=int(order[0]), prob=1.0, kept=1, lo=1, hi=1, ids=order[:1], cum=np.ones(1))
    with np.errstate(invalid="ignore"):
        w = np.where(x == top, 1.0, np.exp2(-(top - x) * np.log2(np.e) / temperature))
    W = np.rint(w * 2.0 ** 31)[order]
    k = top_k if 0 < top_k < V else V
    W[k:] = 0
    total = W.sum()
    before = np.cumsum(W) - W

    def count(e):
        ok = (W > 0) & (w[order] >= min_p * (1 - e))
        if top_p < 1.0:
            ok &= before < top_p * total * (1 + e)
        return max(1, int(ok.sum()))

    # the sums carry the weights' relative error and half a unit for each entry
    err = WEIGHT_ERR + 0.5 * min(k, V) / total
    n, lo, hi = count(0.0), count(-err), count(err)
    ids = np.sort(order[:n])
    full = np.zeros(V)
    full[order] = W
    cum = np.cumsum(full[ids])
    at = min(int(np.searchsorted(cum, np.floor(u * cum[-1]), side="right")), n - 1)
    return dict(tok=int(ids[at]), prob=float(full[ids[at]] / cum[-1]), kept=n, lo=lo, hi=hi,
                ids=np.sort(order[:hi]), cum=cum)
