"""The 8-bit products in float64, from their definitions (include/ssd.h), one
block of 128 after the other.  Test infrastructure only."""
from __future__ import annotations

import numpy as np

from oracle.cache import LEAST, TOP

GROUP = 128


def quantize(x, block_rows):
    """x [rows, K]: (what the entries stand for before rounding, over their scale [rows, K];
    the scales [ceil(K / 128), ceil(rows / block_rows)])."""
    rows, K = x.shape
    R, C = -(-rows // block_rows), -(-K // GROUP)
    want, scale = np.empty(x.shape), np.empty((C, R))
    for i in range(R):
        for j in range(C):
            at = np.s_[i * block_rows:(i + 1) * block_rows, j * GROUP:(j + 1) * GROUP]
            b = x[at]
            m = np.abs(b[np.isfinite(b)]).max(initial=0.0)
            scale[j, i] = max(m, LEAST) / TOP
            want[at] = np.clip(b / scale[j, i], -TOP, TOP)
    return want, scale


def matmul(a, a_scale, w, w_scale, add=None):
    """a [M, K], w [N, K] the entries, a_scale [C, M], w_scale [C, ceil(N / 128)].  Returns the
    products and the sum of their terms' magnitudes."""
    M, N = len(a), len(w)
    y, mag = np.zeros((M, N)), np.zeros((M, N))
    col = np.arange(N) // GROUP
    for j in range(a_scale.shape[0]):
        at = np.s_[:, j * GROUP:(j + 1) * GROUP]
        x, z = a[at] * a_scale[j][:, None], w[at] * w_scale[j][col][:, None]
        y += x @ z.T
        mag += np.abs(x) @ np.abs(z).T
    if add is not None:
        y, mag = y + add, mag + np.abs(add)
    return y, mag
