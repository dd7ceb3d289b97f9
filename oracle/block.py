"""What stands between a block's linears, in 64 bits: norm to MXINT, low-rank adapters, a 4-bit cache and its attention.

TEST INFRASTRUCTURE ONLY (see oracle/__init__.py).
"""
from __future__ import annotations

import numpy as np

from . import mxint


def rmsnorm(h, weight, eps):
    """h / sqrt(mean(h^2) + eps) * weight along the last axis; a row of zeros stays zero."""
    h = np.asarray(h, np.float64)
    m = np.mean(h * h, axis=-1, keepdims=True) + eps
    return h * np.where(m > 0, 1.0 / np.sqrt(np.where(m > 0, m, 1.0)), 0.0) * np.asarray(weight, np.float64)


def adapters(X, ids, A, B, Y, ranks=None, scales=None):
    """Y + scales[a] (X A_a^T) B_a^T for every row's adapter a (none outside [0, n)); and the sum of magnitudes of what is added."""
    X, Y = np.asarray(X, np.float64), np.array(Y, np.float64)
    mag = np.zeros_like(Y)
    n, R = A.shape[:2]
    for a in range(n):
        rows = np.nonzero(np.asarray(ids) == a)[0]
        r = R if ranks is None else min(max(int(ranks[a]), 0), R)
        if rows.size == 0 or r == 0:
            continue
        s = 1.0 if scales is None else float(scales[a])
        Aa, Ba = np.asarray(A[a, :r], np.float64), np.asarray(B[a, :, :r], np.float64)
        Y[rows] += s * ((X[rows] @ Aa.T) @ Ba.T)
        mag[rows] += abs(s) * ((np.abs(X[rows]) @ np.abs(Aa).T) @ np.abs(Ba).T)
    return Y, mag
