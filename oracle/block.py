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
