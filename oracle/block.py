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


# ---- the 4-bit cache --------------------------------------------------------------------------------------------------------
KV4_MAX_EXP = 247          # larger block maxima saturate


def kv4_quantize(v):
    """MXINT4 of [.., D]: codes int8 [.., D] and exponent bytes [.., D / 16], the bytes at most KV4_MAX_EXP."""
    v = np.asarray(v, np.float64)
    b = v.reshape(*v.shape[:-1], v.shape[-1] // 16, 16)
    e = np.minimum(mxint.block_exponent(np.abs(b).max(-1)), KV4_MAX_EXP - 127)
    codes = np.clip(np.rint(np.ldexp(b, (2 - e)[..., None])), -7, 7).astype(np.int8)
    return codes.reshape(v.shape), (e + 127).astype(np.uint8)


def kv4_values(codes, exps):
    b = np.asarray(codes, np.float64).reshape(*exps.shape, 16)
    return np.ldexp(b, exps.astype(np.int64)[..., None] - 129).reshape(codes.shape)


def kv4_words(codes):
    """codes [.., D] -> the bytes of their words [.., D / 8, 4]"""
    c = np.asarray(codes).reshape(*codes.shape[:-1], codes.shape[-1] // 8, 8).astype(np.int16)
    mag, neg = np.abs(c), (c < 0).astype(np.int16)
    out = np.zeros(c.shape[:-1] + (4,), np.int16)
    for i in range(4):
        out[..., i] = mag[..., i] | (neg[..., 4 + (i + 3) % 4] << 3) | (mag[..., 4 + i] << 4) | (neg[..., i] << 7)
    return out.astype(np.uint8)


def kv4_store(pool, P, D, page, head, off, which, codes, exps):
    """One token's codes and exponents into a pool uint8 [pages][heads][P D 9 / 8]; which: 0 keys, 1 values."""
    rec = pool[page, head]
    w = kv4_words(codes)
    if which == 0:
        rec[off * D // 2: (off + 1) * D // 2] = w.reshape(-1)
        rec[P * D + off * D // 16: P * D + (off + 1) * D // 16] = exps
        return
    cells = rec[P * D // 2: P * D].reshape(P // 4, D // 8, 4, 4)
    cells[off // 4, :, off % 4] = w
    rec[P * D * 17 // 16:].reshape(P // 4, D // 16, 4)[off // 4, :, off % 4] = exps


def attention(q, K, V, scale, begin, end, seen=None):
    """One head: q [n][D], K and V [t][D]; query i sees the tokens begin[i] .. end[i] - 1 (of `seen`, where given).  Returns the output and
    the sum of weight times |V|; 0 for a query that sees nothing."""
    out, mag = np.zeros(q.shape), np.zeros(q.shape)
    for i in range(q.shape[0]):
        t = np.arange(max(begin[i], 0), max(min(end[i], K.shape[0]), 0))
        if seen is not None:
            t = t[seen[t]]
        if t.size == 0:
            continue
        s = (K[t] @ q[i]) * scale
        w = np.exp(s - s.max())
        w /= w.sum()
        out[i], mag[i] = w @ V[t], w @ np.abs(V[t])
    return out, mag
