"""CPU oracle, part 5: matrices in 4 bits and the products with them (test infrastructure only; nothing in the product path imports this).

An element is a code q of 0 .. 15; `group` consecutive features of a row share a scale s and a zero point z (8 where there are none), and it
stands for (q - z) * s.
"""
from __future__ import annotations

import numpy as np

from .medusa import round_to_storage

F32 = np.float32


def _groups(k, group):
    return [slice(a, min(a + group, k)) for a in range(0, k, group)]


def quantize(w, group, zeros, dtype):
    """w [n, k] (values of dtype) -> codes uint8 [n, k], scales (float64, values of dtype) [n, groups], zero points uint8 [n, groups]; the decisions
    in fp32 on the rounded scale."""
    w = np.asarray(w, dtype=F32)
    n, k = w.shape
    cut = _groups(k, group)
    codes, scales, points = np.full((n, k), 8, np.uint8), np.zeros((n, len(cut))), np.full((n, len(cut)), 8, np.uint8)
    for g, at in enumerate(cut):
        v = w[:, at]
        bad = ~np.isfinite(v).all(axis=1)
        lo, hi = np.minimum(np.where(bad, F32(0), v.min(axis=1)), F32(0)), np.maximum(np.where(bad, F32(0), v.max(axis=1)), F32(0))
        s = (hi / F32(15) - lo / F32(15)).astype(F32) if zeros else (np.maximum(hi, np.abs(lo)) / F32(7)).astype(F32)
        s = round_to_storage(s, dtype).astype(F32)
        some = (s > 0) & ~bad
        div = np.where(some, s, F32(1))
        z = np.where(some, np.clip(np.rint((-lo / div).astype(F32)), 0, 15), 8).astype(F32) if zeros else np.full(n, 8, F32)
        with np.errstate(invalid="ignore"):
            q = np.clip(np.rint((v / div[:, None]).astype(F32)) + z[:, None], 0, 15)
        codes[:, at] = np.where(some[:, None], q, 8)
        scales[:, g], points[:, g] = np.where(bad, np.nan, s), z
    return codes, scales, points


def values(codes, scales, zeros, group):
    """What the codes stand for, in 64 bits."""
    k = codes.shape[1]
    spread = lambda t: np.repeat(np.asarray(t, dtype=np.float64), group, axis=1)[:, :k]  # noqa: E731
    return (codes.astype(np.float64) - (8.0 if zeros is None else spread(zeros))) * spread(scales)


def linear(x, w):
    return np.asarray(x, dtype=np.float64) @ w.T


def swiglu(x, gate, up):
    g = linear(x, gate)
    return g / (1.0 + np.exp(-g)) * linear(x, up)
