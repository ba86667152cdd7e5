"""CPU oracle, part 4: rows in 8-bit integers and the operators on them (test infrastructure only; nothing in the product path
imports this).

A row t in 8 bits: scale = max|t| / 127 (1 where that is zero), code = the integer nearest to t / scale, ties to even, clamped to
+-127, decided in fp32; a row with a NaN or an infinity has the scale NaN and codes 0.  The row stands for code x scale.
"""
from __future__ import annotations

import numpy as np

F32 = np.float32


def quantize_rows(t):
    """t [..., d] -> (codes int8 [..., d], scale fp32 [...]), the decision in fp32 on the fp32 values of t."""
    t = np.asarray(t, dtype=F32)
    bad = ~np.isfinite(t).all(axis=-1)
    amax = np.where(bad, F32(0), np.max(np.abs(np.where(np.isfinite(t), t, 0)), axis=-1)).astype(F32)
    scale = (amax / F32(127)).astype(F32)
    scale = np.where(scale > 0, scale, F32(1)).astype(F32)
    with np.errstate(over="ignore", invalid="ignore"):
        q = np.rint((t / scale[..., None]).astype(F32))
    codes = np.where(bad[..., None], 0, np.clip(q, -127, 127))
    return codes.astype(np.int8), np.where(bad, F32(np.nan), scale).astype(F32)


def rmsnorm_rows(x, delta, gain, eps):
    """x' = x + delta in fp32; codes of x' * gain; the norm's factor, in 64 bits, goes into the scale (float64), but for a row without a code
    other than zero, which keeps the scale 1."""
    x = np.asarray(x, dtype=F32)
    if delta is not None:
        x = (x + np.asarray(delta, dtype=F32)).astype(F32)
    with np.errstate(over="ignore", invalid="ignore", divide="ignore"):
        codes, s = quantize_rows((x * np.asarray(gain, dtype=F32)).astype(F32))
        x64 = x.astype(np.float64)
        factor = 1.0 / np.sqrt((x64 * x64).mean(axis=-1) + eps)
        empty = ~codes.any(axis=-1) & (s == 1)
        return x, codes, np.where(empty, 1.0, s.astype(np.float64) * factor)


def swiglu_rows(gate_up):
    """SiLU(gate) * up of rows [gate | up], in 64 bits."""
    g, u = np.split(np.asarray(gate_up, dtype=np.float64), 2, axis=-1)
    return g / (1.0 + np.exp(-g)) * u


def linear(codes, scales, w_codes, w_scales):
    """Exact sums (as float64: every partial sum is an integer below 2^53) and the scaled product in 64 bits."""
    sums = np.asarray(codes, dtype=np.float64) @ np.asarray(w_codes, dtype=np.float64).T
    return sums, sums * np.asarray(scales, dtype=np.float64)[:, None] * np.asarray(w_scales, dtype=np.float64)[None, :]


def roundtrip_rows(t):
    """What the rows stand for once they are in 8 bits, in 64 bits (code x scale)."""
    codes, scale = quantize_rows(t)
    return codes.astype(np.float64) * scale.astype(np.float64)[..., None]
