"""CPU oracle of the operators around the apply: the base product in 8 bits, the 8-bit
KV cache, and attention over it (include/salt.h gives the definitions).

TEST INFRASTRUCTURE ONLY, like ``ref.py``.  float64 numpy; the scales, their
reciprocals and the products that are rounded to codes are the fp32 numbers the
definitions name, everything behind the codes is float64.
"""
from __future__ import annotations

import numpy as np

BLOCK = 128


def round_e4m3(v: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value (ties to even): three fraction bits, steps of 2^-9 below 2^-6.  |v| <= 448."""
    v = np.asarray(v, np.float64)
    _, e = np.frexp(v)
    step = np.ldexp(1.0, np.maximum(e - 1, -6) - 3)
    with np.errstate(invalid="ignore"):
        return np.rint(v / step) * step


def e4m3_value(code: np.ndarray) -> np.ndarray:
    """Values of 8-bit codes (0x7f and 0xff: NaN)."""
    c = np.asarray(code).astype(np.int64)
    e, m = (c >> 3) & 15, c & 7
    v = np.where(e > 0, np.ldexp(8.0 + m, e - 10), np.ldexp(m.astype(np.float64), -9))
    v = np.where((c & 127) == 127, np.nan, v)
    return np.where(c & 128, -v, v)


def _f32(a):
    return np.asarray(a, np.float64).astype(np.float32)


def quantise_block(v: np.ndarray) -> np.ndarray:
    """code * scale (float64) of one block; NaN throughout where a value is not finite."""
    v = np.asarray(v, np.float64)
    if not np.isfinite(v).all():
        return np.full(v.shape, np.nan)
    amax = float(np.abs(v).max()) if v.size else 0.0
    with np.errstate(over="ignore", invalid="ignore"):
        s = np.maximum(_f32(np.float64(np.float32(amax)) * np.float64(np.float32(1.0 / 448.0))), np.float32(2.0 ** -126))
        r = _f32(1.0 / np.float64(s))
        q = round_e4m3(_f32(v * np.float64(r)).astype(np.float64))
        return q * np.float64(s)


def quantise_weight(w: np.ndarray) -> np.ndarray:
    """The base weight [in][out] as it is held (blocks of 128 x 128)."""
    out = np.empty(w.shape, np.float64)
    for k in range(0, w.shape[0], BLOCK):
        for n in range(0, w.shape[1], BLOCK):
            out[k:k + BLOCK, n:n + BLOCK] = quantise_block(w[k:k + BLOCK, n:n + BLOCK])
    return out


def quantise_x(x: np.ndarray) -> np.ndarray:
    """Activations [T][in] as the product sees them (per token, blocks of 128 inputs)."""
    out = np.empty(x.shape, np.float64)
    for t in range(x.shape[0]):
        for k in range(0, x.shape[1], BLOCK):
            out[t, k:k + BLOCK] = quantise_block(x[t, k:k + BLOCK])
    return out


def quantise_kv(x: np.ndarray, fmt: str) -> np.ndarray:
    """code * scale of vectors along the last axis; NaN throughout where a value is not finite."""
    x = np.asarray(x, np.float64)
    bad = ~np.isfinite(x).all(-1, keepdims=True)
    x = np.where(bad, 0.0, x)
    amax = np.abs(x).max(-1, keepdims=True)
    if fmt == "int8":
        s = np.maximum(_f32(amax * np.float64(np.float32(1.0 / 127.0))), np.float32(2.0 ** -100)).astype(np.float64)
        r = _f32(1.0 / s).astype(np.float64)
        q = np.clip(np.rint(_f32(x * r).astype(np.float64)), -127, 127)
    else:
        m, e = np.frexp(amax)
        e = np.where(amax > 0, np.maximum(e - 9 + (m > 0.875), -100), 0)
        s = np.ldexp(1.0, e)
        q = round_e4m3(x / s)
    return np.where(bad, np.nan, q * s)


def attend(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """One query row [D] over keys k [n][D], v [n][D].  Returns (out, sum_j p_j |v_j|, largest
    scale * sum_d |q_d k_jd|); zeros without keys."""
    if k.shape[0] == 0:
        return np.zeros(q.shape[-1]), np.zeros(q.shape[-1]), 0.0
    with np.errstate(invalid="ignore", over="ignore"):
        s = scale * (k @ q)
        p = np.exp(s - s.max())
        p /= p.sum()
        return p @ v, p @ np.abs(v), float(scale * (np.abs(k) @ np.abs(q)).max())
