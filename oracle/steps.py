"""CPU oracle of a decoding server's operators: rotation of heads, gathered weights, eviction, beam search
(include/salt.h gives the definitions).

TEST INFRASTRUCTURE ONLY, like ``ref.py``.  float64 numpy.
"""
from __future__ import annotations

import numpy as np


def rotate(x: np.ndarray, pos: np.ndarray, freq: np.ndarray, interleaved: bool, norm=None, eps: float = 0.0,
           gain: float = 1.0):
    """Heads x [T][heads][D] at pos [T].  Returns (out, the length of each value's pair, or its own size)."""
    x = np.asarray(x, np.float64)
    rot = 2 * len(freq)
    v = x
    if norm is not None:
        v = x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * np.asarray(norm, np.float64)
    t = (np.asarray(pos, np.longdouble)[:, None] * np.asarray(freq, np.longdouble))[:, None, :]
    c, s = np.cos(t).astype(np.float64), np.sin(t).astype(np.float64)
    one, two = (slice(0, rot, 2), slice(1, rot, 2)) if interleaved else (slice(0, rot // 2), slice(rot // 2, rot))
    out, size = v.copy(), np.abs(v)
    a, b = v[..., one], v[..., two]
    out[..., one], out[..., two] = gain * (a * c - b * s), gain * (b * c + a * s)
    size[..., one] = size[..., two] = abs(gain) * np.hypot(a, b)
    return out, size


def weights(q: np.ndarray, k: np.ndarray, scale: float):
    """One query row [D] over the keys it sees [n][D]: softmax, and the largest scale * sum_d |q_d k_jd|.  NaN
    throughout where a logit is NaN or +inf, or none is above -inf."""
    with np.errstate(invalid="ignore", over="ignore"):
        s = scale * (k @ q)
        p = np.exp(s - s.max())
        return p / p.sum(), float(scale * (np.abs(k) @ np.abs(q)).max())


def evict(weight: np.ndarray, pos: np.ndarray, keep: int, recent: int) -> np.ndarray:
    """Where the tokens of one sequence and kv head come from that stand at places 0 .. keep - 1 afterwards."""
    n = len(weight)
    if n <= keep:
        return np.arange(n)
    pos = np.asarray(pos, np.int64)
    new = pos > pos.max() - recent
    w = np.asarray(weight, np.float64)
    # protected ones alike, then NaN, then by weight: ties by place
    rank = [(0 if new[i] else 1 if np.isnan(w[i]) else 2, 0.0 if new[i] or np.isnan(w[i]) else -w[i], i) for i in range(n)]
    stays = np.zeros(n, bool)
    stays[[r[2] for r in sorted(rank)[:keep]]] = True
    src = np.arange(keep)
    src[~stays[:keep]] = keep + np.flatnonzero(stays[keep:])
    return src


def beam_worth(logits: np.ndarray, score: np.ndarray) -> np.ndarray:
    """[width][vocab]: the worth of every continuation; -inf for what is not one."""
    x = np.asarray(logits, np.float64)
    out = np.full(x.shape, -np.inf)
    for b in range(len(x)):
        if not np.isfinite(score[b]) or np.isnan(x[b]).any() or x[b].max() == np.inf or x[b].max() == -np.inf:
            continue
        m = x[b].max()
        out[b] = float(score[b]) + x[b] - (m + np.log(np.exp(x[b] - m).sum()))
    return out


def beam_select(worth: np.ndarray, n_out: int):
    """(worth, beam, token) of the n_out best: ties by the lower beam, then the lower token."""
    width, vocab = worth.shape
    order = np.argsort(-worth.reshape(-1), kind="stable")[:n_out]
    order = order[worth.reshape(-1)[order] > -np.inf]
    value, beam, token = np.full(n_out, -np.inf), np.full(n_out, -1), np.full(n_out, -1)
    value[: len(order)], beam[: len(order)], token[: len(order)] = worth.reshape(-1)[order], order // vocab, order % vocab
    return value, beam, token
