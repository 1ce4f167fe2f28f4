"""How many bits of q and of the probabilities reach an attention row: batches that show it, bounds, and a model of the
arithmetic with a given number of bf16 terms (8 bits each) of either, against which the bounds are held.

fp32 contexts are built for three terms of both.  u = 2^-24 is fp32's rounding, big a row's scale * sum_d |q_d k_jd|
at its largest, mass its sum_j p_j |v_j|:
    logits: chains of 3 dim / 32 + 5 roundings of partial sums, which are a fifth of big or so, and two of the product
        with the scales: 2^-22 big covers them four times and more; each moves its probability by as much
    the exponential (an ulp), the sums over keys, the division and the result: 2^-20.5 mass covers 10 u
A missing third term shows as 2^-18 of a probability, or as about 2^-20 big of a logit, at random over the keys; so the
root mean square of error over bound is held to RMS_LIMIT, too, which three terms stay below by 2 and two exceed by 2.

bf16 contexts: q is exact.  The result's own rounding is 2^-9 of it.  Two terms of the probabilities: 2^-17 of
each, and fp32's roundings: 2^-15 mass covers both.  One term: 2^-9 of each and of their sum, so
2^-9 mass + 2^-9 |out| beside the result's rounding.  Where v's signs cancel, |out| is small beside mass and the two are
apart.  One term is taken over an e4m3 cache by tiles of more than 16 rows for keys in runs of 64 that all rows see."""
import numpy as np

from oracle import serve
from tests.serve_harness import Batch

RMS_LIMIT = 0.13

# the cut's kinds of work items (tests/test_gpu_attend_infinite.py names them): rows of up to 130 keys
F32 = {
    "four waves": dict(q_len=[1, 2, 1, 3, 1, 1], length=[2, 5, 9, 33, 100, 130], heads=4, kv_heads=2),
    "one wave": dict(q_len=[1] * 136, length=[2 + i % 70 for i in range(136)], heads=8, kv_heads=8),
    "64 rows": dict(q_len=[20, 30], length=[20, 100], heads=4, kv_heads=1),
}
BF16 = {
    "four waves": dict(q_len=[1, 2, 1, 2], length=[2, 8, 32, 130], heads=4, kv_heads=2),
    "one wave": dict(q_len=[1] * 136, length=[2 + 2 * (i % 35) for i in range(136)], heads=8, kv_heads=8),
    "64 rows": dict(q_len=[16, 10], length=[130, 74], heads=4, kv_heads=1),
    "128 rows": dict(q_len=[50], length=[114], heads=4, kv_heads=1),
}


def f32_batch(kind, std, fmt, dim=64):
    """Logits of some `std`: small ones show the probabilities' terms, large ones those of q."""
    b = Batch(dim=dim, page=16, dtype="f32", fmt=fmt, seed=11, **F32[kind])
    b.q = (b.q * std).astype(np.float32).astype(np.float64)
    return b


def bf16_batch(kind, fmt, dim=64):
    """Nearly equal probabilities and v = +1, -1 in turn: the result is a few thousandths of mass."""
    b = Batch(dim=dim, page=16, dtype="bf16", fmt=fmt, seed=12, **BF16[kind])
    b.q = b.q * 2.0 ** -9
    rng = np.random.default_rng(5)
    for a in b.v:
        sign = np.where(rng.random(a.shape[1:]) < 0.5, -1.0, 1.0)
        a[:] = np.where(np.arange(len(a)) % 2 == 0, 1.0, -1.0)[:, None, None] * sign
    return b


def rows_of(b, every):
    return sorted({0, b.T - 1, *range(0, b.T, every)})


def ratios_f32(b, got, rows):
    """error / ((2^-22 big + 2^-20.5) mass) of every element."""
    out = []
    for t in rows:
        k, v = b.row_keys(t)
        for h in range(b.heads):
            g = h // (b.heads // b.kv_heads)
            ref, mass, big = serve.attend(b.q[t, h], k[:, g], v[:, g], b.scale)
            out.append(np.abs(got[t, h] - ref) / ((2.0 ** -22 * big + 2.0 ** -20.5) * mass + 1e-30))
    return np.concatenate(out)


def ratios_bf16(b, got, rows, terms):
    """error / the bound for `terms` terms of the probabilities."""
    out = []
    for t in rows:
        k, v = b.row_keys(t)
        for h in range(b.heads):
            g = h // (b.heads // b.kv_heads)
            ref, mass, _ = serve.attend(b.q[t, h], k[:, g], v[:, g], b.scale)
            bound = (2.0 ** -9 * np.abs(ref) + 2.0 ** -15 * mass if terms == 2 else
                     2.0 ** -8 * np.abs(ref) + (2.0 ** -9 + 2.0 ** -15) * mass)
            out.append(np.abs(got[t, h] - ref) / (bound + 1e-30))
    return np.concatenate(out)


# ---- the model -------------------------------------------------------------------
def _bf16(x):
    u = np.ascontiguousarray(x, np.float32).view(np.uint32).astype(np.uint64)
    return (((u + 0x7fff + ((u >> 16) & 1)) >> 16 << 16).astype(np.uint32)).view(np.float32)


def _terms(x, n):
    out, r = [], np.asarray(x, np.float32)
    for _ in range(n):
        out.append(_bf16(r))
        r = r - out[-1]
    return out


def model(b, rows, q_terms, p_terms):
    """The kernels' arithmetic in fp32, with terms of q and of the probabilities; [T][heads][dim], other rows NaN."""
    f = np.float32
    got = np.full((b.T, b.heads, b.dim), np.nan)
    for t in rows:
        k, v = b.row_keys(t)
        for h in range(b.heads):
            g = h // (b.heads // b.kv_heads)
            kk, vv = k[:, g].astype(f), v[:, g].astype(f)
            s = np.zeros(len(kk), f)
            for q in _terms(b.q[t, h], q_terms):
                s = s + kk @ q
            y = s * f(b.scale * 1.4426950408889634)
            p = np.exp2(y - y.max()).astype(f)
            parts = _terms(p, p_terms)
            # (one term: the sum is that of the rounded ones)
            total = (parts[0] if p_terms == 1 else p).sum(dtype=f)
            o = np.zeros(b.dim, f)
            for x in parts:
                o = o + x @ vv
            got[t, h] = o * (f(1) / total)
            if b.dtype == "bf16":
                got[t, h] = _bf16(got[t, h])
    return got
