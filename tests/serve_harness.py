"""Test-side driver of the base product, the KV cache and the attention: makes batches, runs
them through libsalt, and holds the same batch for the float64 oracle (oracle/serve.py)."""
from __future__ import annotations

import numpy as np

import oracle
from oracle import serve


def hipmod():
    from paper_2608_03579_amd import hip
    return hip


def store(a: np.ndarray, dtype: str) -> np.ndarray:
    """float64 values in storage form (bf16: rounded to nearest even, as uint16 bits)."""
    a32 = np.ascontiguousarray(a, np.float32)
    if dtype == "f32":
        return a32
    u = a32.view(np.uint32).astype(np.uint64)
    r = (u + 0x7fff + ((u >> 16) & 1)) >> 16
    return np.where(np.isnan(a32), 0x7fc0, r).astype(np.uint16)


def values(shape, seed, dtype, std=1.0, uneven=False) -> np.ndarray:
    """Seeded N(0, std^2) numbers that the dtype holds exactly, as float64; `uneven`: some columns 8 times larger."""
    rng = np.random.default_rng([97, int(seed)])
    v = rng.standard_normal(shape) * std
    if uneven:
        v[..., rng.integers(0, shape[-1], max(1, shape[-1] // 32))] *= 8.0
    return oracle.decode(store(v, dtype), dtype)


def to_dev(a: np.ndarray):
    return hipmod().DeviceArray.from_host(np.ascontiguousarray(a))


class Batch:
    """Sequences and domains with page tables in a random order; k and v of every token, float64."""

    def __init__(self, q_len, length, prefix=(), domain=None, heads=8, kv_heads=2, dim=128, page=16, fmt="e4m3",
                 dtype="bf16", layers=1, seed=0, spare=2):
        self.q_len, self.length = np.asarray(q_len, np.int32), np.asarray(length, np.int32)
        self.prefix = np.asarray(prefix, np.int32)
        self.domain = None if domain is None else np.asarray(domain, np.int32)
        self.heads, self.kv_heads, self.dim, self.page, self.fmt, self.dtype = heads, kv_heads, dim, page, fmt, dtype
        self.layers, self.seed, self.T = layers, seed, int(self.q_len.sum())
        rng = np.random.default_rng([98, seed])
        n_own, n_pre = -(-self.length // page), -(-self.prefix // page)
        self.page_off = np.concatenate([[0], np.cumsum(n_own)]).astype(np.int32)
        self.prefix_off = np.concatenate([[0], np.cumsum(n_pre)]).astype(np.int32)
        self.n_pages = int(self.page_off[-1] + self.prefix_off[-1]) + spare
        order = rng.permutation(self.n_pages).astype(np.int32)
        self.pages = order[: self.page_off[-1]]
        self.prefix_pages = order[self.page_off[-1]: self.page_off[-1] + self.prefix_off[-1]]
        shape = lambda n: (int(n), kv_heads, dim)
        self.k = [values(shape(n), 1000 + 2 * i + seed * 7919, dtype, uneven=True) for i, n in enumerate(self.length)]
        self.v = [values(shape(n), 1001 + 2 * i + seed * 7919, dtype) for i, n in enumerate(self.length)]
        self.pk = [values(shape(n), 5000 + 2 * i + seed * 7919, dtype, uneven=True) for i, n in enumerate(self.prefix)]
        self.pv = [values(shape(n), 5001 + 2 * i + seed * 7919, dtype) for i, n in enumerate(self.prefix)]
        self.q = values((self.T, heads, dim), 9000 + seed, dtype)
        self.scale = float(np.float32(dim ** -0.5))

    # ---- libsalt -----------------------------------------------------------------
    def open(self, n_pages=None):
        from paper_2608_03579_amd import salt
        hip = hipmod()
        self.ctx = salt.Context(self.dtype, [(256, 256)], 0, 0, 1, 0, 1)
        self.kv = self.ctx.kv_cache(self.layers, self.heads, self.kv_heads, self.dim, self.page,
                                    n_pages or self.n_pages, self.fmt)
        self.stream = hip.Stream()
        n, nd = len(self.length), len(self.prefix)
        self.seqs = self.kv.seqs(max(1, n + nd), max(1, self.T), max(1, int(self.page_off[-1] + self.prefix_off[-1])))
        return self

    def close(self):
        self.ctx.close()
        self.stream.destroy()

    def set(self, seqs=None, stream=None):
        (seqs or self.seqs).set(self.q_len, self.length, self.page_off, self.pages, self.domain, self.prefix,
                                self.prefix_off, self.prefix_pages, (stream or self.stream).h)

    def fill(self, layer=0, k=None, v=None, pk=None, pv=None):
        """Every token of the prefixes and the sequences into the cache, as new tokens of sequences."""
        k, v, pk, pv = k or self.k, v or self.v, pk or self.pk, pv or self.pv
        length = np.concatenate([self.prefix, self.length])
        off = np.concatenate([self.prefix_off, self.page_off[1:] + self.prefix_off[-1]])
        pages = np.concatenate([self.prefix_pages, self.pages])
        total = int(length.sum())
        if total == 0:
            return
        fill = self.kv.seqs(len(length), total, max(1, len(pages)))
        fill.set(length, length, off, pages, stream=self.stream.h)
        kd = to_dev(store(np.concatenate(list(pk) + list(k)), self.dtype))
        vd = to_dev(store(np.concatenate(list(pv) + list(v)), self.dtype))
        fill.write(layer, kd.ptr, vd.ptr, self.stream.h)
        self.stream.synchronize()
        fill.close()
        kd.free()
        vd.free()

    def attend(self, layer=0, ldq=0, ldo=0, q=None):
        """out [T][heads][dim], float64; with a row length, what lies between the rows must come back untouched."""
        width = self.heads * self.dim
        sdt = np.float32 if self.dtype == "f32" else np.uint16
        qv = store(self.q if q is None else q, self.dtype).reshape(self.T, width)
        buf = np.zeros((self.T, ldq or width), sdt)
        buf[:, :width] = qv
        mark = np.full((self.T, ldo or width), 77, sdt)
        qd, od = to_dev(buf), to_dev(mark)
        self.seqs.attend(layer, qd.ptr, od.ptr, self.scale, self.stream.h, ldq, ldo)
        self.stream.synchronize()
        out = od.to_host()
        qd.free()
        od.free()
        assert np.all(out[:, width:] == 77), "attend wrote between the rows of out"
        return oracle.decode(out[:, :width], self.dtype).reshape(self.T, self.heads, self.dim)

    # ---- oracle --------------------------------------------------------------------
    def row_keys(self, t):
        """(k, v) [n][kv_heads][dim] of every key row t sees, as the cache holds them."""
        if not hasattr(self, "_held"):
            self._held = [[serve.quantise_kv(a, self.fmt) if a.size else a for a in arr]
                          for arr in (self.k, self.v, self.pk, self.pv)]
        hk, hv, hpk, hpv = self._held
        first = np.concatenate([[0], np.cumsum(self.q_len)])
        s = int(np.searchsorted(first, t, side="right") - 1)
        pos = int(self.length[s] - self.q_len[s] + t - first[s])
        n = max(0, pos + 1)
        d = -1 if self.domain is None else int(self.domain[s])
        if d < 0:
            return hk[s][:n], hv[s][:n]
        return np.concatenate([hpk[d], hk[s][:n]]), np.concatenate([hpv[d], hv[s][:n]])

    def check(self, got, rows=None):
        """Every row (or `rows`) against the oracle, within the bound of its type.

        bf16: the probabilities and the result are rounded to 9 significant bits (2^-9 of
        sum p|v|, and of the result), a quarter more for the fp32 sums.  fp32: a logit
        is a sum of dim products, 4 dim 2^-24 of its largest term sum at most, which scales its
        probability; 2^-17 for the sums, the exponential and the divisions."""
        G = self.heads // self.kv_heads
        worst = 0.0
        for t in range(self.T) if rows is None else rows:
            k, v = self.row_keys(t)
            for h in range(self.heads):
                ref, mass, big = serve.attend(self.q[t, h], k[:, h // G], v[:, h // G], self.scale)
                if not np.isfinite(ref).all():
                    assert np.isnan(got[t, h]).all(), f"row {t}, head {h}: not NaN"
                    continue
                if self.dtype == "bf16":
                    bound = 1.25 * 2.0 ** -9 * (mass + np.abs(ref))
                else:
                    bound = (4 * self.dim * 2.0 ** -24 * big + 2.0 ** -17) * mass
                err = np.abs(got[t, h] - ref)
                if k.shape[0] == 0:
                    assert np.all(got[t, h] == 0), f"row {t}, head {h} without keys is not zero"
                    continue
                ratio = float(np.max(err / (bound + 1e-30)))
                worst = max(worst, ratio)
                assert ratio <= 1.0, f"row {t}, head {h}: {ratio:.3f}x the bound ({k.shape[0]} keys)"
        return worst


