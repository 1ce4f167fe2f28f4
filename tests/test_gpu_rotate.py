"""GPU parity of salt_rotate: norms and rotation of query and key heads against float64.

Bound: of a value's pair (its own size where it is not rotated), in units of 2^-24: the norm's sum of squares 21 at most
(16 terms of a lane, five lane exchanges), halved by the root, with the division, eps, root, reciprocal and two products
17 in all; sine and cosine 5.1 each (the reduced angle rounded, pi 2^-24 at most, and 2 for the functions), the gain
1, products and sum 3: 17 + 1.42 * 6.1 + 3 < 32.  The angle: two roundings in 64 bits, 2^-52 of it, in revolutions times
2 pi.  Then half a step of the result's type."""
import numpy as np
import pytest

import oracle
from oracle import steps as o64
from paper_2608_03579_amd import salt
from tests.serve_harness import hipmod, store, to_dev, values

pytestmark = pytest.mark.gpu


def _freq(rot, base=10000.0):
    return base ** (-np.arange(0, rot, 2) / rot)


class Case:
    def __init__(self, T, heads, kv_heads, dim, rot, dtype, inter, norm, pos, seed=0, eps=1e-6, gain=1.0, std=1.0):
        self.T, self.heads, self.kv_heads, self.dim, self.dtype = T, heads, kv_heads, dim, dtype
        self.q = values((T, heads, dim), 1 + 10 * seed, dtype, std, uneven=True)
        self.k = values((T, kv_heads, dim), 2 + 10 * seed, dtype, std, uneven=True)
        self.norms = [values((dim,), 3 + i + 10 * seed, dtype) for i in range(2)] if norm else [None, None]
        self.pos, self.freq, self.inter = np.asarray(pos, np.int32), _freq(rot), inter
        self.eps, self.gain = float(np.float32(eps)), float(np.float32(gain))

    def run(self, ldq=0, ldk=0, in_place=False):
        hip = hipmod()
        sdt = np.float32 if self.dtype == "f32" else np.uint16
        ctx = salt.Context(self.dtype, [(64, 64)], 0, 0, 1, 0, 1)
        stream = hip.Stream()
        try:
            bufs, outs = [], []
            for x, ld in ((self.q, ldq), (self.k, ldk)):
                width = x.shape[1] * self.dim
                buf = np.full((self.T, ld or width), 77, sdt)
                buf[:, :width] = store(x, self.dtype).reshape(self.T, width)
                bufs.append(to_dev(buf))
                outs.append(bufs[-1] if in_place else to_dev(np.full((self.T, ld or width), 77, sdt)))
            norms = [None if n is None else to_dev(store(n, self.dtype)) for n in self.norms]
            pos = to_dev(self.pos)
            rot = ctx.rotation(self.heads, self.kv_heads, self.dim, self.freq, self.inter, norms[0].ptr if norms[0] else 0,
                               norms[1].ptr if norms[1] else 0, self.eps, self.gain)
            ctx.rotate(rot, self.T, pos.ptr, bufs[0].ptr, outs[0].ptr, bufs[1].ptr, outs[1].ptr, stream.h, ldq, ldq, ldk, ldk)
            stream.synchronize()
            res = []
            for o, x in zip(outs, (self.q, self.k)):
                a = o.to_host()
                width = x.shape[1] * self.dim
                assert np.all(a[:, width:] == 77), "values between the rows changed"
                res.append(oracle.decode(a[:, :width], self.dtype).reshape(x.shape))
            if not in_place:
                for d, x in zip(bufs, (self.q, self.k)):
                    assert np.array_equal(d.to_host()[:, : x.shape[1] * self.dim], store(x, self.dtype).reshape(self.T, -1))
            return res
        finally:
            ctx.close()
            stream.destroy()

    def check(self, got):
        for g, x, n in zip(got, (self.q, self.k), self.norms):
            want, size = o64.rotate(x, self.pos, self.freq, self.inter, n, self.eps, self.gain)
            far = np.abs(self.pos.astype(np.float64)).max(initial=0) * np.abs(self.freq).max()
            half = 2.0 ** -8 if self.dtype == "bf16" else 2.0 ** -24
            bound = (32 * 2.0 ** -24 + 2.0 ** -51 * far) * size
            bound = bound + half * (np.abs(want) + bound) + 1e-37
            err = np.abs(g - want)
            assert np.all(err <= bound), f"{float((err / bound).max()):.3f}x the bound"


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("inter", [False, True])
@pytest.mark.parametrize("dim,rot", [(8, 8), (24, 16), (64, 64), (80, 80), (96, 32), (128, 128), (128, 40), (200, 104),
                                     (256, 256), (256, 64)])
def test_head_layouts(dim, rot, inter, dtype):
    print(f"\n[gpu case] rotate {dtype} dim={dim} rot={rot} inter={inter}", flush=True)
    for norm in (False, True):
        c = Case(5, 7, 3, dim, rot, dtype, inter, norm, [0, 1, 17, 4095, 70000], gain=1.25 if norm else 1.0)
        c.check(c.run())


@pytest.mark.parametrize("T", [1, 2, 63, 300, 4200])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_token_counts_and_rows(T, dtype):
    """Rows apart, in place, and one call for the few tokens of a decode step as for a prompt."""
    print(f"\n[gpu case] rotate {dtype} T={T}", flush=True)
    c = Case(T, 6, 2, 64, 64, dtype, False, True, np.random.default_rng(T).integers(0, 1 << 17, T))
    got = c.run()
    c.check(got)
    for kw in (dict(ldq=392, ldk=136), dict(in_place=True), dict(ldq=400, ldk=128, in_place=True)):
        for a, b in zip(c.run(**kw), got):
            assert np.array_equal(a, b), kw


@pytest.mark.parametrize("far", [1 << 20, 2 ** 31 - 1, -(2 ** 31)])
def test_far_positions(far):
    print(f"\n[gpu case] rotate far={far}", flush=True)
    c = Case(4, 2, 1, 128, 128, "f32", False, False, [far, far - 1 if far > 0 else far + 1, far // 3, -5])
    c.check(c.run())


def test_position_zero_changes_nothing():
    print("\n[gpu case] rotate at 0", flush=True)
    c = Case(3, 4, 2, 64, 32, "bf16", False, False, [0, 0, 0])
    for a, b in zip(c.run(), (c.q, c.k)):
        assert np.array_equal(a, b)


def test_values_that_are_not_finite():
    """An infinity or NaN stays in its pair without a norm, and in its head with one; values behind the rotated ones
    pass as they are."""
    print("\n[gpu case] rotate not finite", flush=True)
    for norm in (False, True):
        c = Case(3, 3, 1, 64, 32, "bf16", False, norm, [3, 4, 5])
        clean = c.run()
        c.q[1, 1, 5] = np.nan
        c.q[1, 2, 40] = np.inf
        c.q[0, 0] = 0.0
        got = c.run()
        assert np.array_equal(got[1], clean[1])
        bad = np.zeros(c.q.shape, bool)
        if norm:
            bad[1, 1] = True
            assert np.all(got[0][0, 0] == 0)                       # (a head of zeros: 0 / sqrt(eps))
            assert np.isnan(got[0][1, 2, 40])                      # inf * 0
        else:
            bad[1, 1, [5, 21]] = True
            assert got[0][1, 2, 40] == np.inf
        assert np.isnan(got[0][bad]).all()
        rest = ~bad
        rest[0, 0] = rest[1, 2] = False
        assert np.array_equal(got[0][rest], clean[0][rest])


def test_one_operand_alone():
    """No key heads (or no query heads): that operand is not looked at."""
    print("\n[gpu case] rotate one operand", flush=True)
    hip = hipmod()
    c = Case(5, 4, 4, 64, 64, "f32", False, False, [1, 2, 3, 4, 5])
    want = c.run()
    ctx = salt.Context("f32", [(64, 64)], 0, 0, 1, 0, 1)
    try:
        pos = to_dev(c.pos)
        for which, (x, w) in enumerate(zip((c.q, c.k), want)):
            d, o = to_dev(store(x, "f32")), to_dev(np.zeros(x.shape, np.float32))
            rot = ctx.rotation(4 if which == 0 else 0, 4 if which else 0, 64, c.freq)
            args = (d.ptr, o.ptr, 0, 0) if which == 0 else (0, 0, d.ptr, o.ptr)
            ctx.rotate(rot, 5, pos.ptr, *args)
            hip.synchronize()
            assert np.array_equal(o.to_host(), w)
    finally:
        ctx.close()


def test_refusals_leave_the_values():
    print("\n[gpu case] rotate refusals", flush=True)
    hip = hipmod()
    ctx = salt.Context("bf16", [(64, 64)], 0, 0, 1, 0, 1)
    try:
        x, pos = to_dev(np.full((2, 192), 5, np.uint16)), to_dev(np.arange(2, dtype=np.int32))
        ok = ctx.rotation(2, 1, 64, _freq(64))
        p = x.ptr
        for rot, args in ((ctx.rotation(2, 1, 60, _freq(56)), (2, pos.ptr, p, p, p, p)),
                          (ctx.rotation(2, 1, 64, _freq(72)), (2, pos.ptr, p, p, p, p)),
                          (ctx.rotation(2, 1, 64, np.full(32, np.nan)), (2, pos.ptr, p, p, p, p)),
                          (ok, (2, 0, p, p, p, p)), (ok, (2, pos.ptr, p + 2, p, p, p)), (ok, (2, pos.ptr, p, 0, p, p))):
            assert ctx.rotate_status(rot, *args) == salt.ERR_INVALID_ARG
        assert ctx.rotate_status(ok, -1, pos.ptr, p, p, p, p) == salt.ERR_OUT_OF_RANGE
        assert ctx.rotate_status(ok, 2, pos.ptr, p, p, p, p, ldq=192, ldqo=200) == salt.ERR_INVALID_ARG
        hip.synchronize()
        assert np.all(x.to_host() == 5)
    finally:
        ctx.close()


def test_q_and_k_of_one_buffer():
    """q and k as columns of one buffer of rows (a joint projection's output), in place; v beside them stays."""
    print("\n[gpu case] rotate in one buffer", flush=True)
    c = Case(9, 4, 2, 64, 64, "bf16", False, True, np.arange(9) * 100)
    want = c.run()
    hip, ctx = hipmod(), salt.Context("bf16", [(64, 64)], 0, 0, 1, 0, 1)
    try:
        buf = np.full((9, 512), 77, np.uint16)
        buf[:, :256], buf[:, 256:384] = store(c.q, "bf16").reshape(9, -1), store(c.k, "bf16").reshape(9, -1)
        d, pos, n = to_dev(buf), to_dev(c.pos), [to_dev(store(x, "bf16")) for x in c.norms]
        rot = ctx.rotation(4, 2, 64, c.freq, False, n[0].ptr, n[1].ptr, c.eps)
        ctx.rotate(rot, 9, pos.ptr, d.ptr, d.ptr, d.ptr + 512, d.ptr + 512, 0, 512, 512, 512, 512)
        hip.synchronize()
        got = d.to_host()
        assert np.array_equal(got[:, :256], store(want[0], "bf16").reshape(9, -1))
        assert np.array_equal(got[:, 256:384], store(want[1], "bf16").reshape(9, -1)) and np.all(got[:, 384:] == 77)
    finally:
        ctx.close()
