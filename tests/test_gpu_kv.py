"""GPU parity of the paged 8-bit KV cache (salt_kv_write, salt_kv_read): what is read back must be, bit for
bit, the oracle's code * scale rounded to the context dtype."""
import numpy as np
import pytest

import oracle
from oracle import serve
from tests.serve_harness import Batch, hipmod, store, to_dev

pytestmark = pytest.mark.gpu


def _read(b, what, rows, layer=0, ld=0):
    width = b.kv_heads * b.dim
    sdt = np.float32 if b.dtype == "f32" else np.uint16
    k, v = (to_dev(np.full((rows, ld or width), 77, sdt)) for _ in range(2))
    b.seqs.read(layer, what, k.ptr, v.ptr, b.stream.h, ld, ld)
    b.stream.synchronize()
    out = [a.to_host() for a in (k, v)]
    k.free()
    v.free()
    for a in out:
        assert np.all(a[:, width:] == 77)
    return [oracle.decode(a[:, :width], b.dtype).reshape(rows, b.kv_heads, b.dim) for a in out]


def _same(got, want, dtype):
    want = oracle.decode(store(want, dtype), dtype)
    assert np.array_equal(got, want, equal_nan=True), f"{int(np.sum(got != want))} of {got.size} values differ"


def _write_new(b, layer=0, ld=0, k=None, v=None):
    new = lambda arr: np.concatenate([a[max(0, len(a) - q):] if q <= len(a) else
                                      np.concatenate([np.full((q - len(a),) + a.shape[1:], 3.0), a])
                                      for a, q in zip(arr, b.q_len)])
    width = b.kv_heads * b.dim
    bufs = []
    for arr in (k or b.k, v or b.v):
        rows = store(new(arr), b.dtype).reshape(b.T, width)
        buf = np.full((b.T, ld or width), store(np.array([np.inf]), b.dtype)[0])
        buf[:, :width] = rows
        bufs.append(to_dev(buf))
    b.seqs.write(layer, bufs[0].ptr, bufs[1].ptr, b.stream.h, ld, ld)
    b.stream.synchronize()
    for d in bufs:
        d.free()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,kv_heads,page,ld", [(64, 1, 16, 0), (128, 3, 64, 408), (256, 2, 32, 0), (128, 8, 256, 1032)])
def test_write_and_read(dim, kv_heads, page, ld, dtype, fmt):
    print(f"\n[gpu case] kv {dtype} {fmt} dim={dim} kv={kv_heads} page={page}", flush=True)
    b = Batch([5, 1, 17, 0, 33, 1], [5, 1, 17, 9, 70, 300], kv_heads=kv_heads, heads=kv_heads, dim=dim, page=page,
              fmt=fmt, dtype=dtype, layers=2).open()
    try:
        b.fill(layer=1)
        b.set()
        k, v = _read(b, "own", int(b.length.sum()), 1, ld)
        _same(k, serve.quantise_kv(np.concatenate(b.k), fmt), dtype)
        _same(v, serve.quantise_kv(np.concatenate(b.v), fmt), dtype)
        # the step's tokens over it: other values into the same places, the rest as it was
        other = Batch(b.q_len, b.length, kv_heads=kv_heads, heads=kv_heads, dim=dim, page=page, fmt=fmt, dtype=dtype,
                      seed=5)
        _write_new(b, 1, ld, other.k, other.v)
        new = [np.concatenate([a[len(a) - q:] for a, q in zip(arr, b.q_len)]) for arr in (other.k, other.v)]
        for got, want in zip(_read(b, "new", b.T, 1, ld), new):
            _same(got, serve.quantise_kv(want, fmt), dtype)
        mixed = [np.concatenate([np.concatenate([a[: len(a) - q], o[len(o) - q:]]) for a, o, q in zip(x, y, b.q_len)])
                 for x, y in ((b.k, other.k), (b.v, other.v))]
        for got, want in zip(_read(b, "own", int(b.length.sum()), 1), mixed):
            _same(got, serve.quantise_kv(want, fmt), dtype)
        # the other layer was never written
        for got in _read(b, "own", int(b.length.sum()), 0):
            assert np.all(got == 0)
    finally:
        b.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_edges_of_the_range(dtype, fmt):
    """Zero vectors, vectors at powers of two around the scale's steps, huge and tiny ones, ties, infinities and NaN."""
    print(f"\n[gpu case] kv edges {dtype} {fmt}", flush=True)
    b = Batch([24], [24], kv_heads=1, heads=1, dim=64, page=16, fmt=fmt, dtype=dtype).open()
    try:
        k, v = b.k[0], b.v[0]
        rng = np.random.default_rng(1)
        k[0] = 0.0
        k[1, 0, 0], k[1, 0, 1:] = 448.0, 0.0
        k[2] *= 448.0 / np.abs(k[2]).max()
        k[3] *= 2.0 ** 100
        k[4] *= 2.0 ** -115
        k[5] = np.where(rng.random(k[5].shape) < 0.5, 3.4e38, -1.0)
        k[6, 0, 5] = np.nan
        k[7, 0, 63] = -np.inf
        v[8, 0, 0] = np.inf
        v[9] = np.nan
        k[10] = rng.integers(-127, 128, k[10].shape)
        k[10, 0, 0] = 127
        k[11] = (rng.integers(-127, 127, k[11].shape) + 0.5)
        k[11, 0, 0] = 127
        k[12] = 449.0 * np.sign(k[12])
        k[13] = 2.0 ** -140
        b.k[0], b.v[0] = (oracle.decode(store(a, dtype), dtype) for a in (k, v))
        b.fill()
        b.set()
        gk, gv = _read(b, "own", 24)
        wv = serve.quantise_kv(b.v[0], fmt)
        wk = np.where(np.isnan(wv).any(-1, keepdims=True), np.nan, serve.quantise_kv(b.k[0], fmt))
        _same(gk, wk, dtype)
        _same(gv, wv, dtype)
    finally:
        b.close()


def test_tokens_without_a_place_and_empty_batches():
    print("\n[gpu case] kv tokens without a place", flush=True)
    b = Batch([4, 3, 2], [2, 0, 2], kv_heads=2, heads=2, dim=64, page=16).open()
    try:
        b.set()
        _write_new(b)
        k, v = _read(b, "new", b.T)
        want = serve.quantise_kv(np.concatenate([np.zeros((2, 2, 64)), b.k[0], np.zeros((3, 2, 64)), b.k[2]]), "e4m3")
        _same(k, want, "bf16")
        b.seqs.set([], [], [0], [])
        b.seqs.write(0, 0, 0)                               # T == 0: no operand is looked at
        b.seqs.read(0, "own", 0, 0)
        b.seqs.attend(0, 0, 0, 1.0)
    finally:
        b.close()


def test_pool_offsets_past_32_bits():
    """A pool of more than 4 GiB: the last pages are read and written in their own place."""
    print("\n[gpu case] kv large pool", flush=True)
    from paper_2608_03579_amd import salt
    hip = hipmod()
    ctx = salt.Context("bf16", [(256, 256)], 0, 0, 1, 0, 1)
    try:
        n_pages = 40000
        kv = ctx.kv_cache(1, 8, 8, 128, 64, n_pages, "e4m3")            # 2.6 GB of codes each
        assert kv.nbytes > (1 << 32)
        b = Batch([40, 30, 20], [40, 30, 20], heads=8, kv_heads=8, dim=128, page=64)
        b.pages = np.array([n_pages - 1, 0, n_pages - 2], np.int32)
        b.ctx, b.kv, b.stream = ctx, kv, hip.Stream()
        b.seqs = kv.seqs(3, 90, 3)
        b.set()
        _write_new(b)
        for got, want in zip(_read(b, "own", 90), (b.k, b.v)):
            _same(got, serve.quantise_kv(np.concatenate(want), "e4m3"), "bf16")
        b.check(b.attend(), rows=[0, 39, 40, 69, 89])
        b.stream.destroy()
    finally:
        ctx.close()


def test_refusals():
    print("\n[gpu case] kv refusals", flush=True)
    from paper_2608_03579_amd import salt
    lib, C = salt.lib, salt.C
    b = Batch([2, 1], [20, 3], prefix=[5], domain=[0, -1], heads=4, kv_heads=2, dim=64, page=16).open()
    buf = to_dev(np.zeros(1 << 16, np.uint16))
    try:
        s = b.seqs
        assert s.write_status(0, buf.ptr, buf.ptr) == salt.ERR_BAD_STATE          # no batch was set
        good = dict(q_len=[2, 1], length=[20, 3], page_off=[0, 2, 3], pages=[0, 1, 2], domain=[0, -1], prefix_len=[5],
                    prefix_off=[0, 1], prefix_pages=[3])
        assert s.set_status(**good) == salt.OK
        for change, want in [
            (dict(pages=[0, 6, 2]), salt.ERR_OUT_OF_RANGE),                        # (a pool of 6: pages 0 .. 5)
            (dict(pages=[0, -1, 2]), salt.ERR_OUT_OF_RANGE),
            (dict(prefix_pages=[6]), salt.ERR_OUT_OF_RANGE),
            (dict(length=[33, 3]), salt.ERR_OUT_OF_RANGE),                         # three pages are needed
            (dict(length=[-1, 3]), salt.ERR_OUT_OF_RANGE),
            (dict(q_len=[-1, 1]), salt.ERR_OUT_OF_RANGE),
            (dict(q_len=[3, 1]), salt.ERR_OUT_OF_RANGE),                           # four new tokens of at most three
            (dict(domain=[1, -1]), salt.ERR_OUT_OF_RANGE),
            (dict(domain=[-2, -1]), salt.ERR_OUT_OF_RANGE),
            (dict(prefix_len=[17]), salt.ERR_OUT_OF_RANGE),
            (dict(page_off=[1, 2, 3]), salt.ERR_INVALID_ARG),
            (dict(page_off=[0, 3, 2]), salt.ERR_OUT_OF_RANGE),
        ]:
            assert s.set_status(**{**good, **change}) == want, change
        assert s.set_status(q_len=[1] * 4, length=[1] * 4, page_off=[0, 1, 2, 3, 4], pages=[0, 1, 2, 3]) == salt.ERR_OUT_OF_RANGE
        # the batch set before a refusal stays
        assert s.write_status(0, buf.ptr, buf.ptr) == salt.OK
        assert s.write_status(1, buf.ptr, buf.ptr) == salt.ERR_OUT_OF_RANGE
        assert s.write_status(-1, buf.ptr, buf.ptr) == salt.ERR_OUT_OF_RANGE
        assert s.write_status(0, 0, buf.ptr) == salt.ERR_INVALID_ARG
        assert s.write_status(0, buf.ptr + 2, buf.ptr) == salt.ERR_INVALID_ARG
        assert s.write_status(0, buf.ptr, buf.ptr, ldk=120) == salt.ERR_INVALID_ARG
        assert s.write_status(0, buf.ptr, buf.ptr, ldv=132) == salt.ERR_INVALID_ARG
        assert lib.salt_kv_read(s.ctx.h, s.h, 0, 2, buf.ptr, 0, buf.ptr, 0, None) == salt.ERR_INVALID_ARG
        for scale in (0.0, -1.0, float("nan"), float("inf")):
            assert s.attend_status(0, buf.ptr, buf.ptr, scale) == salt.ERR_INVALID_ARG
        assert s.attend_status(0, buf.ptr, buf.ptr, 1.0, ldq=248) == salt.ERR_INVALID_ARG
        assert s.attend_status(0, 0, buf.ptr, 1.0) == salt.ERR_INVALID_ARG
        # two sequences that would write one page
        assert s.set_status(q_len=[1, 1], length=[3, 4], page_off=[0, 1, 2], pages=[2, 2]) == salt.OK
        assert s.write_status(0, buf.ptr, buf.ptr) == salt.ERR_INVALID_ARG
        assert s.attend_status(0, buf.ptr, buf.ptr + 4096, 1.0) == salt.OK
        for bad in (dict(head_dim=96), dict(page_tokens=24), dict(page_tokens=8), dict(n_pages=0), dict(n_heads=3),
                    dict(n_kv_heads=0), dict(n_layers=0), dict(format=2), dict(flags=1), dict(n_heads=1024)):
            cfg = dict(n_layers=1, n_heads=4, n_kv_heads=2, head_dim=64, page_tokens=16, n_pages=4, format=0, flags=0)
            cfg.update(bad)
            c, h = salt.KvConfig(**cfg), C.c_void_p()
            assert lib.salt_kv_create(b.ctx.h, C.byref(c), C.byref(h)) == salt.ERR_INVALID_ARG, bad
            assert not h.value and lib.salt_kv_bytes(C.byref(c)) == 0
        hipmod().synchronize()
    finally:
        b.close()
