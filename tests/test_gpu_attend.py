"""GPU parity of attention over the 8-bit cache (salt_attend) with the float64 oracle on the cache's own
values; the bounds are those of tests.serve_harness.Batch.check."""
import numpy as np
import pytest

import oracle
from tests.serve_harness import Batch, hipmod, store, to_dev

pytestmark = pytest.mark.gpu

EDGES = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129]


def _run(name, rows=None, ldq=0, ldo=0, **kw):
    print(f"\n[gpu case] attend {name}", flush=True)
    b = Batch(**kw).open()
    try:
        b.fill()
        b.set()
        got = b.attend(ldq=ldq, ldo=ldo)
        worst = b.check(got, rows)
        print(f"worst {worst:.3f}x the bound", flush=True)
        return got
    finally:
        b.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim,page", [(64, 16), (128, 64), (256, 32)])
def test_single_tokens(dim, page, dtype, fmt):
    _run(f"single {dtype} {fmt} dim={dim}", q_len=[1] * len(EDGES), length=EDGES, heads=6, kv_heads=2, dim=dim,
         page=page, fmt=fmt, dtype=dtype)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("heads,kv_heads", [(1, 1), (5, 5), (8, 1), (16, 1), (24, 8), (14, 2), (64, 1), (34, 2)])
def test_head_layouts(heads, kv_heads, dtype):
    _run(f"heads {heads}/{kv_heads} {dtype}", q_len=[1, 3, 2, 1], length=[40, 3, 200, 1], heads=heads,
         kv_heads=kv_heads, dim=64, page=16, dtype=dtype)


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128])
def test_shared_prefixes(dim, dtype, fmt):
    """Domains of several, one and no users; prefixes that end inside a tile, of one token, and empty."""
    _run(f"prefixes {dtype} {fmt} dim={dim}", q_len=[1, 1, 1, 2, 1, 1, 1, 3, 1], length=[1, 17, 64, 5, 130, 8, 90, 70, 2],
         prefix=[100, 1, 0, 257, 64], domain=[0, 0, 0, 0, -1, 1, 3, 2, 2], heads=6, kv_heads=2, dim=dim, page=16,
         dtype=dtype, fmt=fmt)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_many_users_of_one_prefix(dtype):
    n = 45
    _run(f"45 users {dtype}", q_len=[1] * n, length=[1 + 7 * i % 90 for i in range(n)], prefix=[333],
         domain=[0] * n, heads=8, kv_heads=2, dim=64, page=32, dtype=dtype,
         rows=None if dtype == "bf16" else range(0, n, 5))


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("dim", [64, 128, 256])
def test_prompts(dim, dtype, fmt):
    """Prompts of odd lengths behind a history and a prefix: the causal edge crosses tiles of rows and keys."""
    _run(f"prompts {dtype} {fmt} dim={dim}", q_len=[70, 150, 1, 33], length=[70, 213, 66, 33], prefix=[129, 20],
         domain=[0, 0, 0, 1], heads=6, kv_heads=2, dim=dim, page=64, dtype=dtype, fmt=fmt,
         rows=list(range(0, 254, 11)) + [69, 70, 219, 220, 253])


def test_long_sequences_in_pieces():
    _run("long", q_len=[1, 2, 1], length=[5000, 3001, 777], prefix=[4100], domain=[0, 0, -1], heads=8, kv_heads=2,
         dim=128, page=16, dtype="bf16")
    _run("long f32", q_len=[1, 40], length=[2500, 1800], prefix=[900], domain=[0, 0], heads=4, kv_heads=1, dim=128,
         page=128, dtype="f32", fmt="int8", rows=[0, 1, 20, 40])


def test_rows_without_keys_and_tokens_before_the_first():
    _run("no keys", q_len=[2, 3, 1, 40, 0, 2], length=[0, 1, 0, 20, 7, 0], prefix=[0, 30],
         domain=[-1, -1, 0, -1, 1, 1], heads=4, kv_heads=2, dim=64, page=16)


def test_strided_rows():
    _run("strided", q_len=[1, 5, 20], length=[30, 5, 300], heads=4, kv_heads=2, dim=64, page=16, ldq=768, ldo=264)
    _run("strided f32", q_len=[1, 5, 20], length=[30, 5, 300], heads=4, kv_heads=2, dim=64, page=16, ldq=264, ldo=512,
         dtype="f32")


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("q_len", [2, 40, 150])
def test_values_that_are_not_finite_reach_only_rows_that_see_them(q_len, fmt, dtype):
    """Pages start out holding nothing but NaN and huge values; a late token's k and another's v are not finite."""
    print(f"\n[gpu case] attend non-finite {fmt} {dtype} q_len={q_len}", flush=True)
    b = Batch([q_len, 1, 1], [q_len + 21, 50, 37], prefix=[45, 30], domain=[-1, 0, 0], heads=4, kv_heads=2, dim=64,
              page=64, fmt=fmt, dtype=dtype).open()
    try:
        junk = Batch([64 * b.n_pages], [64 * b.n_pages], heads=4, kv_heads=2, dim=64, page=64, fmt=fmt, dtype=dtype)
        rows = np.arange(64 * b.n_pages)
        junk.k[0][rows % 3 == 0] = np.nan
        junk.v[0][rows % 3 == 1] = np.inf
        junk.k[0][rows % 3 == 2] *= 2.0 ** 100
        junk.v[0][rows % 3 == 2] *= 2.0 ** 100
        junk.pages = np.arange(b.n_pages, dtype=np.int32)
        junk.page_off = np.array([0, b.n_pages], np.int32)
        junk.ctx, junk.kv, junk.stream = b.ctx, b.kv, b.stream
        junk.fill()
        n = q_len + 21
        b.k[0][n - 1, 0, 3] = np.nan                    # seen by the last row, kv head 0
        b.v[0][n - 2, 1, 5] = -np.inf                   # seen by the last two, kv head 1
        b.fill()
        b.set()
        got = b.attend()
        assert np.isnan(got[q_len - 1, :2]).all() and np.isnan(got[q_len - 2: q_len, 2:]).all()
        assert np.isfinite(got[: q_len - 2]).all() and np.isfinite(got[q_len:]).all()
        assert np.isfinite(got[q_len - 2, :2]).all()
        b.check(got, rows=[t for t in range(b.T) if t < 3 or t >= q_len or t in (q_len // 2, q_len - 3) and t < q_len - 2])
        # q: a row that is not finite is NaN alone
        q = b.q.copy()
        q[0, 1, 0] = np.nan
        other = b.attend(q=q)
        assert np.isnan(other[0, 1]).all()
        keep = np.ones(got.shape[:2], bool)
        keep[0, 1] = False
        assert np.array_equal(other[keep], got[keep], equal_nan=True)
    finally:
        b.close()


def test_large_logits():
    """Logits in the thousands: the running maximum keeps every exponential in range."""
    print("\n[gpu case] attend large logits", flush=True)
    for dtype in ("bf16", "f32"):
        b = Batch([1, 30], [200, 90], heads=4, kv_heads=2, dim=64, page=16, dtype=dtype)
        b.q = oracle.decode(store(b.q * 64, dtype), dtype)
        b.open()
        try:
            b.fill()
            b.set()
            b.check(b.attend())
        finally:
            b.close()


def test_repeats_are_bit_identical_on_any_stream():
    """Write on one stream, attend on others without waiting in between; several layers of one batch."""
    print("\n[gpu case] attend streams", flush=True)
    hip = hipmod()
    b = Batch([1] * 9 + [60], [40 * (i + 1) for i in range(9)] + [400], prefix=[700], domain=[0] * 6 + [-1] * 4, heads=8,
              kv_heads=2, dim=128, page=64, layers=2).open()
    others = [hip.Stream(), hip.Stream()]
    try:
        b.fill(0)
        b.fill(1)
        b.set()
        want = b.attend()
        b.check(want, rows=[0, 5, 9, 40, 68])
        new = [to_dev(store(np.concatenate([a[len(a) - q:] for a, q in zip(arr, b.q_len)]), "bf16"))
               for arr in (b.k, b.v)]
        qd = to_dev(store(b.q, "bf16"))
        outs = [to_dev(np.zeros((b.T, b.heads * b.dim), np.uint16)) for _ in range(6)]
        for i, o in enumerate(outs):
            layer = i % 2
            b.seqs.write(layer, new[0].ptr, new[1].ptr, others[i % 2].h)
            b.seqs.attend(layer, qd.ptr, o.ptr, b.scale, others[(i + 1) % 2].h)
        hip.synchronize()
        for o in outs:
            assert np.array_equal(oracle.decode(o.to_host(), "bf16").reshape(want.shape), want)
    finally:
        b.close()
        for s in others:
            s.destroy()


def test_batches_one_after_another_in_one_object():
    """The same object serves larger and smaller batches, set without waiting for the last one's work."""
    print("\n[gpu case] attend batches in turn", flush=True)
    big = Batch([1, 30, 4], [300, 77, 40], prefix=[90], domain=[0, -1, 0], heads=4, kv_heads=2, dim=64, page=16).open()
    small = Batch([2], [9], heads=4, kv_heads=2, dim=64, page=16, seed=3)
    try:
        small.pages = np.array([p for p in range(big.n_pages) if p not in set(big.pages) | set(big.prefix_pages)][:1], np.int32)
        small.ctx, small.kv, small.stream, small.seqs = big.ctx, big.kv, big.stream, big.seqs
        big.fill()
        small.fill()
        outs, qs = [], []
        for b in (big, small, big, small, small, big):
            b.set()
            qd = to_dev(store(b.q, "bf16"))
            od = to_dev(np.zeros((b.T, b.heads * b.dim), np.uint16))
            b.seqs.attend(0, qd.ptr, od.ptr, b.scale, b.stream.h)
            outs.append((b, od))
            qs.append(qd)
        big.stream.synchronize()
        for b, od in outs:
            b.check(oracle.decode(od.to_host(), "bf16").reshape(b.T, b.heads, b.dim))
    finally:
        big.close()
