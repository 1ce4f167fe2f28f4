"""A tracked cache's marks behind salt_kv_write: they start at weight 0 and the place in the sequence, whatever the page
held before, and stay as they are where salt_kv_write_marks gave them first."""
import numpy as np
import pytest

from oracle import steps as o64
from tests.serve_harness import hipmod, store, to_dev
from tests.test_gpu_marks import Tracked
from tests.test_gpu_serve_graphs import _Graph

pytestmark = pytest.mark.gpu


def _write(b, seqs, k, v, layer=0):
    d = [to_dev(store(a, b.dtype)) for a in (k, v)]
    seqs.write(layer, d[0].ptr, d[1].ptr, b.stream.h)
    b.stream.synchronize()


def _places(length):
    return np.concatenate([np.arange(m) for m in length] + [np.zeros(0)]).astype(int)


@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("f32", "int8")])
@pytest.mark.parametrize("dim,kv_heads,page", [(64, 3, 16), (128, 2, 64), (256, 1, 256)])
def test_pages_that_held_another_sequence(dim, kv_heads, page, dtype, fmt):
    """A prompt written in two chunks, the second alone scored, in pages with marks of an earlier owner; then evicted."""
    print(f"\n[gpu case] marks of reused pages {dtype} {fmt} dim={dim} page={page}", flush=True)
    b = Tracked([9, 5, 1], [2 * page + 9, 40, page], heads=2 * kv_heads, kv_heads=kv_heads, dim=dim, page=page, fmt=fmt,
                dtype=dtype, layers=2).open()
    first = b.kv.seqs(3, int(b.length.sum()), int(b.page_off[-1]))
    old = (b.length - b.q_len).astype(np.int32)
    row0 = np.concatenate([[0], np.cumsum(b.length)])
    try:
        owner = b.kv.seqs(3, b.T, int(b.page_off[-1]))
        b.set(owner)
        for layer in range(2):
            b.put(layer, b.weight + 1000, b.place + 7, owner)      # (heavy, and far behind)
        b.set()
        first.set(old, old, b.page_off, b.pages, stream=b.stream.h)
        part = lambda arr, new: np.concatenate([a[o:] if new else a[:o] for a, o in zip(arr, old)])
        _write(b, first, part(b.k, False), part(b.v, False))
        _write(b, b.seqs, part(b.k, True), part(b.v, True))
        weight, place = b.get()
        assert np.all(weight == 0) and np.array_equal(place, np.broadcast_to(_places(b.length)[:, None], place.shape))
        b.score(window=4)
        weight, place = b.get()
        add, bound = b.added(window=4)
        assert np.all(np.abs(weight - add) <= bound + 2.0 ** -23 * (add + bound) + 1e-30)
        assert np.array_equal(place, np.broadcast_to(_places(b.length)[:, None], place.shape))
        b.seqs.evict(0, 20, 6, b.stream.h)
        b.stream.synchronize()
        _, after = b.get()
        for s in range(3):
            for h in range(kv_heads):
                at = slice(row0[s], row0[s + 1])
                src = o64.evict(weight[at, h], place[at, h], 20, 6)
                assert np.array_equal(after[at, h][: len(src)], place[at, h][src]), (s, h)
        weight, place = b.get(1)                                   # the other layer was not written
        assert np.array_equal(weight, b.weight + 1000) and np.array_equal(place, b.place + 7)
    finally:
        b.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_a_step_leaves_older_marks(dtype):
    """Only the written tokens' marks start anew; tokens before the sequence's first have none."""
    print(f"\n[gpu case] marks of a step {dtype}", flush=True)
    b = Tracked([1, 0, 3, 6, 70], [33, 20, 64, 4, 90], heads=4, kv_heads=2, dim=64, page=16, dtype=dtype).open()
    try:
        b.fill()
        b.set()
        other = b.kv.seqs(8, b.T, int(b.page_off[-1]))
        b.set(other)
        b.put()
        k = np.concatenate([np.concatenate([np.zeros((max(0, n - m), 2, 64), np.float32), a[max(0, m - n):]])
                            for a, n, m in zip(b.k, b.q_len, b.length)])
        _write(b, b.seqs, k, k)                                    # (its marks were given by `put`)
        weight, place = b.get()
        assert np.array_equal(weight, b.weight) and np.array_equal(place, b.place)
        _write(b, other, k, k)
        weight, place = b.get()
        new, _ = b.fresh()
        assert np.array_equal(weight, np.where(new[:, None], np.float32(0), b.weight))
        assert np.array_equal(place, np.where(new[:, None], _places(b.length)[:, None], b.place))
    finally:
        b.close()


def test_recorded_writes():
    """Every replay of a recorded write starts the marks of its tokens, with eager work on the marks in between."""
    print("\n[gpu case] captured writes of a tracked cache", flush=True)
    hip = hipmod()
    b = Tracked([2, 1, 17], [50, 16, 17], heads=4, kv_heads=2, dim=64, page=16).open()
    step = b.kv.seqs(3, b.T, int(b.page_off[-1]))
    try:
        b.fill()
        b.set()
        b.set(step)
        k = to_dev(store(np.concatenate([a[m - n:] for a, n, m in zip(b.k, b.q_len, b.length)]), b.dtype))
        b.stream.synchronize()
        go = lambda: step.write(0, k.ptr, k.ptr, b.stream.h)
        go()
        b.stream.synchronize()
        g = _Graph(hip, b.stream, go)
        new, _ = b.fresh()
        for i in range(4):
            b.put(0, b.weight + i, b.place + i)
            g.launch()
            if i == 2:
                go()
            b.stream.synchronize()
            weight, place = b.get()
            assert np.array_equal(weight, np.where(new[:, None], np.float32(0), b.weight + np.float32(i))), i
            assert np.array_equal(place, np.where(new[:, None], _places(b.length)[:, None], b.place + i)), i
        g.close()
    finally:
        b.close()
