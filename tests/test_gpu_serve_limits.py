"""Batches and objects at their limits: page references past a sequence's last token, launches that
would be too large, and calls on objects whose cache was closed."""
import numpy as np
import pytest

from paper_2608_03579_amd import salt
from tests.serve_harness import hipmod, to_dev

pytestmark = pytest.mark.gpu


def test_closed_objects_are_refused():
    hipmod()
    ctx = salt.Context("bf16", [(64, 64)], 0, 0, 1, 0, 1)
    try:
        kv = ctx.kv_cache(1, 1, 1, 64, 16, 4)
        seqs, other = kv.seqs(4, 4, 4), kv.seqs(4, 4, 4)
        other.close()
        seqs.set([1], [1], [0, 1], [0])
        buf = to_dev(np.zeros((4, 64), np.uint16))
        kv.close()
        for q in (seqs, other):
            assert q.h is None
            assert q.set_status([1], [1], [0, 1], [0]) == salt.ERR_INVALID_ARG
            assert q.write_status(0, buf.ptr, buf.ptr) == salt.ERR_INVALID_ARG
            assert q.read_status(0, "own", buf.ptr, buf.ptr) == salt.ERR_INVALID_ARG
            assert q.attend_status(0, buf.ptr, buf.ptr, 1.0) == salt.ERR_INVALID_ARG
            q.close()
        buf.free()
    finally:
        ctx.close()


def test_launches_that_are_too_large_are_refused():
    """2^24 page references would be read by 2^32 threads. The batch set before stays."""
    hip = hipmod()
    ctx = salt.Context("f32", [(64, 64)], 0, 0, 1, 0, 1)
    try:
        kv = ctx.kv_cache(1, 1, 1, 64, 16, 1, "int8")
        n_ref = 1 << 24
        seqs = kv.seqs(1, 1, n_ref)
        seqs.set([1], [1], [0, 1], [0])
        assert seqs.set_status([1], [1], [0, n_ref], np.zeros(n_ref, np.int32)) == salt.ERR_OUT_OF_RANGE
        x, out = to_dev(np.full((1, 64), 127.0, np.float32)), [to_dev(np.zeros((1, 64), np.float32)) for _ in range(2)]
        seqs.write(0, x.ptr, x.ptr)
        seqs.read(0, "own", out[0].ptr, out[1].ptr)
        hip.synchronize()
        assert all(np.all(o.to_host() == 127.0) for o in out)
        for d in (x, *out):
            d.free()
    finally:
        ctx.close()


def test_page_references_past_the_end():
    """A sequence may hold more pages than its tokens need: the others are neither read nor written."""
    hip = hipmod()
    ctx = salt.Context("f32", [(64, 64)], 0, 0, 1, 0, 1)
    try:
        kv = ctx.kv_cache(1, 1, 1, 64, 256, 3, "int8")
        n_ref = (1 << 23) + 5                   # the last ones' first token passes 2^31
        seqs = kv.seqs(2, 4, n_ref + 1)
        pages = np.ones(n_ref + 1, np.int32)
        pages[0], pages[-1] = 0, 2
        seqs.set([1, 2], [1, 2], [0, n_ref, n_ref + 1], pages)
        x = np.arange(3 * 64, dtype=np.float32).reshape(3, 64) - 90.0
        k, v = to_dev(x), to_dev(-x)
        seqs.write(0, k.ptr, v.ptr)
        out = [to_dev(np.full((4, 64), 7.0, np.float32)) for _ in range(2)]
        seqs.read(0, "own", out[0].ptr, out[1].ptr)
        hip.synchronize()
        # int8: half a step of amax / 127, and the rounding of the scale
        for got, want in zip((o.to_host() for o in out), (x, -x)):
            step = np.abs(want).max(1, keepdims=True) / 127
            assert np.all(np.abs(got[:3] - want) <= 0.5001 * step)
            assert np.all(got[3:] == 7.0)
        for d in (k, v, *out):
            d.free()
    finally:
        ctx.close()
