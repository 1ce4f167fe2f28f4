"""GPU parity of salt_attend where the batch's cut into work items takes its less usual ways: one-wave items in
pieces, tiles whose last rows are of another kind, whole and split key runs side by side, and a pool whose
offsets pass 32 bits.  Against the float64 oracle on the cache's own values, within the bounds of
tests.serve_harness.Batch.check."""
import numpy as np
import pytest

from tests.serve_harness import Batch, hipmod
from tests.test_gpu_attend import _run

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("dtype,fmt", [("bf16", "e4m3"), ("f32", "int8")])
def test_one_wave_items_whole_and_in_pieces(dtype, fmt):
    """Enough single tokens for a wave each: with a shared prefix (joined, so cut short), with one of their own, without."""
    n = 136
    length = [1 + (i * 397) % 700 for i in range(n)]
    _run(f"one wave {dtype} {fmt}", q_len=[1] * n, length=length, prefix=[200, 70, 33],
         domain=[2 if i == 7 else i % 3 - 1 for i in range(n)], heads=16, kv_heads=8, dim=64, page=16, dtype=dtype,
         fmt=fmt, rows=sorted({7, int(np.argmax(length)), int(np.argmin(length)), *range(0, n, 13)}))


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_last_rows_of_another_kind(dtype):
    """Prompts whose last tile holds 1, 4, 8 and 17 tokens of 4 heads, behind histories of many lengths."""
    q_len = [33, 36, 40, 49]
    ends = np.cumsum(q_len)
    _run(f"tails {dtype}", q_len=q_len, length=[1500, 36, 700, 130], prefix=[90], domain=[-1, 0, 0, -1], heads=8,
         kv_heads=2, dim=128, page=32, dtype=dtype,
         rows=sorted({0, *(ends - 1), *(ends[:-1]), 15, 16, 31, 32, 68, 69 + 32, 109 + 31, 109 + 32}))


def test_short_and_long_key_runs_side_by_side():
    """One sequence of 20000 keys among ones of a few: its pieces are joined, theirs finished at once."""
    _run("mixed lengths", q_len=[1, 1, 1, 4, 1], length=[3, 20000, 512, 513, 1], heads=8, kv_heads=4, dim=64, page=64,
         dtype="bf16")


def test_pool_offsets_past_4_gib():
    """k and v pools of more than 2^32 bytes each: rows over their first and last pages."""
    print("\n[gpu case] attend large pool", flush=True)
    from paper_2608_03579_amd import salt
    ctx = salt.Context("bf16", [(256, 256)], 0, 0, 1, 0, 1)
    stream = hipmod().Stream()
    try:
        n_pages = 66000
        kv = ctx.kv_cache(1, 8, 8, 128, 64, n_pages, "e4m3")
        b = Batch([1, 40, 2], [150, 90, 64], heads=8, kv_heads=8, dim=128, page=64)
        b.pages = np.array([n_pages - 1, 0, n_pages - 2, n_pages - 3, 1, n_pages - 4], np.int32)
        b.ctx, b.kv, b.stream = ctx, kv, stream
        b.seqs = kv.seqs(3, b.T, 6)
        b.fill()
        b.set()
        b.check(b.attend())
    finally:
        ctx.close()
        stream.destroy()
