"""Evictions of sequences that no block holds in registers: up to 2^19 tokens, where the selection's bits take more than 64
KiB of LDS beside its lists, and with weights and positions of every kind."""
import numpy as np
import pytest

from tests.test_gpu_marks import Tracked, _evict

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,keep,recent", [(326016, 200000, 5000), (326080, 1000, 0), (1 << 19, 300001, 64), (1 << 19, 7, 7),
                                           ((1 << 19) - 1, (1 << 19) - 2, 100)])
def test_the_longest_sequences(n, keep, recent):
    print(f"\n[gpu case] evict n={n} keep={keep} recent={recent}", flush=True)
    b = Tracked([0, 0], [n, 50], heads=1, kv_heads=1, dim=64, page=256, dtype="bf16").open()
    b.weight = np.round(b.weight, 2).astype(np.float32)            # (many alike)
    try:
        b.fill()
        b.set()
        _evict(b, keep, recent)
    finally:
        b.close()


def test_long_sequences_of_every_kind():
    """Ties, zeros of both signs, subnormals, infinities, NaNs, negative weights; positions alike, negative, at the ends."""
    print("\n[gpu case] evict values of long sequences", flush=True)
    n = 20011
    b = Tracked([0] * 8, [n] * 8, heads=1, kv_heads=1, dim=64, page=128).open()
    rng = np.random.default_rng(5)
    w, p = b.weight.reshape(8, n), b.place.reshape(8, n)
    w[0] = 1.0
    w[1] = rng.choice([0.0, -0.0, 1e-42, -1e-42], n)
    w[2] = rng.choice([np.nan, np.inf, -np.inf, 1.0], n)
    w[3] = -w[3]
    w[4] = np.nan
    w[5].view(np.uint32)[...] = rng.choice([0x7f800001, 0xffc00001, 0x7f7fffff, 0x3f800000], n)
    p[0] = np.arange(n) - 2 ** 31                                  # (newest - recent below the least position)
    p[6] = 5
    p[7] = rng.choice([-(2 ** 31), 2 ** 31 - 1, 0], n)
    try:
        b.fill()
        b.set()
        for keep, recent in ((10000, 0), (10000, 3000), (15000, 15000), (3, 1), (n - 1, n - 1)):
            b.fill()
            _evict(b, keep, recent)
    finally:
        b.close()
