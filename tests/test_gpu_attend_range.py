"""salt_attend at the ends of the range that include/salt.h gives for finite results: v up to 2^119 over a row's keys, q up
to 2^110, with keys as small as keep the logits moderate.  Every kind of work item; bounds of
tests.serve_harness.Batch.check."""
import numpy as np
import pytest

import oracle
from tests.serve_harness import Batch, store
from tests.test_gpu_attend_infinite import KINDS

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_large_values(kind, dtype, fmt):
    print(f"\n[gpu case] attend large values, {kind} {dtype} {fmt}", flush=True)
    b = Batch(dim=64, page=16, fmt=fmt, dtype=dtype, **KINDS[kind])
    most = int(b.length.max() + (b.prefix.max() if len(b.prefix) else 0))
    top = 2.0 ** (119 - int(np.ceil(np.log2(most))))
    hold = lambda a: oracle.decode(store(a, dtype), dtype)
    for a in (*b.v, *b.pv):
        a[:] = hold(a / np.abs(a).max() * top)
    for a in (*b.k, *b.pk):
        a[:] = hold(a * 2.0 ** -95)
    b.q = hold(b.q * 2.0 ** 95)
    b.q[0] = hold(b.q[0] / np.abs(b.q[0]).max() * 2.0 ** 110)
    b.open()
    try:
        b.fill()
        b.set()
        got = b.attend()
        assert np.isfinite(got).all()
        b.check(got, rows=sorted({0, 1, b.T // 3, b.T - 1}))
    finally:
        b.close()
