"""GPU parity of salt_attend where logits are infinite.  Softmax over keys whose logits are all -inf is not a number, as
is every row with a logit of +inf: such a row must not come back as the zeros of a row without keys.  Keys at
-inf beside finite ones have no weight.  Every kind of work item, finished at once and joined."""
import numpy as np
import pytest

import oracle
from tests.serve_harness import Batch, store

pytestmark = pytest.mark.gpu

# q_len, len, prefix, domain, heads, kv_heads: what the cut makes of them
KINDS = {
    "four waves": dict(q_len=[1, 2, 1, 1], length=[1, 30, 64, 130], heads=4, kv_heads=2),
    "four waves, joined": dict(q_len=[1, 1, 1], length=[40, 1300, 3], prefix=[70], domain=[0, -1, 0], heads=4, kv_heads=2),
    "one wave": dict(q_len=[1] * 136, length=[1 + i % 70 for i in range(136)], heads=16, kv_heads=8),
    "one wave, joined": dict(q_len=[1] * 136, length=[1 + i % 70 for i in range(136)], prefix=[90, 33],
                             domain=[i % 3 - 1 for i in range(136)], heads=16, kv_heads=8),
    "64 rows": dict(q_len=[16, 25], length=[16, 130], heads=8, kv_heads=2),
    "128 rows": dict(q_len=[70, 33], length=[70, 180], prefix=[100], domain=[-1, 0], heads=8, kv_heads=2),
    "rows in pieces": dict(q_len=[40, 1], length=[1500, 5], heads=8, kv_heads=2),
}


def _batch(kind, dtype, fmt, lead=3.0, **kw):
    """A batch of the kind whose keys all have `lead` in their first place."""
    b = Batch(dim=64, page=16, fmt=fmt, dtype=dtype, **KINDS[kind], **kw)
    for arr in (b.k, b.pk):
        for a in arr:
            a[..., 0] = lead
    return b


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_infinite_queries(kind, dtype, fmt):
    """q = -inf against keys that are all positive there (every logit -inf), and +inf: NaN in that row alone."""
    print(f"\n[gpu case] attend infinite q, {kind} {dtype} {fmt}", flush=True)
    b = _batch(kind, dtype, fmt).open()
    try:
        b.fill()
        b.set()
        want = b.attend()
        some = sorted({0, b.T // 3, b.T // 2, b.T - 1})
        b.check(want, rows=some)
        q = b.q.copy()
        bad = np.zeros((b.T, b.heads), bool)
        for i, t in enumerate(some):
            for h in (i % b.heads, (i + 2) % b.heads):
                q[t, h, 0] = -np.inf if (i + h) % 2 == 0 else np.inf
                bad[t, h] = True
        q[b.T - 1, 0, 0], bad[b.T - 1, 0] = -np.inf, True
        got = b.attend(q=q)
        assert np.isnan(got[bad]).all(), f"{int(np.sum(~np.isnan(got[bad]).all(-1)))} of {int(bad.sum())} rows are not NaN"
        assert np.array_equal(got[~bad], want[~bad])
    finally:
        b.close()


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_some_logits_overflow(kind, dtype, fmt):
    """Finite q and k whose products pass fp32 for some keys: those have no weight, the others theirs.  Where they are
    all of a row's own keys, and behind a prefix all of one part, the rest of the row is unharmed."""
    print(f"\n[gpu case] attend logits past fp32, {kind} {dtype} {fmt}", flush=True)
    b = _batch(kind, dtype, fmt, lead=0.0)
    for i, a in enumerate(b.k):                     # (the first key of each sequence keeps a finite logit ..
        a[1:, :, 0] = 2.0 ** 11
    for s, a in enumerate(b.k):                     # .. unless there is a prefix of finite ones)
        if b.domain is not None and b.domain[s] >= 0:
            a[:, :, 0] = 2.0 ** 11
    b.q[1::2, :, 0] = -(2.0 ** 126)
    b.q = oracle.decode(store(b.q, dtype), dtype)
    b.open()
    try:
        b.fill()
        b.set()
        got = b.attend()
        assert np.isfinite(got).all()
        rows = sorted({0, 1, b.T // 3, b.T // 2 | 1, b.T - 1, *range(1, b.T, 17)} & set(range(b.T)))
        b.check(got, rows=[t for t in rows if t % 2 == 0])
        whole = b.row_keys
        b.row_keys = lambda t: tuple(a[whole(t)[0][:, 0, 0] == 0] for a in whole(t))     # the keys that are left
        b.check(got, rows=[t for t in rows if t % 2 == 1])
    finally:
        b.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_without_keys_stay_zero(dtype):
    """No key at all: zeros, whatever q holds."""
    print(f"\n[gpu case] attend infinite q without keys, {dtype}", flush=True)
    b = Batch([2, 40, 3], [0, 20, 1], prefix=[0, 30], domain=[0, -1, -1], heads=8, kv_heads=2, dim=64, page=16,
              dtype=dtype).open()
    try:
        b.fill()
        b.set()
        q = b.q.copy()
        none = [0, 1, *range(2, 22), 42, 43]
        q[none, :, 0] = np.array([-np.inf, np.inf, np.nan, 1.0])[np.arange(len(none)) % 4][:, None]
        got = b.attend(q=q)
        assert np.all(got[none] == 0)
        b.check(got, rows=[22, 41, 44])
    finally:
        b.close()
