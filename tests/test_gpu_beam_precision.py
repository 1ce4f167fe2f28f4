"""How far salt_beam_select's worth is off, where the rounding of the output hides nothing: a beam's score is the log
probability of its best token with the sign changed, so that the best continuation is worth about 0.

Bound, in units of 2^-24 and of the sum of exponentials.  A term's argument is rounded twice, and log2 e once (0.3): 2.3 of
it, 1.6 of its term for every power of two below the maximum, of which the terms have log2 V on average at most.  The
exponential 2; eight additions in fp32 and the two parts' 9; each time that a lane's maximum rises its sum is scaled
by an exponential, 2, and so it is when lanes, waves and pieces meet, 6 in all.  (What the exponents of those add up to is
in the term's own distance from the maximum.)"""
import numpy as np
import pytest

from tests.serve_harness import values
from tests.test_gpu_beam import Select

pytestmark = pytest.mark.gpu
RUN = 4096                                                         # logits that a block's four waves take in turn


def _rows(vocab):
    step = np.arange(vocab) // RUN                                 # the maximum rises with every run
    tail = np.full(vocab, -np.log(vocab))
    tail[vocab // 3] = 0.0                                         # half the sum in the peak, half in the rest
    rng = np.random.default_rng(vocab)
    rows = [values((vocab,), 1, "f32", s) for s in (0.3, 2.5, 8.0)]
    rows += [np.zeros(vocab), tail, np.linspace(-20, 0, vocab), 0.37 * step, 0.1 * step + rng.uniform(0, 0.01, vocab),
             -0.37 * step + 30]
    return np.stack(rows).astype(np.float32)


@pytest.mark.parametrize("copies", [1, 114])                       # (1026 rows: a row in one piece)
@pytest.mark.parametrize("vocab", [5, 4096, 50000, 131072])
def test_the_worth_itself(vocab, copies):
    print(f"\n[gpu case] worth vocab={vocab} copies={copies}", flush=True)
    x = _rows(vocab)
    n = len(x)
    top = x.max(-1).astype(np.float64)
    lse = top + np.log(np.exp(x.astype(np.float64) - top[:, None]).sum(-1))
    score = (lse - top).astype(np.float32)
    want = score.astype(np.float64) + top - lse
    s = Select("f32", n * copies, 1)
    try:
        got = s.run(np.tile(x, (copies, 1))[:, None], np.tile(score, copies)[:, None], 1, -(-vocab // 8) * 8)
    finally:
        s.close()
    assert np.array_equal(got[2].reshape(copies, n), np.tile(x.argmax(-1), (copies, 1)))
    err = np.abs(got[0].reshape(copies, n) - want).max(0)
    rises = -(-vocab // RUN)
    bound = 2.0 ** -24 * (1.6 * np.log2(vocab) + 17 + 2 * rises)
    print("errors", " ".join(f"{e:.1e}" for e in err), f"bound {bound:.1e}", flush=True)
    assert np.all(err <= bound)
