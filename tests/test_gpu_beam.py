"""GPU parity of salt_beam_select against float64.

The order within a beam is the logits' own, so it has to be exact.  Across beams two worths can be as close as
the sum of exponentials is off: a term's argument is rounded twice (2^-23 of up to 40 in powers of two: the terms
that count) and its exponential 2^-22, so 2^-23 * 28 + 2^-22 < 5e-6 of the sum, and of the worth.  A continuation in
another place than the oracle's is right only where both are of other beams and within twice that."""
import numpy as np
import pytest

import oracle
from oracle import steps as o64
from paper_2608_03579_amd import salt
from tests.serve_harness import hipmod, store, to_dev, values

pytestmark = pytest.mark.gpu
TOL = 5e-6


class Select:
    def __init__(self, dtype, max_rows, max_out):
        self.hip, self.dtype = hipmod(), dtype
        self.ctx = salt.Context(dtype, [(64, 64)], 0, 0, 1, 0, 1)
        self.beams, self.stream = self.ctx.beams(max_rows, max_out), self.hip.Stream()

    def run(self, logits, score, n_out, ld=0):
        reqs, width, vocab = logits.shape
        rows = reqs * width
        buf = np.full((rows, ld or vocab), store(np.array([np.inf]), self.dtype)[0])     # (behind the vocabulary: not read)
        buf[:, :vocab] = store(logits, self.dtype).reshape(rows, vocab)
        d = [to_dev(buf), to_dev(np.ascontiguousarray(score, np.float32))]
        out = [to_dev(np.full((reqs + 1, n_out), 7, t)) for t in (np.float32, np.int32, np.int32)]
        self.beams.select(reqs, width, vocab, d[0].ptr, d[1].ptr, n_out, *[o.ptr for o in out], self.stream.h, ld=ld)
        self.stream.synchronize()
        res = [o.to_host() for o in out]
        assert all(np.all(r[reqs:] == 7) for r in res), "written behind the last request"
        return [r[:reqs] for r in res]

    def close(self):
        self.ctx.close()
        self.stream.destroy()


def _check(logits, score, n_out, got):
    for r in range(len(logits)):
        worth = o64.beam_worth(logits[r], np.float32(score[r]))
        value, beam, token = o64.beam_select(worth, n_out)
        gv, gb, gt = (g[r] for g in got)
        none = value == -np.inf
        assert np.all(gb[none] == -1) and np.all(gt[none] == -1) and np.all(gv[none] == -np.inf), r
        n = int((~none).sum())
        assert len(set(zip(gb[:n].tolist(), gt[:n].tolist()))) == n, f"request {r}: a continuation twice"
        for i in range(n):
            assert 0 <= gb[i] < worth.shape[0] and 0 <= gt[i] < worth.shape[1], (r, i)
            mine = worth[gb[i], gt[i]]
            assert abs(float(gv[i]) - mine) <= TOL + 2.0 ** -24 * abs(mine), (r, i)
            if (gb[i], gt[i]) != (beam[i], token[i]):
                assert gb[i] != beam[i] and abs(mine - value[i]) <= 2 * TOL, (r, i, mine, value[i])
        for b in range(worth.shape[0]):                            # a beam's own: its best tokens, in order
            mine = gt[:n][gb[:n] == b]
            x = logits[r, b]
            best = np.lexsort((np.arange(len(x)), -x))[: len(mine)]
            assert np.array_equal(mine, best), (r, b)


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("reqs,width,vocab,n_out", [
    (1, 1, 1, 1), (1, 1, 3, 5), (2, 3, 7, 6), (3, 2, 63, 64), (1, 4, 511, 8), (5, 5, 512, 10), (2, 8, 513, 16),
    (1, 4, 32001, 8), (3, 64, 2049, 64), (1, 1, 200000, 64), (70, 4, 5000, 1), (600, 2, 4100, 4), (9, 16, 50261, 32)])
def test_shapes(reqs, width, vocab, n_out, dtype):
    print(f"\n[gpu case] select {dtype} reqs={reqs} width={width} vocab={vocab} n_out={n_out}", flush=True)
    s = Select(dtype, reqs * width, n_out)
    try:
        ld = -(-vocab // 8) * 8
        x = values((reqs, width, vocab), vocab + n_out, dtype, 2.5)
        score = np.random.default_rng(vocab).uniform(-12, 0, (reqs, width))
        _check(x, score, n_out, s.run(x, score, n_out, ld))
        if vocab % 8 == 0:
            _check(x, score, n_out, s.run(x, score, n_out, 0))
        _check(x, score, n_out, s.run(x, score, n_out, ld + 64))
    finally:
        s.close()


@pytest.mark.parametrize("order", ["rising", "falling", "flat", "few values", "the last chunk", "one lane"])
def test_orders_and_ties(order):
    """Rising logits replace the whole list all the way; equal ones go by beam and token."""
    print(f"\n[gpu case] select {order}", flush=True)
    reqs, width, vocab, n_out = 2, 5, 20003, 24
    rng = np.random.default_rng(5)
    x = np.zeros((reqs, width, vocab))
    if order in ("rising", "falling"):
        x += np.linspace(-8, 8, vocab) * (1 if order == "rising" else -1)
    elif order == "few values":
        x += rng.integers(-3, 3, x.shape)
    elif order == "the last chunk":
        x[..., -37:] = rng.uniform(3, 5, (reqs, width, 37))
    elif order == "one lane":
        x[..., 8 * 31:8 * 32] = 4 + np.arange(8)
        x[..., 512 * 9 + 8 * 31:512 * 9 + 8 * 32] = 4 + np.arange(8)[::-1]
    x = oracle.decode(store(x, "f32"), "f32")
    score = np.repeat(np.float32([[-1.0, -2.5]]).T, width, 1)       # (equal scores: ties across beams, too)
    s = Select("f32", reqs * width, n_out)
    try:
        got = s.run(x, score, n_out, 20008)
        _check(x, score, n_out, got)
        for r in range(reqs):
            # equal rows have equal sums, to the bit: ties are exact here
            if order != "few values" and order != "the last chunk":
                _, beam, token = o64.beam_select(o64.beam_worth(x[r], score[r]), n_out)
                assert np.array_equal(got[1][r], beam) and np.array_equal(got[2][r], token)
    finally:
        s.close()


def test_dead_beams_and_masked_tokens():
    """Beams that are not live or whose row is no distribution offer nothing; masked tokens are never taken, also where
    too few others are left; the type's lowest value is a value."""
    print("\n[gpu case] select dead beams", flush=True)
    reqs, width, vocab, n_out = 3, 8, 1201, 12
    x = values((reqs, width, vocab), 77, "f32", 2.0)
    score = np.random.default_rng(8).uniform(-5, 0, (reqs, width)).astype(np.float32)
    x[0, 0, 700] = np.nan
    x[0, 1, 3] = np.inf
    x[0, 2] = -np.inf
    score[0, 3], score[0, 4], score[0, 5] = -np.inf, np.nan, np.inf
    x[0, 6, 5:] = -np.inf
    low = float(np.finfo(np.float32).min)
    x[1, 0] = low                                                  # an even distribution, however low
    x[1, 1:] = -np.inf
    x[1, 1, [9, 1200]] = [low, 2.0]
    score[2] = -np.inf
    s = Select("f32", reqs * width, n_out)
    try:
        got = s.run(x, score, n_out, 1208)
        _check(x, score, n_out, got)
        assert set(got[1][0]) <= {6, 7} and np.sum(got[1][0] == 6) <= 5
        assert np.all(got[1][2] == -1) and np.all(got[2][2] == -1)
        x[2], score[2] = -np.inf, 0.0
        x[2, 3, 17] = -40.0                                        # one continuation: certain
        got = s.run(x, score, n_out, 1208)
        assert got[1][2].tolist() == [3] + [-1] * 11 and got[2][2, 0] == 17 and got[0][2, 0] == 0.0
    finally:
        s.close()


def test_objects_and_streams_repeat_the_result():
    """The same call on another stream, behind a call of another shape through the same scratch: the same bits."""
    print("\n[gpu case] select repeats", flush=True)
    x, y = values((4, 6, 9001), 3, "bf16", 2.0), values((1, 2, 40000), 4, "bf16", 2.0)
    sx, sy = np.linspace(-3, 0, 24).reshape(4, 6), np.zeros((1, 2))
    s = Select("bf16", 24, 16)
    try:
        first = s.run(x, sx, 16, 9008)
        other = s.hip.Stream()
        for _ in range(3):
            s.run(y, sy, 7, 40000)
            mine, s.stream = s.stream, other
            again = s.run(x, sx, 16, 9008)
            s.stream = mine
            for a, b in zip(first, again):
                assert np.array_equal(a, b)
        s.stream.synchronize()
        other.synchronize()
        other_call = s.beams.select_status(5, 5, 10, 16, 16, 1, 16, 16, 16)
        assert other_call == salt.ERR_OUT_OF_RANGE                 # 25 rows of 24
        s.beams.close()
        assert s.beams.h is None
    finally:
        s.close()
