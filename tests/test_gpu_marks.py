"""GPU parity of a tracked cache: gathered weights (salt_kv_score) against float64, eviction (salt_kv_evict) exactly.

Bound of a weight: each of its terms p as the attention's probabilities in fp32 (a logit is a sum of dim products,
4 dim 2^-24 of its largest term sum, which scales p; 2^-17 for the sum, the exponential and the division), and 2^-24 of
the sum for each of its additions."""
import numpy as np
import pytest

import oracle
from oracle import serve
from oracle import steps as o64
from paper_2608_03579_amd import salt
from tests.serve_harness import Batch, hipmod, store, to_dev

pytestmark = pytest.mark.gpu


class Tracked(Batch):
    def open(self, n_pages=None):
        super().open(n_pages)
        self.kv.track()
        rng = np.random.default_rng([61, self.seed])
        n = int(self.length.sum())
        self.weight = np.exp(rng.standard_normal((n, self.kv_heads)) * 2 - 2).astype(np.float32)
        self.place = rng.integers(0, 1 << 20, (n, self.kv_heads)).astype(np.int32)
        return self

    def put(self, layer=0, weight=None, place=None, seqs=None):
        d = [to_dev(self.weight if weight is None else weight), to_dev(self.place if place is None else place)]
        (seqs or self.seqs).write_marks(layer, d[0].ptr, d[1].ptr, self.stream.h)
        self.stream.synchronize()

    def get(self, layer=0, rows=None, seqs=None):
        rows = int(self.length.sum()) if rows is None else rows
        d = [to_dev(np.full((rows + 1, self.kv_heads), 77, t)) for t in (np.float32, np.int32)]
        (seqs or self.seqs).read_marks(layer, d[0].ptr, d[1].ptr, self.stream.h)
        self.stream.synchronize()
        out = [a.to_host() for a in d]
        assert all(np.all(a[rows:] == 77) for a in out), "written behind the last sequence"
        return [a[:rows] for a in out]

    def score(self, layer=0, window=0, pos=None, ldq=0, q=None):
        width = self.heads * self.dim
        buf = np.full((max(1, self.T), ldq or width), store(np.array([np.nan]), self.dtype)[0])
        buf[: self.T, :width] = store(self.q if q is None else q, self.dtype).reshape(self.T, width)
        qd = to_dev(buf)
        pd = None if pos is None else to_dev(np.asarray(pos, np.int32))
        self.seqs.score(layer, qd.ptr, pd.ptr if pd else 0, self.scale, window, self.stream.h, ldq)
        self.stream.synchronize()

    def added(self, window=0, q=None):
        """(weights that the step adds to each own token, their bound), [sum of len][kv_heads]."""
        q = self.q if q is None else q
        w, bound = np.zeros((2, int(self.length.sum()), self.kv_heads))
        row0 = np.concatenate([[0], np.cumsum(self.length)])
        G, t = self.heads // self.kv_heads, 0
        for s, (n, m) in enumerate(zip(self.q_len, self.length)):
            for j in range(int(n)):
                if not window or n - j <= window:
                    k, _ = self.row_keys(t)
                    see = max(0, int(m - n + j + 1))
                    for h in range(self.heads):
                        if k.shape[0] == 0 or see == 0:
                            continue
                        p, big = o64.weights(q[t, h], k[:, h // G], self.scale)
                        at = slice(row0[s], row0[s] + see)
                        w[at, h // G] += p[-see:]
                        bound[at, h // G] += p[-see:] * (4 * self.dim * 2.0 ** -24 * big + 2.0 ** -17)
                t += 1
        return w, bound + 2.0 ** -24 * (self.T * G + 2) * np.abs(w)

    def fresh(self):
        """(own tokens that are the step's, their rows of q)."""
        row = np.concatenate([np.arange(m) - (m - n) for n, m in zip(self.q_len, self.length)] + [np.zeros(0)]).astype(int)
        first = np.concatenate([[0], np.cumsum(self.q_len)])[:-1]
        return row >= 0, np.repeat(first, self.length) + row

    def check_score(self, window=0, pos=None, ldq=0):
        self.put()
        self.score(0, window, pos, ldq)
        weight, place = self.get()
        new, rows = self.fresh()
        add, bound = self.added(window)
        touched = np.repeat(self.q_len > 0, self.length)
        had = np.where(new[:, None], 0.0, self.weight.astype(np.float64))
        want = had + add
        bound = bound + 2.0 ** -23 * (np.abs(want) + bound)
        err = np.abs(weight - want)
        assert np.array_equal(weight[~touched], self.weight[~touched])
        assert np.all(err[touched] <= bound[touched] + 1e-30), f"{float((err / (bound + 1e-30))[touched].max()):.3f}x the bound"
        where = np.concatenate([np.arange(m) for m in self.length] + [np.zeros(0)]).astype(int)
        at = where if pos is None else np.asarray(pos)[np.where(new, rows, 0)]
        assert np.array_equal(place, np.where(new[:, None], at[:, None], self.place))
        return weight


KINDS = {
    "one token": dict(q_len=[1], length=[1]),
    "decode": dict(q_len=[1, 1, 0, 1, 1], length=[1, 17, 40, 64, 333]),
    "drafts": dict(q_len=[4, 1, 7], length=[4, 90, 130]),
    "tokens before the first": dict(q_len=[5, 9, 3], length=[3, 9, 0]),
    "domains": dict(q_len=[1, 2, 1, 1, 3], length=[9, 30, 64, 130, 3], prefix=[70, 1, 130], domain=[0, 0, -1, 2, 1]),
    "long": dict(q_len=[1, 1], length=[2500, 3]),
    "one wave each": dict(q_len=[1] * 140, length=[1 + 5 * i % 70 for i in range(140)], prefix=[90, 33],
                          domain=[i % 3 - 1 for i in range(140)]),
    "prompts": dict(q_len=[33, 70, 1], length=[33, 131, 64], prefix=[50], domain=[-1, 0, -1]),
    "a long prompt": dict(q_len=[300], length=[420]),
}


@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("kind", KINDS)
def test_scores(kind, dtype, fmt):
    print(f"\n[gpu case] score {kind} {dtype} {fmt}", flush=True)
    heads, kv_heads, dim, page = {"one wave each": (16, 8, 64, 16), "long": (8, 2, 128, 64), "domains": (6, 2, 64, 16),
                                  "prompts": (8, 2, 128, 64), "a long prompt": (3, 1, 64, 128)}.get(kind, (4, 2, 64, 32))
    b = Tracked(heads=heads, kv_heads=kv_heads, dim=dim, page=page, fmt=fmt, dtype=dtype, **KINDS[kind]).open()
    try:
        b.fill()
        b.set()
        b.check_score(pos=np.random.default_rng(1).integers(-5, 1 << 30, b.T))
        b.check_score(window=1)
        b.check_score(window=20, ldq=heads * dim + 24)
    finally:
        b.close()


@pytest.mark.parametrize("dim,heads,kv_heads,page", [(256, 10, 2, 16), (256, 1, 1, 256), (128, 40, 1, 64), (64, 64, 1, 32),
                                                     (128, 15, 5, 128), (64, 21, 3, 64)])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_score_heads_and_pages(dim, heads, kv_heads, page, dtype):
    print(f"\n[gpu case] score {dtype} dim={dim} heads={heads}/{kv_heads} page={page}", flush=True)
    b = Tracked([1, 20, 3], [page, 20 + page // 2, 2 * page + 5], heads=heads, kv_heads=kv_heads, dim=dim, page=page,
                dtype=dtype, prefix=[page + 1], domain=[0, -1, 0]).open()
    try:
        b.fill()
        b.set()
        b.check_score()
        b.check_score(window=2)
    finally:
        b.close()


def test_scores_repeat_and_layers_stay_apart():
    """The same step from the same marks: the same bits; the other layer's marks as they were."""
    print("\n[gpu case] score repeats", flush=True)
    b = Tracked([1, 90, 4], [700, 200, 64], heads=8, kv_heads=2, dim=64, page=16, layers=2).open()
    try:
        b.fill(0)
        b.fill(1)
        b.set()
        b.put(1, b.weight + 1, b.place + 1)
        first = b.check_score()
        for _ in range(3):
            assert np.array_equal(b.check_score(), first)
        weight, place = b.get(1)
        assert np.array_equal(weight, b.weight + 1) and np.array_equal(place, b.place + 1)
        # twice without new marks between: the old tokens gather twice, the step's own once
        b.put()
        b.score()
        once, _ = b.get()
        b.score()
        twice, _ = b.get()
        new, _ = b.fresh()
        assert np.array_equal(twice[new], once[new]) and np.all(twice[~new] >= once[~new])
    finally:
        b.close()


@pytest.mark.parametrize("kind", ["decode", "drafts", "prompts", "long"])
@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_rows_that_are_no_distribution(kind, dtype):
    """A row with a logit of +inf or NaN, or all at -inf, adds NaN to what it sees and to nothing else."""
    print(f"\n[gpu case] score not finite {kind} {dtype}", flush=True)
    b = Tracked(heads=4, kv_heads=2, dim=64, page=16, dtype=dtype, **KINDS[kind])
    for arr in (b.k, b.pk):
        for a in arr:
            a[..., 0] = 3.0                                        # (a q of -inf there: every logit -inf)
    b.open()
    try:
        b.fill()
        b.set()
        b.put()
        b.score()
        clean, _ = b.get()
        first = np.concatenate([[0], np.cumsum(b.q_len)])
        row0 = np.concatenate([[0], np.cumsum(b.length)])
        for bad in (np.inf, -np.inf, np.nan):
            q = b.q.copy()
            hit = np.zeros(clean.shape, bool)
            for s in (0, len(b.q_len) - 1):
                if b.q_len[s] == 0:
                    continue
                j = int(b.q_len[s]) // 2
                q[first[s] + j, s % 4, 0] = bad
                hit[row0[s]: row0[s] + int(b.length[s] - b.q_len[s]) + j + 1, (s % 4) // 2] = True
            b.put()
            b.score(q=q)
            got, _ = b.get()
            assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], clean[~hit]), bad
    finally:
        b.close()


# ---- eviction --------------------------------------------------------------------------------
def _evict(b, keep, recent, layer=0):
    """One eviction against the oracle: marks, and k and v of every kept token, to the bit."""
    b.put(layer)
    hip = hipmod()
    sdt = np.float32 if b.dtype == "f32" else np.uint16
    kept = np.minimum(b.length, keep).astype(np.int32)
    left = b.kv.seqs(max(1, len(kept)), 1, max(1, int(b.page_off[-1])))
    zero = np.zeros_like(kept)
    left.set(zero, kept, b.page_off, b.pages, stream=b.stream.h)

    def read(seqs, rows):
        d = [to_dev(np.zeros((max(1, rows), b.kv_heads, b.dim), sdt)) for _ in range(2)]
        seqs.read(layer, "own", d[0].ptr, d[1].ptr, b.stream.h)
        b.stream.synchronize()
        return [a.to_host()[:rows] for a in d]

    n = int(b.length.sum())
    before = read(b.seqs, n)
    b.seqs.evict(layer, keep, recent, b.stream.h)
    b.stream.synchronize()
    after, (weight, place) = read(b.seqs, n), b.get(layer)
    row = 0
    for m in b.length:
        m = int(m)
        for h in range(b.kv_heads):
            src = o64.evict(b.weight[row: row + m, h], b.place[row: row + m, h], keep, recent)
            src = np.concatenate([src, np.arange(len(src), m)]) + row       # (places from `keep` on: as they were)
            at = slice(row, row + m)
            assert np.array_equal(weight[at, h].view(np.int32), b.weight[src, h].view(np.int32)), (row, h)
            assert np.array_equal(place[at, h], b.place[src, h]), (row, h)
            for a, o in zip(after, before):
                assert np.array_equal(a[at, h], o[src, h]), (row, h)
        row += m
    # what the next batch reads: the first `keep` of each
    rows = np.concatenate([r0 + np.arange(c) for r0, c in zip(np.cumsum(b.length) - b.length, kept)] + [np.zeros(0)]).astype(int)
    for a, o in zip(read(left, int(kept.sum())), after):
        assert np.array_equal(a, o[rows])
    left.close()
    hip.synchronize()


@pytest.mark.parametrize("fmt,dtype", [("e4m3", "bf16"), ("int8", "f32")])
@pytest.mark.parametrize("dim,kv_heads,page", [(64, 3, 16), (128, 8, 64), (256, 1, 256)])
@pytest.mark.parametrize("keep,recent", [(1, 0), (1, 1), (7, 3), (63, 0), (64, 64), (65, 20), (150, 10), (399, 32), (5000, 10)])
def test_eviction(keep, recent, dim, kv_heads, page, fmt, dtype):
    print(f"\n[gpu case] evict keep={keep} recent={recent} dim={dim} kv={kv_heads} page={page} {fmt}", flush=True)
    b = Tracked([0] * 9, [1, 2, 0, 64, 65, 66, 151, 400, 300], heads=kv_heads, kv_heads=kv_heads, dim=dim, page=page, fmt=fmt,
                dtype=dtype, layers=2).open()
    try:
        b.fill(1)
        b.set()
        _evict(b, keep, recent, 1)
    finally:
        b.close()


@pytest.mark.parametrize("n,keep,recent", [(4096, 2048, 100), (4097, 4096, 0), (9000, 8000, 7000), (16384, 100, 0),
                                           (16385, 16000, 64), (40000, 20001, 1000)])
def test_long_evictions(n, keep, recent):
    """Blocks of 256 and 1024 threads, keys in LDS or read again, more moves than are listed at a time."""
    print(f"\n[gpu case] evict n={n} keep={keep}", flush=True)
    b = Tracked([0, 0], [n, 50], heads=2, kv_heads=2, dim=64, page=256, dtype="bf16").open()
    try:
        b.fill()
        b.set()
        _evict(b, keep, recent)
    finally:
        b.close()


def test_weights_and_positions_of_every_kind():
    """Ties, zeros of both signs, negative weights, subnormals, infinities and NaNs; positions alike, negative, at the ends."""
    print("\n[gpu case] evict values", flush=True)
    b = Tracked([0] * 8, [200] * 8, heads=4, kv_heads=4, dim=64, page=16).open()
    rng = np.random.default_rng(4)
    w, p = b.weight.reshape(8, 200, 4), b.place.reshape(8, 200, 4)
    w[0] = 1.0
    w[1] = rng.choice([0.0, -0.0, 1e-42, -1e-42], w[1].shape)
    w[2] = rng.choice([np.nan, np.inf, -np.inf, 1.0], w[2].shape)
    w[3] = -w[3]
    w[4] = np.nan
    w[5].view(np.uint32)[...] = rng.choice([0x7f800001, 0xffc00001, 0x7f7fffff, 0x3f800000], w[5].shape)
    p[6] = 5
    p[7] = rng.choice([-(2 ** 31), 2 ** 31 - 1, 0], p[7].shape)
    try:
        b.fill()
        b.set()
        for keep, recent in ((100, 0), (100, 30), (150, 150), (3, 1)):
            b.fill()
            _evict(b, keep, recent)
        p[0] = np.arange(200)[:, None] - 2 ** 31                   # newest - recent below the least position
        b.fill()
        _evict(b, 199, 199)
    finally:
        b.close()


def test_eviction_leaves_the_rest():
    """keep = 0 and budgets that no sequence exceeds change nothing; other sequences' pages and the other layer stay."""
    print("\n[gpu case] evict nothing", flush=True)
    b = Tracked([0, 0, 0], [30, 90, 55], heads=2, kv_heads=2, dim=64, page=16, layers=2).open()
    try:
        b.fill(0)
        b.fill(1)
        b.set()
        b.put(0)
        b.put(1)
        half = b.kv.seqs(1, 1, 8)
        half.set([0], [90], [0, 6], b.pages[b.page_off[1]: b.page_off[2]], stream=b.stream.h)
        half.evict(0, 10, 0, b.stream.h)
        for keep in (0, 90, 4000):
            b.seqs.evict(1, keep, 0, b.stream.h)
        b.stream.synchronize()
        weight, place = b.get(1)
        assert np.array_equal(weight, b.weight) and np.array_equal(place, b.place)
        weight, place = b.get(0)
        for at in (slice(0, 30), slice(120, 175)):
            assert np.array_equal(weight[at], b.weight[at]) and np.array_equal(place[at], b.place[at])
        assert not np.array_equal(weight[30:40], b.weight[30:40])
    finally:
        b.close()


# ---- copies of pages -----------------------------------------------------------------------------
@pytest.mark.parametrize("tracked", [True, False])
@pytest.mark.parametrize("dim,kv_heads,page,fmt,layers", [(64, 3, 16, "int8", 3), (128, 2, 64, "e4m3", 2), (256, 1, 256, "e4m3", 1)])
def test_copies(dim, kv_heads, page, fmt, layers, tracked):
    print(f"\n[gpu case] copy dim={dim} page={page} tracked={tracked}", flush=True)
    n = 300 if page == 16 else 5                                   # (more than one launch's pairs)
    length = np.random.default_rng(2).integers(1, page + 1, n)
    make = Tracked if tracked else Batch
    b = make(np.zeros(n, int), length, heads=kv_heads, kv_heads=kv_heads, dim=dim, page=page, fmt=fmt, layers=layers,
             spare=n + 3).open()
    try:
        free = np.setdiff1d(np.arange(b.n_pages), b.pages)[:n].astype(np.int32)
        other = b.kv.seqs(n, 1, n)
        other.set(b.q_len, length, b.page_off, free, stream=b.stream.h)
        b.set()
        for i in range(layers):
            b.fill(i)
            if tracked:
                b.put(i, b.weight + i, b.place + i)
        rows = int(length.sum())
        cut = np.random.default_rng(3).integers(0, length + 1).astype(np.int32)

        def read(seqs, layer):
            d = [to_dev(np.zeros((rows, kv_heads, dim), np.uint16)) for _ in range(2)]
            seqs.read(layer, "own", d[0].ptr, d[1].ptr, b.stream.h)
            b.stream.synchronize()
            return [a.to_host() for a in d] + (b.get(layer, seqs=seqs) if tracked else [])

        b.kv.copy(b.pages, free, cut, b.stream.h)
        copied = np.concatenate([np.arange(m) < c for m, c in zip(length, cut)])
        for i in range(layers):
            for a, o in zip(read(other, i), read(b.seqs, i)):
                assert np.array_equal(a[copied], o[copied]) and np.all(a[~copied] == 0)
        b.kv.copy(b.pages, free, None, b.stream.h)
        for i in range(layers):
            for a, o in zip(read(other, i), read(b.seqs, i)):
                assert np.array_equal(a, o)
    finally:
        b.close()


# ---- layouts and values beyond the kinds above --------------------------------------------------------
@pytest.mark.parametrize("group", [1, 2, 3, 5, 6, 7, 8, 12, 16, 17, 24, 33, 64])
@pytest.mark.parametrize("dtype,dim", [("bf16", 64), ("f32", 64), ("bf16", 128)])
def test_score_groups_of_heads(group, dtype, dim):
    """Sequences of many rows for every way that a group's heads fill a tile of 16 rows; and few rows beside them."""
    print(f"\n[gpu case] score group={group} {dtype} dim={dim}", flush=True)
    b = Tracked([200 // group + 3, 1, 133 // group + 1], [200 // group + 70, 65, 133 // group + 1], heads=2 * group, kv_heads=2,
                dim=dim, page=64, dtype=dtype, prefix=[40], domain=[0, -1, -1]).open()
    try:
        b.fill()
        b.set()
        b.check_score()
        b.check_score(window=150 // group + 1, ldq=2 * group * dim + 8)
    finally:
        b.close()


@pytest.mark.parametrize("page", [16, 32, 256])
@pytest.mark.parametrize("fmt", ["e4m3", "int8"])
def test_score_of_many_rows_over_pages(page, fmt):
    """Units that end inside a page, and pages that end inside a unit."""
    print(f"\n[gpu case] score pages of {page} {fmt}", flush=True)
    b = Tracked([90, 130, 64], [155, 130, 320], heads=8, kv_heads=2, dim=64, page=page, fmt=fmt, dtype="bf16", layers=2).open()
    try:
        b.fill(0)
        b.set()
        b.check_score()
    finally:
        b.close()


@pytest.mark.parametrize("kind", ["decode", "drafts", "prompts", "a long prompt"])
@pytest.mark.parametrize("what", ["k", "v"])
def test_keys_that_are_not_finite(kind, what):
    """A key (or value) with a NaN: the rows that see it add NaN to all they see, and to nothing else."""
    print(f"\n[gpu case] score NaN in {what}, {kind}", flush=True)
    b = Tracked(heads=4, kv_heads=2, dim=64, page=16, **KINDS[kind]).open()
    try:
        b.fill()
        b.set()
        b.put()
        b.score()
        clean, _ = b.get()
        s = int(np.argmax(b.q_len))
        j = int(b.length[s]) - int(b.q_len[s]) // 2 - 1             # seen by the sequence's last rows alone
        arr = [a.copy() for a in (b.k if what == "k" else b.v)]
        arr[s][j, 1, 3] = np.nan
        b.fill(**{what: arr})
        b.put()
        b.score()
        got, _ = b.get()
        row0 = int(np.sum(b.length[:s]))
        hit = np.zeros(clean.shape, bool)
        hit[row0: row0 + int(b.length[s]), 1] = True
        assert np.isnan(got[hit]).all() and np.array_equal(got[~hit], clean[~hit])
    finally:
        b.close()


@pytest.mark.parametrize("n", [255, 256, 257, 511, 1023, 1024, 1025, 2047, 4095, 16383])
@pytest.mark.parametrize("drop", [1, 3])
def test_a_few_over_the_budget(n, drop):
    """The step of a bounded server, at sizes around a block's rows of tokens; equal weights among them."""
    print(f"\n[gpu case] evict {drop} of {n}", flush=True)
    b = Tracked([0], [n], heads=2, kv_heads=2, dim=64, page=64, dtype="bf16").open()
    b.weight = np.round(b.weight, 1).astype(np.float32)
    try:
        b.fill()
        b.set()
        _evict(b, n - drop, min(20, n - drop))
    finally:
        b.close()


def test_two_streams():
    """Scores and evictions of one cache from two streams and two objects in turn: ordered by the library."""
    print("\n[gpu case] marks from two streams", flush=True)
    hip = hipmod()
    b = Tracked([1, 40], [600, 90], heads=4, kv_heads=2, dim=64, page=16).open()
    try:
        b.fill()
        b.set()
        b.put()
        b.score()
        b.seqs.evict(0, 50, 5, b.stream.h)
        want = b.get()
        other, mine = b.kv.seqs(2, 41, 60), b.stream
        second = hip.Stream()
        b.set(other, second)
        for _ in range(3):
            b.fill()
            d = [to_dev(b.weight), to_dev(b.place)]
            q = to_dev(store(b.q, b.dtype))
            out = [to_dev(np.zeros((690, 2), t)) for t in (np.float32, np.int32)]
            b.seqs.write_marks(0, d[0].ptr, d[1].ptr, mine.h)
            other.score(0, q.ptr, 0, b.scale, 0, second.h)
            b.seqs.evict(0, 50, 5, mine.h)
            other.read_marks(0, out[0].ptr, out[1].ptr, second.h)
            second.synchronize()
            mine.synchronize()
            for o, w in zip(out, want):
                assert np.array_equal(o.to_host(), w)
        b.stream = mine
        other.close()
        second.destroy()
    finally:
        b.close()


def test_a_pool_past_4_gib():
    """Pages whose codes lie past 4 GiB: marks, scores, an eviction and copies there."""
    print("\n[gpu case] pool past 4 GiB", flush=True)
    n_pages = (5 << 30) // (256 * 8 * 256) + 4                     # of k alone
    b = Tracked([1, 70], [300, 70], heads=8, kv_heads=8, dim=256, page=256, dtype="bf16", spare=0)
    shift = n_pages - b.n_pages
    b.pages = (b.pages + shift).astype(np.int32)
    b.open(n_pages)
    try:
        b.fill()
        b.set()
        b.check_score()
        b.fill()
        _evict(b, 64, 8)
        b.fill()
        b.put()
        b.kv.copy(b.pages, np.arange(len(b.pages)), None, b.stream.h)
        low = b.kv.seqs(2, 71, 8)
        low.set(b.q_len, b.length, b.page_off, np.arange(len(b.pages)), stream=b.stream.h)
        for a, w in zip(b.get(seqs=low), (b.weight, b.place)):
            assert np.array_equal(a, w)
    finally:
        b.close()
