"""The operators of a decoding server together, as a server runs them: rotation, cache, attention, scoring and eviction
step after step; the same recorded into a graph; beams that fork; and what the calls refuse."""
import ctypes as C

import numpy as np
import pytest

import oracle
from oracle import serve
from oracle import steps as o64
from paper_2608_03579_amd import salt
from tests.serve_harness import Batch, hipmod, store, to_dev, values
from tests.test_gpu_serve_graphs import _Graph

pytestmark = pytest.mark.gpu
HEADS, KV, DIM, PAGE = 4, 2, 64, 16
SCALE = float(np.float32(DIM ** -0.5))
FREQ = 10000.0 ** (-np.arange(0, DIM, 2) / DIM)


class Server:
    def __init__(self, n_seqs, pages_each, dtype="f32", layers=1):
        self.hip, self.dtype = hipmod(), dtype
        self.ctx = salt.Context(dtype, [(64, 64)], 0, 0, 1, 0, 1)
        self.kv = self.ctx.kv_cache(layers, HEADS, KV, DIM, PAGE, n_seqs * pages_each + 8, "int8")
        self.kv.track()
        self.stream = self.hip.Stream()
        self.rot = self.ctx.rotation(HEADS, KV, DIM, FREQ)
        self.off = (np.arange(n_seqs + 1) * pages_each).astype(np.int32)
        self.pages = np.random.default_rng(1).permutation(n_seqs * pages_each).astype(np.int32)
        self.n = n_seqs

    def buffers(self, T):
        sdt = np.float32 if self.dtype == "f32" else np.uint16
        z = lambda h: to_dev(np.zeros((T, h, DIM), sdt))
        return dict(q=z(HEADS), k=z(KV), v=z(KV), out=z(HEADS), pos=to_dev(np.zeros(T, np.int32)))

    def upload(self, d, q, k, v, pos):
        for name, a in (("q", q), ("k", k), ("v", v)):
            d[name].upload(store(a, self.dtype))
        d["pos"].upload(np.asarray(pos, np.int32))

    def step(self, seqs, d, T, keep=None, recent=0, layer=0):
        s = self.stream.h
        self.ctx.rotate(self.rot, T, d["pos"].ptr, d["q"].ptr, d["q"].ptr, d["k"].ptr, d["k"].ptr, s)
        seqs.write(layer, d["k"].ptr, d["v"].ptr, s)
        seqs.attend(layer, d["q"].ptr, d["out"].ptr, SCALE, s)
        seqs.score(layer, d["q"].ptr, d["pos"].ptr, SCALE, 0, s)
        if keep is not None:
            seqs.evict(layer, keep, recent, s)

    def close(self):
        self.ctx.close()
        self.stream.destroy()


def _inputs(T, seed):
    return [values((T, h, DIM), seed * 10 + i, "f32") for i, h in enumerate((HEADS, KV, KV))]


def test_bounded_decoding_against_float64():
    """Prompts, then tokens one at a time under a budget: attention over what eviction left. The oracle holds the
    rotated, quantised keys of every kv head in the order of their places, and takes the eviction's choice from the marks
    that libsalt read back (they equal the oracle's own within the bound of a weight)."""
    print("\n[gpu case] bounded decoding", flush=True)
    lens, keep, recent, steps = [40, 9, 25], 24, 6, 12
    sv = Server(3, 4)
    seqs = sv.kv.seqs(3, 80, 12)
    try:
        total = np.array(lens)                                     # tokens seen so far
        held = None
        cur = np.array(lens)
        for step in range(steps):
            q_len = np.array(lens) if step == 0 else np.ones(3, int)
            T = int(q_len.sum())
            if step:
                total = total + 1
                cur = np.minimum(cur, keep) + 1
            pos = np.concatenate([np.arange(t - n, t) for t, n in zip(total, q_len)])
            q, k, v = _inputs(T, 50 + step)
            d = sv.buffers(T)
            sv.upload(d, q, k, v, pos)
            seqs.set(q_len, cur, sv.off, sv.pages, stream=sv.stream.h)
            sv.step(seqs, d, T)
            sv.stream.synchronize()
            out = d["out"].to_host().astype(np.float64)
            rq = d["q"].to_host().astype(np.float64)
            assert np.abs(rq - o64.rotate(q, pos, FREQ, False)[0]).max() < 1e-4
            rk = serve.quantise_kv(d["k"].to_host().astype(np.float64), "int8")
            rv = serve.quantise_kv(v, "int8")
            if held is None:
                held = [[(np.zeros((0, DIM)), np.zeros((0, DIM)), np.zeros(0)) for _ in range(KV)] for _ in range(3)]
            marks = [to_dev(np.zeros((int(cur.sum()), KV), t)) for t in (np.float32, np.int32)]
            seqs.read_marks(0, marks[0].ptr, marks[1].ptr, sv.stream.h)
            sv.stream.synchronize()
            weight, place = (m.to_host() for m in marks)
            seqs.evict(0, keep, recent, sv.stream.h)
            t0, r0 = np.concatenate([[0], np.cumsum(q_len)]), np.concatenate([[0], np.cumsum(cur)])
            for s in range(3):
                for h in range(KV):
                    hk, hv, hw = held[s][h]
                    rows = slice(t0[s], t0[s + 1])
                    hk, hv = np.concatenate([hk, rk[rows, h]]), np.concatenate([hv, rv[rows, h]])
                    hw = np.concatenate([hw, np.zeros(q_len[s])])
                    old = len(hk) - q_len[s]
                    for j in range(q_len[s]):
                        for g in range(HEADS // KV):
                            row = rq[t0[s] + j, h * (HEADS // KV) + g]
                            ref, mass, big = serve.attend(row, hk[: old + j + 1], hv[: old + j + 1], SCALE)
                            err = np.abs(out[t0[s] + j, h * (HEADS // KV) + g] - ref)
                            assert np.all(err <= (4 * DIM * 2.0 ** -24 * big + 2.0 ** -17) * mass + 1e-30), (step, s, h, j)
                            hw[: old + j + 1] += o64.weights(row, hk[: old + j + 1], SCALE)[0]
                    mine = weight[r0[s]: r0[s + 1], h]
                    assert np.allclose(mine, hw, rtol=1e-4, atol=1e-9), (step, s, h)
                    src = o64.evict(mine, place[r0[s]: r0[s + 1], h], keep, recent)
                    held[s][h] = hk[src], hv[src], hw[src]
    finally:
        sv.close()


def test_a_step_replays():
    """Rotation, write, attention, scoring and eviction of a steady step (one token over the budget) in a graph: the same
    state and outputs as the eager steps on a second cache, also with eager steps in between."""
    print("\n[gpu case] captured bounded step", flush=True)
    n, keep = 5, 37
    servers = [Server(n, 3, "bf16") for _ in range(2)]
    seqs, bufs = [], []
    try:
        for sv in servers:
            first = sv.kv.seqs(n, n * keep, 3 * n)
            first.set([keep] * n, [keep] * n, sv.off, sv.pages, stream=sv.stream.h)
            d = sv.buffers(n * keep)
            sv.upload(d, *_inputs(n * keep, 7), np.tile(np.arange(keep), n))
            sv.step(first, d, n * keep)
            q = sv.kv.seqs(n, n, 3 * n)
            q.set([1] * n, [keep + 1] * n, sv.off, sv.pages, stream=sv.stream.h)
            seqs.append(q)
            bufs.append(sv.buffers(n))
            sv.stream.synchronize()
        eager, taped = servers
        go = lambda i: servers[i].step(seqs[i], bufs[i], n, keep, 5)
        graph = _Graph(taped.hip, taped.stream, lambda: go(1))
        for step in range(8):
            x = _inputs(n, 100 + step) + [np.full(n, keep + step)]
            for sv, d in zip(servers, bufs):
                sv.upload(d, *x)
            go(0)
            if step == 3:
                go(1)
            else:
                graph.launch()
            got = []
            for sv, q, d in zip(servers, seqs, bufs):
                marks = [to_dev(np.zeros((n * (keep + 1), KV), t)) for t in (np.float32, np.int32)]
                kv = [to_dev(np.zeros((n * (keep + 1), KV, DIM), np.uint16)) for _ in range(2)]
                q.read_marks(0, marks[0].ptr, marks[1].ptr, sv.stream.h)
                q.read(0, "own", kv[0].ptr, kv[1].ptr, sv.stream.h)
                sv.stream.synchronize()
                got.append([a.to_host() for a in (d["out"], *marks, *kv)])
            for a, b in zip(*got):
                assert np.array_equal(a, b), step
        graph.close()
    finally:
        for sv in servers:
            sv.close()


def test_selection_and_rotation_replay():
    print("\n[gpu case] captured selection", flush=True)
    hip = hipmod()
    ctx = salt.Context("bf16", [(64, 64)], 0, 0, 1, 0, 1)
    stream = hip.Stream()
    beams = ctx.beams(12, 8)
    xs = [store(values((12, 5000), 40 + i, "bf16", 2.0), "bf16") for i in range(3)]
    x, score = to_dev(xs[0]), to_dev(np.linspace(-2, 0, 12).astype(np.float32))
    out = [to_dev(np.zeros((3, 8), t)) for t in (np.float32, np.int32, np.int32)]
    pos, rot = to_dev(np.arange(12, dtype=np.int32)), ctx.rotation(4, 0, 64, FREQ)
    y = to_dev(np.zeros((12, 256), np.uint16))
    try:
        def run():
            beams.select(3, 4, 5000, x.ptr, score.ptr, 8, *[o.ptr for o in out], stream.h)
            ctx.rotate(rot, 12, pos.ptr, x.ptr, y.ptr, 0, 0, stream.h, ldq=5000)

        want = []
        for v in xs:
            x.upload(v)
            run()
            stream.synchronize()
            want.append([d.to_host() for d in (*out, y)])
        g = _Graph(hip, stream, run)
        for i in (1, 0, 2, 2, 1):
            x.upload(xs[i])
            g.launch()
            stream.synchronize()
            for d, w in zip((*out, y), want[i]):
                assert np.array_equal(d.to_host(), w), i
            run()
            stream.synchronize()
        # a capture elsewhere may not be ordered behind the scratch's last work
        other, graph = hip.Stream(), C.c_void_p()
        hip.check(g.lib.hipStreamBeginCapture(other.h, 0), "begin capture")
        st = beams.select_status(3, 4, 5000, x.ptr, score.ptr, 8, *[o.ptr for o in out], other.h)
        hip.check(g.lib.hipStreamEndCapture(other.h, C.byref(graph)), "end capture")
        hip.check(g.lib.hipGraphDestroy(graph), "destroy")
        assert st == salt.ERR_BAD_STATE
        g.close()
    finally:
        ctx.close()
        stream.destroy()


def test_beams_fork_over_the_cache():
    """Four beams of a request share the full pages of their past; each step the host reorders the tables and copies the
    last pages of beams that go on twice. Attention of every beam against its own history in float64."""
    print("\n[gpu case] beams over the cache", flush=True)
    width, vocab, steps, layers = 4, 301, 20, 2
    sv = Server(width, 8, "f32", layers)
    seqs, beams = sv.kv.seqs(width, width, 8 * width), sv.ctx.beams(width, width)
    rng = np.random.default_rng(9)
    try:
        tables, free = [[] for _ in range(width)], list(range(width * 8 + 8))
        hist = [[np.zeros((0, KV, DIM)), np.zeros((0, KV, DIM))] for _ in range(width)]
        score = np.array([0, -np.inf, -np.inf, -np.inf], np.float32)
        d = sv.buffers(width)
        for step in range(steps):
            if step % PAGE == 0:
                for t in tables:
                    t.append(free.pop())
            off = np.concatenate([[0], np.cumsum([len(t) for t in tables])])
            seqs.set([1] * width, [step + 1] * width, off, np.concatenate(tables), stream=sv.stream.h)
            q, k, v = _inputs(width, 300 + step)
            sv.upload(d, q, k, v, [step] * width)
            s = sv.stream.h
            sv.ctx.rotate(sv.rot, width, d["pos"].ptr, d["q"].ptr, d["q"].ptr, d["k"].ptr, d["k"].ptr, s)
            for layer in range(layers):
                seqs.write(layer, d["k"].ptr, d["v"].ptr, s)
            logits = values((width, vocab), 600 + step, "f32", 2.0)
            ld, lg = -(-vocab // 8) * 8, np.zeros((width, -(-vocab // 8) * 8), np.float32)
            lg[:, :vocab] = logits
            x, sc = to_dev(lg), to_dev(score)
            out = [to_dev(np.zeros((1, width), t)) for t in (np.float32, np.int32, np.int32)]
            beams.select(1, width, vocab, x.ptr, sc.ptr, width, *[o.ptr for o in out], s, ld=ld)
            for layer in range(layers):
                seqs.attend(layer, d["q"].ptr, d["out"].ptr, SCALE, s)
                sv.stream.synchronize()
                got, rq = d["out"].to_host().astype(np.float64), d["q"].to_host().astype(np.float64)
                if layer == 0:
                    rk, rv = serve.quantise_kv(d["k"].to_host().astype(np.float64), "int8"), serve.quantise_kv(v, "int8")
                    for b in range(width):
                        hist[b] = [np.concatenate([hist[b][0], rk[b:b + 1]]), np.concatenate([hist[b][1], rv[b:b + 1]])]
                for b in range(width):
                    for h in range(HEADS):
                        ref, mass, big = serve.attend(rq[b, h], hist[b][0][:, h // 2], hist[b][1][:, h // 2], SCALE)
                        assert np.all(np.abs(got[b, h] - ref) <= (4 * DIM * 2.0 ** -24 * big + 2.0 ** -17) * mass + 1e-30), (step, b, h)
            worth, parent, token = (o.to_host()[0] for o in out)
            wv, wb, wt = o64.beam_select(o64.beam_worth(logits, score), width)
            assert np.array_equal(parent, wb) and np.array_equal(token, wt) and np.allclose(worth, wv, atol=1e-5)
            score = worth
            # the first child of a beam keeps its last page, others get a copy; full pages are shared
            taken, src, dst, new = set(), [], [], []
            used = {p for b in set(parent.tolist()) for p in tables[b]}
            spare = [p for p in range(width * 8 + 8) if p not in used]
            for b in parent.tolist():
                t = list(tables[b])
                if b in taken and (step + 1) % PAGE:
                    src.append(t[-1])
                    dst.append(spare.pop())
                    t[-1] = dst[-1]
                taken.add(b)
                new.append(t)
            sv.kv.copy(src, dst, [(step % PAGE) + 1] * len(src), s)
            tables, free = new, spare
            hist = [list(hist[b]) for b in parent.tolist()]
    finally:
        sv.close()


def test_refusals():
    """Every call that is refused leaves marks and cache as they were."""
    print("\n[gpu case] refusals", flush=True)
    sv = Server(2, 3, "f32")
    plain = sv.ctx.kv_cache(1, HEADS, KV, DIM, PAGE, 4)
    seqs, untracked, unset = sv.kv.seqs(4, 8, 8), plain.seqs(2, 4, 4), sv.kv.seqs(2, 4, 4)
    d = sv.buffers(8)
    m = [to_dev(np.zeros((64, KV), np.float32)) for _ in range(2)]
    p = m[0].ptr
    bad, rng_, arg = salt.ERR_BAD_STATE, salt.ERR_OUT_OF_RANGE, salt.ERR_INVALID_ARG
    try:
        untracked.set([1, 1], [4, 4], [0, 1, 2], [0, 1])
        seqs.set([1, 1], [20, 30], [0, 2, 4], [0, 1, 2, 3])
        for q in (untracked, unset):
            assert q.score_status(0, d["q"].ptr, 0, SCALE) == bad
            assert q.evict_status(0, 3, 1) == bad
            assert q.read_marks_status(0, p, p) == bad
            assert q.write_marks_status(0, p, p) == bad
        assert seqs.score_status(1, d["q"].ptr, 0, SCALE) == rng_
        assert seqs.score_status(0, d["q"].ptr, 0, SCALE, -1) == rng_
        assert seqs.score_status(0, 0, 0, SCALE) == arg
        assert seqs.score_status(0, d["q"].ptr + 4, 0, SCALE) == arg
        assert seqs.score_status(0, d["q"].ptr, 2, SCALE) == arg
        assert seqs.score_status(0, d["q"].ptr, 0, SCALE, ldq=HEADS * DIM - 8) == arg
        assert seqs.score_status(0, d["q"].ptr, 0, SCALE, ldq=HEADS * DIM + 4) == arg
        for scale in (0.0, -1.0, np.nan, np.inf):
            assert seqs.score_status(0, d["q"].ptr, 0, scale) == arg
        for keep, recent in ((-1, 0), (5, -1), (5, 6)):
            assert seqs.evict_status(0, keep, recent) == rng_
        assert seqs.evict_status(-1, 5, 0) == rng_
        assert seqs.read_marks_status(0, 0, p) == arg and seqs.write_marks_status(0, p, p + 4) == arg
        # a page that holds tokens of two sequences, of one twice, or of a sequence and a domain
        for args in (([1, 1], [20, 20], [0, 2, 4], [0, 1, 0, 2]), ([1], [20], [0, 2], [1, 1]),
                     ([1], [20], [0, 2], [0, 1], [0], [16], [0, 1], [1])):
            seqs.set(*args)
            assert seqs.score_status(0, d["q"].ptr, 0, SCALE) == arg
            assert seqs.evict_status(0, 3, 1) == arg
            assert seqs.write_marks_status(0, p, p) == arg
            assert seqs.read_marks_status(0, p, p) == salt.OK
        # (a shared page past the last token is none)
        seqs.set([1, 1], [16, 16], [0, 2, 4], [0, 1, 2, 1])
        assert seqs.write_marks_status(0, p, p) == salt.OK
        kv = sv.kv
        for src, dst, tok, want in (([0], [6 + 8], None, rng_), ([-1], [1], None, rng_), ([0], [1], [17], rng_),
                                    ([0], [1], [-1], rng_), ([0, 1], [2, 2], None, arg), ([0, 1], [1, 2], None, arg),
                                    ([3], [3], None, arg), (list(range(14)) + [0], list(range(15)), None, rng_)):
            assert kv.copy_status(src, dst, tok) == want, (src, dst, tok)
        assert kv.copy_status([], []) == salt.OK and kv.copy_status([0, 0], [1, 2], [0, 16]) == salt.OK
        sv.hip.synchronize()
    finally:
        sv.close()
    assert seqs.h is None and seqs.score_status(0, 16, 0, SCALE) == arg and seqs.evict_status(0, 1, 0) == arg


def test_objects_end_with_their_context_or_before():
    print("\n[gpu case] object ends", flush=True)
    hipmod()
    ctx = salt.Context("f32", [(64, 64)], 0, 0, 1, 0, 1)
    other = salt.Context("f32", [(64, 64)], 0, 0, 1, 0, 1)
    a, b = ctx.beams(4, 4), ctx.beams(8, 64)
    assert salt.lib.salt_beam_select(other.h, a.h, 1, 1, 8, 16, 0, 16, 1, 16, 16, 16, None) == salt.ERR_INVALID_ARG
    salt.lib.salt_beams_destroy(other.h, a.h)                      # (not its own: nothing happens)
    gone = a.h
    a.close()
    assert a.select_status(1, 1, 8, 16, 16, 1, 16, 16, 16) == salt.ERR_INVALID_ARG
    assert salt.lib.salt_beam_select(ctx.h, gone, 1, 1, 8, 16, 0, 16, 1, 16, 16, 16, None) == salt.ERR_INVALID_ARG
    kv = ctx.kv_cache(1, 1, 1, 64, 16, 4)
    assert salt.lib.salt_kv_track(other.h, kv.h) == salt.ERR_INVALID_ARG
    kv.track()
    kv.track()                                                     # (a second call does nothing)
    kv.close()
    assert salt.lib.salt_kv_track(ctx.h, None) == salt.ERR_INVALID_ARG
    ctx.close()
    other.close()
    assert b.h is None
