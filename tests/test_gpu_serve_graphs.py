"""The base product, the cache write and read and the attention recorded into a HIP graph and replayed with other
inputs in the same buffers, the program's own eager work in between: every replay equals the eager
result.  And what a capture refuses: work ordered behind another stream, and a new batch for recorded calls."""
import ctypes as C

import numpy as np
import pytest

from tests.serve_harness import Batch, hipmod, store, to_dev, values
from tests.test_plan_capture import _graph_api

pytestmark = pytest.mark.gpu


class _Graph:
    def __init__(self, hip, stream, work):
        self.hip, self.lib, self.stream = hip, _graph_api(hip), stream
        graph = C.c_void_p()
        self.ex = C.c_void_p()
        hip.check(self.lib.hipStreamBeginCapture(stream.h, 0), "begin capture")
        work()
        hip.check(self.lib.hipStreamEndCapture(stream.h, C.byref(graph)), "end capture")
        hip.check(self.lib.hipGraphInstantiate(C.byref(self.ex), graph, None, None, 0), "instantiate")
        hip.check(self.lib.hipGraphDestroy(graph), "destroy")

    def launch(self):
        self.hip.check(self.lib.hipGraphLaunch(self.ex, self.stream.h), "launch")

    def close(self):
        self.hip.check(self.lib.hipGraphExecDestroy(self.ex), "destroy")


@pytest.mark.parametrize("T", [3, 40, 700])
def test_base_product_replays(T):
    print(f"\n[gpu case] captured base product T={T}", flush=True)
    from paper_2608_03579_amd import salt
    hip = hipmod()
    n_in, n_out = 392, 264
    ctx = salt.Context("bf16", [(n_in, n_out)], 0, 0, 1, 0, T)
    s, other = hip.Stream(), hip.Stream()
    wd = to_dev(store(values((n_in, n_out), 5, "bf16", 0.02), "bf16"))
    xs = [store(values((T, n_in), 30 + i, "bf16"), "bf16") for i in range(4)]
    x, y = to_dev(xs[0]), to_dev(np.zeros((T, n_out), np.uint16))
    try:
        ctx.pin_base(0, wd.ptr, n_out, s.h)
        run = lambda: ctx.base_product([0], T, x.ptr, [y.ptr], s.h)
        want = []
        for v in xs:
            x.upload(v)
            run()
            s.synchronize()
            want.append(y.to_host())
        g = _Graph(hip, s, run)
        for k in (2, 0, 1, 3, 2, 0):
            x.upload(xs[k])
            y.upload(np.full((T, n_out), 9, np.uint16))
            g.launch()
            s.synchronize()
            assert np.array_equal(y.to_host(), want[k]), k
            if k == 1:
                run()                                        # eager work in between
                s.synchronize()
        # a capture elsewhere may not be ordered behind the last product: refused, and nothing is broken
        lib = g.lib
        graph = C.c_void_p()
        hip.check(lib.hipStreamBeginCapture(other.h, 0), "begin capture")
        st = salt.lib.salt_base_product(ctx.h, 1, (C.c_int32 * 1)(0), T, x.ptr, (C.c_void_p * 1)(y.ptr), other.h)
        hip.check(lib.hipStreamEndCapture(other.h, C.byref(graph)), "end capture")
        hip.check(lib.hipGraphDestroy(graph), "destroy")
        assert st == salt.ERR_BAD_STATE
        run()
        s.synchronize()
        g.close()
    finally:
        ctx.close()


def test_cache_and_attention_replay():
    print("\n[gpu case] captured cache and attention", flush=True)
    from paper_2608_03579_amd import salt
    hip = hipmod()
    b = Batch([1] * 20 + [70, 3], [30 + 9 * i for i in range(20)] + [300, 40], prefix=[200, 90],
              domain=[0] * 15 + [-1] * 5 + [1, 0], heads=8, kv_heads=2, dim=128, page=64).open()
    rng = np.random.default_rng(3)
    shape = (b.T, b.kv_heads, b.dim)
    sets = [[store(rng.standard_normal(sh), "bf16") for sh in (shape, shape, (b.T, b.heads, b.dim))] for _ in range(3)]
    k, v, q = (to_dev(a) for a in sets[0])
    out, rk, rv = to_dev(np.zeros((b.T, b.heads, b.dim), np.uint16)), to_dev(np.zeros(shape, np.uint16)), to_dev(np.zeros(shape, np.uint16))
    try:
        b.fill()
        b.set()

        def run():
            b.seqs.write(0, k.ptr, v.ptr, b.stream.h)
            b.seqs.attend(0, q.ptr, out.ptr, b.scale, b.stream.h)
            b.seqs.read(0, "new", rk.ptr, rv.ptr, b.stream.h)

        def load(i):
            for d, a in zip((k, v, q), sets[i]):
                d.upload(a)

        want = []
        for i in range(3):
            load(i)
            run()
            b.stream.synchronize()
            want.append([d.to_host() for d in (out, rk, rv)])
        g = _Graph(hip, b.stream, run)
        for i in (1, 0, 2, 2, 1, 0):
            load(i)
            g.launch()
            b.stream.synchronize()
            for d, w in zip((out, rk, rv), want[i]):
                assert np.array_equal(d.to_host(), w), i
            if i == 2:
                run()
                b.stream.synchronize()
        # the graph keeps the batch: no other takes its place
        assert b.seqs.set_status(b.q_len, b.length, b.page_off, b.pages, stream=b.stream.h) == salt.ERR_BAD_STATE
        g.launch()
        b.stream.synchronize()
        assert np.array_equal(out.to_host(), want[0][0])
        # nor can a batch be set under capture
        fresh = b.kv.seqs(1, 1, 1)
        graph = C.c_void_p()
        hip.check(g.lib.hipStreamBeginCapture(b.stream.h, 0), "begin capture")
        st = fresh.set_status([1], [1], [0, 1], [0], stream=b.stream.h)
        hip.check(g.lib.hipStreamEndCapture(b.stream.h, C.byref(graph)), "end capture")
        hip.check(g.lib.hipGraphDestroy(graph), "destroy")
        assert st == salt.ERR_BAD_STATE
        g.close()
    finally:
        b.close()
