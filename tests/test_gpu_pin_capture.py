"""salt_pin_base and salt_pin_base_fp8 on a stream under capture: the first pin of a table allocates and makes its
weight ready for calls that are not recorded, so it is refused and the capture goes on; a table that is pinned
can be pinned anew by a recorded call."""
import ctypes as C

import numpy as np
import pytest

import oracle
from oracle import serve
from tests.serve_harness import hipmod, store, to_dev, values
from tests.test_gpu_base import _check, _ctx
from tests.test_gpu_serve_graphs import _Graph
from tests.test_plan_capture import _graph_api

pytestmark = pytest.mark.gpu


def test_first_pin_under_capture_is_refused():
    print("\n[gpu case] first pin under capture", flush=True)
    from paper_2608_03579_amd import salt
    hip = hipmod()
    n_in, n_out, T = 264, 136, 5
    tables = [(n_in, n_out)] * 3
    ctx = _ctx("bf16", tables, T)
    s = hip.Stream()
    ws = [values((n_in, n_out), 5 + i, "bf16", 0.02) for i in range(2)]
    wd = [to_dev(store(w, "bf16")) for w in ws]
    codes, scales = to_dev(np.zeros((n_out, n_in), np.uint8)), to_dev(np.ones((2, 3), np.float32))
    xv = values((T, n_in), 3, "bf16")
    x, y = to_dev(store(xv, "bf16")), to_dev(np.zeros((T, n_out), np.uint16))

    def pins(tables_):
        return [f for t in tables_ for f in (lib.salt_pin_base(ctx.h, t, wd[0].ptr, n_out, s.h),
                                             lib.salt_pin_base_fp8(ctx.h, t, codes.ptr, n_in, scales.ptr, s.h))]

    lib, api = salt.lib, _graph_api(hip)
    try:
        for pinned in (False, True):                  # before the context has any base weight, and with one
            if pinned:
                ctx.pin_base(0, wd[0].ptr, n_out, s.h)
            graph = C.c_void_p()
            hip.check(api.hipStreamBeginCapture(s.h, 0), "begin capture")
            got = pins([1, 2])
            hip.check(api.hipStreamEndCapture(s.h, C.byref(graph)), "end capture")
            hip.check(api.hipGraphDestroy(graph), "destroy")
            assert got == [salt.ERR_BAD_STATE] * 4, got
            # (nothing was left pinned)
            n = C.c_int32(1)
            assert lib.salt_read_base(ctx.h, 1, x.ptr, n_out, s.h) == salt.ERR_BAD_STATE
            assert lib.salt_base_product(ctx.h, 1, C.byref(n), T, x.ptr, (C.c_void_p * 1)(y.ptr), s.h) == salt.ERR_BAD_STATE
        # a recorded pin of a pinned table: the products behind a replay see the new weight
        run = lambda: ctx.base_product([0], T, x.ptr, [y.ptr], s.h)
        g = _Graph(hip, s, lambda: ctx.pin_base(0, wd[1].ptr, n_out, s.h))
        xd = serve.quantise_x(xv)
        for replays, w in ((0, ws[0]), (1, ws[1])):
            for _ in range(replays):
                g.launch()
            run()
            s.synchronize()
            _check(oracle.decode(y.to_host(), "bf16"), xd, serve.quantise_weight(w), "bf16")
        for t in (1, 2):
            ctx.pin_base(t, wd[1].ptr, n_out, s.h)
        ctx.base_product([2], T, x.ptr, [y.ptr], s.h)
        s.synchronize()
        _check(oracle.decode(y.to_host(), "bf16"), xd, serve.quantise_weight(ws[1]), "bf16")
        g.close()
    finally:
        ctx.close()
        s.destroy()
