"""GPU parity of the base product in each of its kernels, at the edges where they can go wrong: one, two, an odd and an
even number of input blocks, more of them than a block's waves; tokens and outputs that end inside a tile; several
tables; grids that are and are not a multiple of 8, token tiles that fill no band of four.  A zero token and one that is
not finite stand among the others.  Which kernel a case takes is pinned by tests/test_base_rule.py, with the
rule that the library uses.  Bounds as in tests/test_gpu_base.py."""
import numpy as np
import pytest

import oracle
from oracle import serve
from tests.serve_harness import hipmod, store, to_dev, values
from tests.test_gpu_base import _check, _ctx, _pin, _product
from tests.test_gpu_serve_graphs import _Graph

pytestmark = pytest.mark.gpu

CASES = [  # dtype, in, outs, T, kernel (outputs x tokens of a block; few: tiles of 16 outputs a block)
    ("bf16", 4360, [520], 13, "few 1"), ("f32", 4360, [520], 7, "few 1"),
    ("bf16", 136, [4104, 264], 1, "few 2"), ("bf16", 4360, [4104], 3, "few 2"), ("bf16", 264, [4104], 16, "few 2"),
    ("f32", 264, [4120], 8, "few 2"), ("f32", 4360, [4104], 2, "few 2"),
    ("bf16", 1032, [600], 511, "split 32x32"), ("f32", 1032, [600], 511, "split 32x32"),
    ("bf16", 640, [2056], 200, "split 32x64"), ("f32", 264, [2056, 8], 190, "split 32x64"),
    ("bf16", 1032, [4104], 250, "split 64x64"), ("f32", 1032, [4104], 203, "split 64x64"),
    ("bf16", 136, [2056, 2056], 257, "split 64x64"), ("f32", 136, [4104], 250, "split 64x64"),
    ("bf16", 72, [2952], 900, "tile 128x128"), ("bf16", 264, [2952], 1100, "tile 128x128"),
    ("bf16", 512, [1288, 1672], 1100, "tile 128x128"),
    ("f32", 72, [2952], 900, "tile 128x128"), ("f32", 136, [2824], 1100, "tile 128x128"),
    ("f32", 392, [1288, 1672], 1100, "tile 128x128"),
    ("bf16", 392, [3848], 1500, "tile 128x256"), ("bf16", 72, [4000], 1600, "tile 128x256"),
    ("bf16", 136, [2056, 2000], 1600, "tile 128x256"),
    ("bf16", 72, [3080, 2568], 2200, "tile 256x256"), ("bf16", 136, [2824], 3841, "tile 256x256"),
    ("bf16", 264, [2824], 3841, "tile 256x256"), ("bf16", 520, [5896], 1900, "tile 256x256"),
]
_name = lambda c: f"{c[0]}-{c[4]}-{c[1]}-{'+'.join(map(str, c[2]))}-T{c[3]}".replace(" ", "")


@pytest.mark.parametrize("case", CASES, ids=_name)
def test_parity(case):
    dtype, n_in, outs, T, kernel = case
    print(f"\n[gpu case] base {kernel}: {dtype} {n_in}->{outs} T={T}", flush=True)
    ctx = _ctx(dtype, [(n_in, o) for o in outs], T)
    try:
        ws = [values((n_in, o), 10 + i, dtype, 0.02) for i, o in enumerate(outs)]
        for i, w in enumerate(ws):
            _pin(ctx, i, w, dtype)
        x = values((T, n_in), 3, dtype, uneven=True)
        good = np.ones(T, bool)
        if T > 2:
            x[T // 2] = 0.0
            x[T - 2, n_in - 1] = np.nan
            good[T - 2] = False
        got = _product(ctx, list(range(len(outs))), outs, x, dtype)
        xd = serve.quantise_x(x[good])
        for y, w in zip(got, ws):
            assert np.isnan(y[~good]).all()
            _check(y[good], xd, serve.quantise_weight(w), dtype)
            assert np.all(y[(x == 0).all(1)] == 0)
    finally:
        ctx.close()


ONE_EACH = [c for i, c in enumerate(CASES) if (c[0], c[4]) not in [(d[0], d[4]) for d in CASES[:i]]]


@pytest.mark.parametrize("case", ONE_EACH, ids=_name)
def test_weights_that_are_not_finite(case):
    """An infinity in W: the outputs of its block are NaN, those of the blocks beside it as without."""
    dtype, n_in, outs, T, kernel = case
    print(f"\n[gpu case] base {kernel}, weight not finite: {dtype} {n_in}->{outs} T={T}", flush=True)
    n_out = outs[0]
    w = values((n_in, n_out), 10, dtype, 0.02)
    block = (n_out // 2) // 128 * 128
    bad = w.copy()
    bad[n_in - 1, block + 3] = np.inf
    ctx = _ctx(dtype, [(n_in, o) for o in outs], T)
    try:
        for i, o in enumerate(outs[1:]):
            _pin(ctx, i + 1, np.zeros((n_in, o)), dtype)
        x = values((T, n_in), 3, dtype)
        y = []
        for v in (w, bad):
            _pin(ctx, 0, v, dtype)
            y.append(_product(ctx, list(range(len(outs))), outs, x, dtype)[0])
        cols = np.zeros(n_out, bool)
        cols[block: block + 128] = True
        assert np.isnan(y[1][:, cols]).all() and np.array_equal(y[1][:, ~cols], y[0][:, ~cols])
    finally:
        ctx.close()


@pytest.mark.parametrize("case", ONE_EACH, ids=_name)
def test_replays_and_streams(case):
    """Recorded into a graph and replayed with other inputs, eager calls on the same and on another stream in between,
    none of them waited for: every result equals, bit for bit, the one alone."""
    dtype, n_in, outs, T, kernel = case
    print(f"\n[gpu case] base {kernel}, replays: {dtype} {n_in}->{outs} T={T}", flush=True)
    hip = hipmod()
    sdt = np.float32 if dtype == "f32" else np.uint16
    ctx = _ctx(dtype, [(n_in, o) for o in outs], T)
    s, other = hip.Stream(), hip.Stream()
    n = len(outs)
    try:
        for i, o in enumerate(outs):
            _pin(ctx, i, values((n_in, o), 10 + i, dtype, 0.02), dtype)
        xs = [to_dev(store(values((T, n_in), 30 + i, dtype), dtype)) for i in range(3)]
        x = to_dev(np.zeros((T, n_in), sdt))
        ys = [[to_dev(np.zeros((T, o), sdt)) for o in outs] for _ in range(4)]
        run = lambda xd, y, st: ctx.base_product(list(range(n)), T, xd.ptr, [d.ptr for d in y], st.h)
        want = []
        for i in range(3):
            run(xs[i], ys[0], s)
            s.synchronize()
            want.append([d.to_host() for d in ys[0]])
            assert all(np.isfinite(oracle.decode(h, dtype)).all() for h in want[i])
        # two streams in turn, nothing waited for
        for i in range(3):
            run(xs[i], ys[i], other if i == 1 else s)
        s.synchronize()
        other.synchronize()
        for i in range(3):
            assert all(np.array_equal(d.to_host(), w) for d, w in zip(ys[i], want[i])), i
        g = _Graph(hip, s, lambda: run(x, ys[3], s))
        for i in (2, 0, 1, 1, 0):
            for d in ys[3]:
                d.upload(np.full(d.shape, 9, sdt))
            x.copy_from(xs[i], s)
            g.launch()
            run(xs[(i + 1) % 3], ys[0], s)
            s.synchronize()
            assert all(np.array_equal(d.to_host(), w) for d, w in zip(ys[3], want[i])), i
            assert all(np.array_equal(d.to_host(), w) for d, w in zip(ys[0], want[(i + 1) % 3])), i
        g.close()
    finally:
        ctx.close()
        s.destroy()
        other.destroy()
