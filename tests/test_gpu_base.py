"""GPU parity of the base product in 8 bits (salt_pin_base, salt_pin_base_fp8, salt_read_base,
salt_base_product) with the float64 oracle.

The weight must be held exactly as the oracle quantises it.  The product's bound per element, with
A = sum_k |xq wq| (scales included): bf16 contexts 2^-8 |ref| for y's rounding and 2^-12 A for the
matrix instruction's short sums (a dropped block of 128 inputs moves y by about 2^-7 A or more);
fp32 contexts 2^-22 |ref| + (in / 16 + 8) 2^-24 A, the fp32 chain."""
import numpy as np
import pytest

import oracle
from oracle import serve
from tests.serve_harness import hipmod, store, to_dev, values

pytestmark = pytest.mark.gpu


def _ctx(dtype, tables, max_tokens):
    from paper_2608_03579_amd import salt
    return salt.Context(dtype, tables, 0, 0, 1, 0, max_tokens)


def _pin(ctx, t, w, dtype, ld=None):
    n_in, n_out = w.shape
    ld = ld or n_out
    buf = np.zeros((n_in, ld), np.float32 if dtype == "f32" else np.uint16)
    buf[:, :n_out] = store(w, dtype)
    buf[:, n_out:] = store(np.full((n_in, ld - n_out), 1e4), dtype)
    wd = to_dev(buf)
    ctx.pin_base(t, wd.ptr, ld)
    hipmod().synchronize()
    wd.free()


def _product(ctx, tables, outs, x, dtype, stream=None):
    T = x.shape[0]
    xd = to_dev(store(x, dtype))
    guard = 64
    ys = [to_dev(np.full(T * o + guard, 7, np.float32 if dtype == "f32" else np.uint16)) for o in outs]
    s = stream or hipmod().Stream()
    ctx.base_product(tables, T, xd.ptr, [y.ptr for y in ys], s.h)
    s.synchronize()
    host = [y.to_host() for y in ys]
    for y in ys + [xd]:
        y.free()
    for h, o in zip(host, outs):
        assert np.all(h[T * o:] == 7), "the product wrote past y"
    return [oracle.decode(h[: T * o].reshape(T, o), dtype) for h, o in zip(host, outs)]


def _check(got, xd, wd, dtype):
    ref, mass = xd @ wd, np.abs(xd) @ np.abs(wd)
    if dtype == "bf16":
        bound = 2.0 ** -8 * np.abs(ref) + 2.0 ** -12 * mass
    else:
        bound = 2.0 ** -22 * np.abs(ref) + (xd.shape[1] / 16 + 8) * 2.0 ** -24 * mass
    bad = np.abs(got - ref) > bound + 1e-37
    assert not bad.any(), f"{int(bad.sum())} of {bad.size} elements out of bound"


CASES = [  # in, outs, T
    (8, [8], 1), (128, [128], 1), (136, [24], 2), (120, [8, 264], 16), (256, [256], 17), (520, [776, 8], 33),
    (1024, [1024, 256, 256], 64), (2056, [520], 65), (392, [1032], 129), (640, [2056], 200), (264, [136, 512], 257),
    (1032, [600], 511),
]


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_in,outs,T", CASES)
def test_product_parity(n_in, outs, T, dtype):
    print(f"\n[gpu case] base {dtype} {n_in}->{outs} T={T}", flush=True)
    ctx = _ctx(dtype, [(n_in, o) for o in outs], T)
    try:
        ws = [values((n_in, o), 10 + i, dtype, 0.02) for i, o in enumerate(outs)]
        for i, w in enumerate(ws):
            _pin(ctx, i, w, dtype, None if i % 2 == 0 else w.shape[1] + 24)
        x = values((T, n_in), 3, dtype, uneven=True)
        x[T // 2] = 0.0
        got = _product(ctx, list(range(len(outs))), outs, x, dtype)
        xd = serve.quantise_x(x)
        for i, w in enumerate(ws):
            _check(got[i], xd, serve.quantise_weight(w), dtype)
            assert np.all(got[i][T // 2] == 0)
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_weight_is_held_as_defined(dtype):
    print(f"\n[gpu case] base weight {dtype}", flush=True)
    n_in, n_out = 264, 392
    w = values((n_in, n_out), 5, dtype, 0.02)
    w[:128, 128:256] = 0.0                                   # a block of zeros
    w[128:, :128] *= 2.0 ** 60
    w[128:256, 256:384] *= 2.0 ** -110                       # codes below the smallest scale
    w = oracle.decode(store(w, dtype), dtype)
    ctx = _ctx(dtype, [(n_in, n_out)], 1)
    try:
        _pin(ctx, 0, w, dtype)
        sdt = np.float32 if dtype == "f32" else np.uint16
        out = to_dev(np.zeros((n_in, n_out + 8), sdt))
        ctx.read_base(0, out.ptr, n_out + 8)
        hipmod().synchronize()
        got = out.to_host()
        want = store(serve.quantise_weight(w), dtype)
        assert np.array_equal(oracle.decode(got[:, :n_out], dtype), oracle.decode(want, dtype))
        assert np.all(got[:, n_out:] == 0)
        out.free()
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("n_in,n_out,T", [(264, 392, 5), (640, 256, 70), (1032, 520, 300)])
def test_weights_that_come_quantised(n_in, n_out, T, dtype):
    """Codes and any fp32 scales, those of no power of two and of either sign of exponent included."""
    print(f"\n[gpu case] base fp8 weights {dtype} {n_in}->{n_out} T={T}", flush=True)
    rng = np.random.default_rng(4)
    codes = rng.integers(0, 256, (n_out, n_in + 8)).astype(np.uint8)
    codes[(codes & 127) == 127] = 0
    scales = np.exp(rng.uniform(-9, 2, (-(-n_out // 128), -(-n_in // 128)))).astype(np.float32)
    ctx = _ctx(dtype, [(n_in, n_out)], T)
    try:
        cd, sd = to_dev(codes), to_dev(scales)
        ctx.pin_base_fp8(0, cd.ptr, n_in + 8, sd.ptr)
        hipmod().synchronize()
        wd = serve.e4m3_value(codes[:, :n_in]).T * np.repeat(np.repeat(scales.astype(np.float64).T, 128, 0)[:n_in], 128, 1)[:, :n_out]
        x = values((T, n_in), 3, dtype, uneven=True)
        got = _product(ctx, [0], [n_out], x, dtype)[0]
        _check(got, serve.quantise_x(x), wd, dtype)
        cd.free()
        sd.free()
    finally:
        ctx.close()


@pytest.mark.parametrize("T", [3, 40, 300])
def test_values_that_are_not_finite(T):
    """NaN or infinity in a token's x: NaN in that token's y alone.  Huge and tiny tokens keep their precision."""
    print(f"\n[gpu case] base non-finite T={T}", flush=True)
    n_in, n_out = 392, 264
    w = values((n_in, n_out), 5, "bf16", 0.02)
    x = values((T, n_in), 3, "bf16")
    x[0] *= 2.0 ** 90
    x[T - 1] *= 2.0 ** -90
    x[1, 130] = np.nan
    if T > 20:
        x[20, 391] = np.inf
        x[17, 0] = -np.inf
    ctx = _ctx("bf16", [(n_in, n_out)], T)
    try:
        _pin(ctx, 0, w, "bf16")
        got = _product(ctx, [0], [n_out], x, "bf16")[0]
        bad = ~np.isfinite(x).all(1)
        assert np.isnan(got[bad]).all()
        _check(got[~bad], serve.quantise_x(x[~bad]), serve.quantise_weight(w), "bf16")
    finally:
        ctx.close()


def test_repeats_are_bit_identical_and_streams_are_ordered():
    """Products on two streams share the context's scratch: each result equals the one alone."""
    print("\n[gpu case] base streams", flush=True)
    hip = hipmod()
    n_in, n_out, T = 1024, 520, 190
    ctx = _ctx("bf16", [(n_in, n_out)], T)
    try:
        _pin(ctx, 0, values((n_in, n_out), 5, "bf16", 0.02), "bf16")
        xs = [store(values((T, n_in), 30 + i, "bf16"), "bf16") for i in range(4)]
        xd = [to_dev(x) for x in xs]
        yd = [to_dev(np.zeros((T, n_out), np.uint16)) for _ in range(8)]
        ss = [hip.Stream(), hip.Stream()]
        for i in range(4):
            ctx.base_product([0], T, xd[i].ptr, [yd[i].ptr], ss[0].h)
            ss[0].synchronize()
        for i in range(4):
            ctx.base_product([0], T, xd[i].ptr, [yd[4 + i].ptr], ss[i % 2].h)
        for s in ss:
            s.synchronize()
        for i in range(4):
            assert np.array_equal(yd[i].to_host(), yd[4 + i].to_host())
    finally:
        ctx.close()


def test_more_tables_than_a_launch_holds():
    print("\n[gpu case] base 20 tables", flush=True)
    outs = [8 * (1 + i) for i in range(20)]
    ctx = _ctx("bf16", [(136, o) for o in outs], 3)
    try:
        ws = [values((136, o), 50 + i, "bf16", 0.02) for i, o in enumerate(outs)]
        for i, w in enumerate(ws):
            _pin(ctx, i, w, "bf16")
        x = values((3, 136), 3, "bf16")
        for y, w in zip(_product(ctx, list(range(20)), outs, x, "bf16"), ws):
            _check(y, serve.quantise_x(x), serve.quantise_weight(w), "bf16")
    finally:
        ctx.close()


def test_refusals():
    print("\n[gpu case] base refusals", flush=True)
    from paper_2608_03579_amd import salt
    lib, C = salt.lib, salt.C
    ctx = _ctx("bf16", [(256, 264), (256, 8), (128, 8)], 16)
    buf = to_dev(np.zeros(256 * 272, np.uint16))
    y = to_dev(np.full(16 * 264, 9, np.uint16))
    try:
        assert lib.salt_pin_base(ctx.h, 3, buf.ptr, 264, None) == salt.ERR_OUT_OF_RANGE
        assert lib.salt_pin_base(ctx.h, -1, buf.ptr, 264, None) == salt.ERR_OUT_OF_RANGE
        assert lib.salt_pin_base(ctx.h, 0, None, 264, None) == salt.ERR_INVALID_ARG
        assert lib.salt_pin_base(ctx.h, 0, buf.ptr + 2, 264, None) == salt.ERR_INVALID_ARG
        assert lib.salt_pin_base(ctx.h, 0, buf.ptr, 256, None) == salt.ERR_INVALID_ARG
        assert lib.salt_pin_base(ctx.h, 0, buf.ptr, 268, None) == salt.ERR_INVALID_ARG
        assert lib.salt_pin_base_fp8(ctx.h, 0, buf.ptr, 256, None, None) == salt.ERR_INVALID_ARG
        assert lib.salt_pin_base_fp8(ctx.h, 0, buf.ptr, 248, buf.ptr, None) == salt.ERR_INVALID_ARG
        assert lib.salt_read_base(ctx.h, 0, buf.ptr, 264, None) == salt.ERR_BAD_STATE

        def call(tables, T, x, ys):
            n = len(tables)
            return lib.salt_base_product(ctx.h, n, (C.c_int32 * n)(*tables), T, x, (C.c_void_p * n)(*ys), None)

        assert call([0], 4, buf.ptr, [y.ptr]) == salt.ERR_BAD_STATE
        for t in range(3):
            ctx.pin_base(t, buf.ptr, 264)
        assert call([3], 4, buf.ptr, [y.ptr]) == salt.ERR_OUT_OF_RANGE
        assert call([0], 17, buf.ptr, [y.ptr]) == salt.ERR_OUT_OF_RANGE
        assert call([0], -1, buf.ptr, [y.ptr]) == salt.ERR_OUT_OF_RANGE
        assert call([0], 4, None, [y.ptr]) == salt.ERR_INVALID_ARG
        assert call([0], 4, buf.ptr + 8, [y.ptr]) == salt.ERR_INVALID_ARG
        assert call([0], 4, buf.ptr, [None]) == salt.ERR_INVALID_ARG
        assert call([0, 2], 4, buf.ptr, [y.ptr, y.ptr]) == salt.ERR_INVALID_ARG     # 256 and 128 inputs
        assert call([], 4, None, []) == salt.OK
        assert call([0], 0, None, [None]) == salt.OK
        hipmod().synchronize()
        assert np.all(y.to_host() == 9), "a refused call wrote y"
        assert call([0], 16, buf.ptr, [y.ptr]) == salt.OK
        hipmod().synchronize()
        assert np.all(y.to_host() == 0)
    finally:
        ctx.close()
