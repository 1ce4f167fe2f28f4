"""Base weights that hold values which are not finite (salt_pin_base, salt_read_base, salt_base_product): an infinity
or a NaN in W takes its whole block of 128 x 128, so that y is NaN at the block's outputs, and nothing else."""
import numpy as np
import pytest

import oracle
from oracle import serve
from tests.serve_harness import hipmod, store, to_dev, values
from tests.test_gpu_base import _check, _ctx, _pin, _product

pytestmark = pytest.mark.gpu

N_IN, N_OUT = 392, 520
BAD = {(5, 7): np.nan, (130, 300): np.inf, (391, 519): -np.inf, (260, 129): np.nan}      # (input, output): value


def _weight(dtype):
    w = values((N_IN, N_OUT), 5, dtype, 0.02)
    held = serve.quantise_weight(w)
    for (k, o), v in BAD.items():
        w[k, o] = v
        held[k // 128 * 128: k // 128 * 128 + 128, o // 128 * 128: o // 128 * 128 + 128] = np.nan
    return w, held


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
def test_blocks_read_back(dtype):
    print(f"\n[gpu case] base weight not finite, read {dtype}", flush=True)
    w, held = _weight(dtype)
    ctx = _ctx(dtype, [(N_IN, N_OUT)], 1)
    try:
        _pin(ctx, 0, w, dtype)
        out = to_dev(np.zeros((N_IN, N_OUT), np.float32 if dtype == "f32" else np.uint16))
        ctx.read_base(0, out.ptr, N_OUT)
        hipmod().synchronize()
        got = oracle.decode(out.to_host(), dtype)
        assert np.array_equal(got, oracle.decode(store(held, dtype), dtype), equal_nan=True)
        out.free()
    finally:
        ctx.close()


@pytest.mark.parametrize("dtype", ["bf16", "f32"])
@pytest.mark.parametrize("T", [1, 12, 40, 300])
def test_outputs_of_the_blocks(T, dtype):
    """x = 0 among the tokens: NaN there, too."""
    print(f"\n[gpu case] base weight not finite, T={T} {dtype}", flush=True)
    w, held = _weight(dtype)
    x = values((T, N_IN), 3, dtype)
    x[T // 2] = 0.0
    ctx = _ctx(dtype, [(N_IN, N_OUT)], T)
    try:
        _pin(ctx, 0, w, dtype)
        got = _product(ctx, [0], [N_OUT], x, dtype)[0]
        bad = np.isnan(held).any(0)
        assert bad.sum() == 128 + 128 + 128 + 8 and np.isnan(got[:, bad]).all()
        _check(got[:, ~bad], serve.quantise_x(x), held[:, ~bad], dtype)
    finally:
        ctx.close()
