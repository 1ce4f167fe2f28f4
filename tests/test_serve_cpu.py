"""CPU-side checks of the base product, the KV cache and the attention: the oracle against torch's own
conversions and a direct softmax, sizes, and refusals that come before any GPU call.  The kernels
of the new sources use no scratch memory (as tests/test_kernel_resources.py checks for the others)."""
import os
import re
import subprocess
import tempfile

import numpy as np
import pytest

from oracle import serve
from paper_2608_03579_amd import build, salt


def test_oracle_rounds_to_e4m3_as_defined():
    codes = np.arange(256)
    v = serve.e4m3_value(codes)
    fin = v[np.isfinite(v)]
    assert np.isnan(v[[0x7f, 0xff]]).all() and len(fin) == 254 and fin.max() == 448.0
    assert np.array_equal(serve.round_e4m3(fin), fin)                       # values are their own codes
    u = np.unique(fin)
    mid = (u[1:] + u[:-1]) / 2                                              # ties: the even neighbour
    even = {float(serve.e4m3_value(c)) for c in codes if (c & 1) == 0 and (c & 127) != 127}
    assert all(float(x) in even or x == 0 for x in serve.round_e4m3(mid))
    torch = pytest.importorskip("torch")
    x = (torch.randn(20000, dtype=torch.float64) * torch.exp(torch.randn(20000) * 4)).clamp(-448, 448).float()
    assert np.array_equal(x.to(torch.float8_e4m3fn).double().numpy(), serve.round_e4m3(x.double().numpy()))


def test_oracle_cache_error_bounds():
    """e4m3 keeps 2^-4 of a value that is not tiny in its vector, int8 half a step of amax / 127."""
    x = np.random.default_rng(0).standard_normal((200, 64)) * np.exp(np.random.default_rng(1).uniform(-20, 20, (200, 1)))
    amax = np.abs(x).max(-1, keepdims=True)
    e = np.abs(serve.quantise_kv(x, "e4m3") - x)
    assert np.all(e <= np.maximum(2.0 ** -4 * np.abs(x), amax * 2.0 ** -17))
    assert np.all(np.abs(serve.quantise_kv(x, "int8") - x) <= amax / 127 * 0.5001)
    x[3, 5] = np.nan
    x[4, 6] = np.inf
    for fmt in ("e4m3", "int8"):
        q = serve.quantise_kv(x, fmt)
        assert np.isnan(q[3:5]).all() and np.isfinite(np.delete(q, [3, 4], 0)).all()


def test_oracle_attention_is_a_weighted_mean():
    rng = np.random.default_rng(2)
    q, k, v = rng.standard_normal(64), rng.standard_normal((9, 64)), rng.standard_normal((9, 64))
    out, mass, _ = serve.attend(q, k, v, 0.125)
    w = np.exp(0.125 * k @ q)
    assert np.allclose(out, (w[:, None] * v).sum(0) / w.sum()) and np.all(mass >= np.abs(out) - 1e-12)
    assert np.allclose(serve.attend(q, k[:1], v[:1], 0.125)[0], v[0])
    assert np.all(serve.attend(q, k[:0], v[:0], 0.125)[0] == 0)


def test_cache_bytes():
    cfg = salt.KvConfig(28, 24, 8, 128, 64, 100, salt.KV_E4M3, 0)
    assert salt.lib.salt_kv_bytes(salt.C.byref(cfg)) == 28 * 2 * 100 * 64 * 8 * (128 + 4)
    assert salt.lib.salt_kv_bytes(None) == 0
    for bad in (dict(head_dim=32), dict(page_tokens=48), dict(n_heads=23), dict(format=-1), dict(n_pages=-1)):
        kw = dict(n_layers=1, n_heads=24, n_kv_heads=8, head_dim=128, page_tokens=64, n_pages=1, format=0, flags=0)
        assert salt.lib.salt_kv_bytes(salt.C.byref(salt.KvConfig(**{**kw, **bad}))) == 0, bad


def test_null_context_is_refused():
    lib, P = salt.lib, salt.C.c_void_p
    h = P()
    cfg = salt.KvConfig(1, 1, 1, 64, 16, 1, 0, 0)
    assert lib.salt_pin_base(None, 0, None, 8, None) == salt.ERR_INVALID_ARG
    assert lib.salt_pin_base_fp8(None, 0, None, 8, None, None) == salt.ERR_INVALID_ARG
    assert lib.salt_read_base(None, 0, None, 8, None) == salt.ERR_INVALID_ARG
    assert lib.salt_base_product(None, 0, None, 0, None, None, None) == salt.ERR_INVALID_ARG
    assert lib.salt_kv_create(None, salt.C.byref(cfg), salt.C.byref(h)) == salt.ERR_INVALID_ARG
    assert lib.salt_seqs_create(None, None, 1, 1, 1, salt.C.byref(h)) == salt.ERR_INVALID_ARG
    assert lib.salt_seqs_set(None, None, None, None) == salt.ERR_INVALID_ARG
    assert lib.salt_kv_write(None, None, 0, None, 0, None, 0, None) == salt.ERR_INVALID_ARG
    assert lib.salt_kv_read(None, None, 0, 0, None, 0, None, 0, None) == salt.ERR_INVALID_ARG
    assert lib.salt_attend(None, None, 0, None, 0, None, 0, 1.0, None) == salt.ERR_INVALID_ARG
    lib.salt_kv_destroy(None, None)
    lib.salt_seqs_destroy(None, None)


@pytest.mark.skipif(not os.path.exists(build.hipcc()), reason="hipcc not installed")
@pytest.mark.parametrize("source", ["salt_base.hip", "salt_kv.hip", "salt_attend.hip"])
def test_no_kernel_uses_scratch_or_too_much_lds(source):
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "k.s")
        flags = [f for f in build.HIPCC_FLAGS if f != "-fPIC"]
        res = subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o",
                              out], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-2000:]
        text = open(out).read()
    kernels = re.findall(r"\.name:\s+(\S+)\n(.*?)(?=\n  - \.|\Z)", text, re.S)
    kernels = [(n, b) for n, b in kernels if "private_segment_fixed_size" in b]
    assert len(kernels) >= 10
    for name, body in kernels:
        assert int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", body).group(1)) == 0, name
        assert int(re.search(r"\.vgpr_spill_count:\s+(\d+)", body).group(1)) == 0, name
    for lds in re.findall(r"\.group_segment_fixed_size:\s+(\d+)", text):
        assert int(lds) <= 160 * 1024
