"""Host build of salt_decode.cpp (with tests/host_checks/decode_hip in place of the HIP runtime): refusals, what reaches
a launch, calls under capture, host memory that runs out.  And the oracle of its operators against direct forms."""
import os
import re
import shutil
import subprocess
import tempfile

import numpy as np
import pytest

from oracle import steps as o64
from paper_2608_03579_amd import build, salt
from tests.test_launch_walk import CSRC, HERE


@pytest.fixture(scope="module")
def decode_host(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("decode") / "decode_host")
    checks = os.path.join(HERE, "host_checks")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
           f"-I{os.path.join(checks, 'decode_hip')}", f"-I{os.path.join(os.path.dirname(HERE), 'include')}", f"-I{CSRC}",
           os.path.join(CSRC, "salt_serve.cpp"), os.path.join(CSRC, "salt_decode.cpp"),
           os.path.join(checks, "decode_host.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    return exe


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("check", ["refusals", "launches", "capture", "memory"])
def test_decode_host(decode_host, check):
    res = subprocess.run([decode_host, check], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr


def test_null_context_is_refused():
    lib, h = salt.lib, salt.C.c_void_p()
    bad = salt.ERR_INVALID_ARG
    assert lib.salt_rotate(None, None, 1, None, None, 0, None, 0, None, 0, None, 0, None) == bad
    assert lib.salt_kv_track(None, None) == bad
    assert lib.salt_kv_score(None, None, 0, None, 0, None, 1.0, 0, None) == bad
    assert lib.salt_kv_evict(None, None, 0, 1, 1, None) == bad
    assert lib.salt_kv_read_marks(None, None, 0, None, None, None) == bad
    assert lib.salt_kv_write_marks(None, None, 0, None, None, None) == bad
    assert lib.salt_beams_create(None, 1, 1, salt.C.byref(h)) == bad
    assert lib.salt_beam_select(None, None, 1, 1, 8, None, 0, None, 1, None, None, None, None) == bad
    assert lib.salt_kv_copy(None, None, 0, None, None, None, None) == bad
    lib.salt_beams_destroy(None, None)


def test_oracle_rotation_is_a_complex_product():
    rng = np.random.default_rng(0)
    x, freq, pos = rng.standard_normal((3, 2, 8)), np.array([1.0, 0.25, 1e-3]), np.array([0, 5, -70000])
    z = np.exp(1j * pos[:, None] * freq)[:, None]
    out, size = o64.rotate(x, pos, freq, True)
    want = (x[..., 0:6:2] + 1j * x[..., 1:6:2]) * z
    assert np.allclose(out[..., 0:6:2], want.real) and np.allclose(out[..., 1:6:2], want.imag)
    assert np.array_equal(out[..., 6:], x[..., 6:]) and np.allclose(size[..., 0:6:2], np.abs(want))
    half, _ = o64.rotate(np.concatenate([x[..., 0:6:2], x[..., 1:6:2], x[..., 6:]], -1), pos, freq, False)
    assert np.allclose(half[..., :3], want.real) and np.allclose(half[..., 3:6], want.imag)
    w = rng.standard_normal(8)
    v, _ = o64.rotate(x, np.zeros(3), freq, False, w, 0.0)
    assert np.allclose((v / w * np.sqrt((x * x).mean(-1, keepdims=True))), x)


def test_oracle_eviction_keeps_the_heaviest_and_the_newest():
    w, p = np.array([3.0, 1.0, 5.0, 4.0, 1.0, 9.0]), np.array([10, 11, 12, 13, 14, 9])
    assert o64.evict(w, p, 3, 0).tolist() == [3, 5, 2]             # kept: 2, 3 and 5; 3 and 5 move into the holes 0 and 1
    assert o64.evict(w, p, 3, 1).tolist() == [4, 5, 2]             # the newest (14) too
    assert o64.evict(w, p, 6, 2).tolist() == list(range(6))
    assert o64.evict(np.array([1.0, np.nan, 1.0, 1.0]), np.zeros(4), 2, 0).tolist() == [0, 1]


def test_oracle_selection_is_a_sort():
    rng = np.random.default_rng(1)
    x, s = np.round(rng.standard_normal((3, 40)), 1), np.array([0.0, 0.0, -np.inf])
    worth = o64.beam_worth(x, s)
    assert np.allclose(np.exp(worth).sum(-1), [1, 1, 0])
    v, b, t = o64.beam_select(worth, 85)
    assert np.all(b[80:] == -1) and np.all(np.diff(v[:80]) <= 0) and set(b[:80]) == {0, 1}
    same = np.flatnonzero(np.diff(v[:80]) == 0)
    assert len(same) and all((b[i], t[i]) < (b[i + 1], t[i + 1]) for i in same)


@pytest.mark.skipif(not os.path.exists(build.hipcc()), reason="hipcc not installed")
@pytest.mark.parametrize("source,least", [("salt_rotate.hip", 8), ("salt_marks.hip", 40), ("salt_beam.hip", 4)])
def test_no_kernel_uses_scratch_or_too_much_lds(source, least):
    with tempfile.TemporaryDirectory() as d:
        out = os.path.join(d, "k.s")
        flags = [f for f in build.HIPCC_FLAGS if f != "-fPIC"]
        res = subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, source), "-o",
                              out], capture_output=True, text=True)
        assert res.returncode == 0, res.stderr[-2000:]
        text = open(out).read()
    kernels = re.findall(r"\.name:\s+(\S+)\n(.*?)(?=\n  - \.|\Z)", text, re.S)
    kernels = [(n, b) for n, b in kernels if "private_segment_fixed_size" in b]
    assert len(kernels) >= least
    for name, body in kernels:
        assert int(re.search(r"\.private_segment_fixed_size:\s+(\d+)", body).group(1)) == 0, name
        assert int(re.search(r"\.vgpr_spill_count:\s+(\d+)", body).group(1)) == 0, name
    for lds in re.findall(r"\.group_segment_fixed_size:\s+(\d+)", text):
        assert int(lds) <= 160 * 1024
