"""The cases of tests/test_gpu_base_kernels.py take the kernels that they are meant for, and every kernel has one: asked
of the library's own rule (salt_base_rule.h), built for the host."""
import shutil
import subprocess

import pytest

from tests.test_gpu_base_kernels import CASES
from tests.test_launch_walk import CSRC, HERE

BOTH = {"few 1", "few 2", "tile 128x128", "split 64x64", "split 32x64", "split 32x32"}


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_cases_reach_every_kernel(tmp_path):
    exe = str(tmp_path / "base_rule")
    subprocess.run(["g++", "-std=c++17", "-O1", f"-I{CSRC}", f"{HERE}/host_checks/base_rule.cpp", "-o", exe], check=True,
                   capture_output=True, text=True)
    for dtype, n_in, outs, T, kernel in CASES:
        args = ["4" if dtype == "f32" else "2", str(T), *map(str, outs)]
        got = subprocess.run([exe, *args], check=True, capture_output=True, text=True).stdout.strip()
        assert got == kernel, (dtype, n_in, outs, T)
    reached = {(c[0], c[4]) for c in CASES}
    assert reached == {(d, k) for d in ("bf16", "f32") for k in BOTH} | {("bf16", "tile 256x256"), ("bf16", "tile 128x256")}
