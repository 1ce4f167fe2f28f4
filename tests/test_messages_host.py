"""Host build of the runtime (tests/host_checks/messages.cpp): a failing call keeps its message and answers, also where
host memory is out."""
import os
import subprocess

import pytest

from tests import cpu_build
from tests.test_launch_walk import CSRC, HERE


@pytest.mark.skipif(not cpu_build.available(), reason="needs the ROCm host clang")
def test_messages_need_no_memory(tmp_path):
    exe = str(tmp_path / "messages")
    include = [f"-I{os.path.join(HERE, 'cpu_kernels')}", f"-I{os.path.join(os.path.dirname(HERE), 'include')}", f"-I{CSRC}"]
    cmd = [cpu_build.CLANG, "-std=c++17", "-O1", "-g", "-w", *include, os.path.join(CSRC, "salt_runtime.cpp"),
           os.path.join(HERE, "host_checks", "messages.cpp"), "-Wl,--unresolved-symbols=ignore-all", "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr
