"""Host build of the calls on a tracked cache (tests/host_checks/marks_host.cpp, with tests/host_checks/decode_hip in place
of the HIP runtime): what reaches a launch, and what is refused."""
import os
import shutil
import subprocess

import pytest

from tests.test_launch_walk import CSRC, HERE


@pytest.fixture(scope="module")
def marks_host(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("marks") / "marks_host")
    checks = os.path.join(HERE, "host_checks")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           f"-I{os.path.join(checks, 'decode_hip')}", f"-I{os.path.join(os.path.dirname(HERE), 'include')}", f"-I{CSRC}",
           os.path.join(CSRC, "salt_serve.cpp"), os.path.join(CSRC, "salt_decode.cpp"),
           os.path.join(checks, "marks_host.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    return exe


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
@pytest.mark.parametrize("check", ["written", "shared", "range"])
def test_marks_host(marks_host, check):
    res = subprocess.run([marks_host, check], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr
