"""Host build of the entry points around the apply (salt_serve.cpp, with tests/host_checks/serve_hip in place of the HIP
runtime): a first pin under capture, and host memory that runs out."""
import os
import shutil
import subprocess

import pytest

from tests.test_launch_walk import CSRC, HERE

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")


@pytest.fixture(scope="module")
def serve_host(tmp_path_factory):
    exe = str(tmp_path_factory.mktemp("serve") / "serve_host")
    checks = os.path.join(HERE, "host_checks")
    include = os.path.join(os.path.dirname(HERE), "include")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
           f"-I{os.path.join(checks, 'serve_hip')}", f"-I{include}", f"-I{CSRC}", os.path.join(CSRC, "salt_serve.cpp"),
           os.path.join(checks, "serve_host.cpp"), "-o", exe]
    res = subprocess.run(cmd, capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-3000:]
    return exe


@pytest.mark.parametrize("check", ["capture", "memory"])
def test_serve_host(serve_host, check):
    res = subprocess.run([serve_host, check], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr
