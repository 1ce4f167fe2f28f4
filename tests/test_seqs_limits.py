"""Host build of a batch's arithmetic at its limits (tests/host_checks/seqs_limits.cpp): pages past a sequence's last
token, and launches of 2^32 threads."""
import os
import shutil
import subprocess

import pytest

from tests.test_launch_walk import CSRC, HERE


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_limits_of_a_batch(tmp_path):
    exe = str(tmp_path / "seqs_limits")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=undefined", "-fno-sanitize-recover=undefined",
           f"-I{CSRC}", os.path.join(HERE, "host_checks", "seqs_limits.cpp"), "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr
