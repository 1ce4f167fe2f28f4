"""Host build of the attention's cut of a batch (tests/host_checks/seqs_joined.cpp): rows that are joined have keys."""
import os
import shutil
import subprocess

import pytest

from tests.test_launch_walk import CSRC, HERE


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_joined_rows_have_keys(tmp_path):
    exe = str(tmp_path / "seqs_joined")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           f"-I{CSRC}", os.path.join(HERE, "host_checks", "seqs_joined.cpp"), "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr
