"""Host build of the attention's cut of a batch into work items (tests/host_checks/seqs_cut.cpp, g++ with
AddressSanitizer and UBSan): every row meets each of its keys once, and its partial results their join."""
import os
import shutil
import subprocess

import pytest

from tests.test_launch_walk import CSRC, HERE


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_every_row_meets_its_keys_once(tmp_path):
    exe = str(tmp_path / "seqs_cut")
    cmd = ["g++", "-std=c++17", "-O1", "-g", "-fsanitize=address,undefined", "-fno-sanitize-recover=undefined",
           f"-I{CSRC}", os.path.join(HERE, "host_checks", "seqs_cut.cpp"), "-o", exe]
    subprocess.run(cmd, check=True, capture_output=True, text=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=600)
    assert res.returncode == 0 and res.stdout.strip().endswith("ok"), res.stdout + res.stderr
