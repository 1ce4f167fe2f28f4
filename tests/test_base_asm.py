"""The copies to LDS in salt_base.hip are written in assembly and set m0.  The compiler keeps that register for itself: it
must not be named as overwritten (the compiler warns, and promises nothing), and every block must put it back."""
import os
import re
import subprocess

import pytest

from paper_2608_03579_amd import build


@pytest.mark.skipif(not os.path.exists(build.hipcc()), reason="hipcc not installed")
def test_copies_to_lds_put_m0_back(tmp_path):
    out = str(tmp_path / "base.s")
    flags = [f for f in build.HIPCC_FLAGS if f != "-fPIC"]
    res = subprocess.run([build.hipcc(), *flags, "--cuda-device-only", "-S", os.path.join(build.CSRC, "salt_base.hip"), "-o",
                          out], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    assert "reserved registers" not in res.stderr
    blocks = [b for b in re.findall(r";;#ASMSTART\n(.*?);;#ASMEND", open(out).read(), re.S) if re.search(r"\bm0\b", b)]
    assert len(blocks) >= 20
    for b in blocks:
        lines = [l.strip() for l in b.strip().splitlines()]
        keep = re.fullmatch(r"s_mov_b32 (s\d+), m0", lines[0])
        assert keep and lines[-1] == f"s_mov_b32 m0, {keep.group(1)}", b
        assert not any(re.match(rf"s_\w+ {keep.group(1)}\b", l) for l in lines[1:-1]), b
