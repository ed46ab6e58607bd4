"""Products of few rows pass x between the lanes of a wavefront through LDS.  Nothing but a meeting of the lanes keeps the compiler from moving one lane's
reads before another's writes: each batch that is put there has one behind it, and one behind its use (no GPU needed)."""
import os
import re
import shutil
import subprocess

import pytest


@pytest.mark.skipif(shutil.which("hipcc") is None, reason="needs hipcc")
def test_a_meeting_on_either_side_of_every_exchange(tmp_path):
    from paper_2009_13003_amd import build
    flags = [f for f in build.FLAGS if f != "-shared"]
    res = subprocess.run(["hipcc"] + flags + ["--cuda-device-only", "-S", "-o", str(tmp_path / "out.s"), os.path.join(build.CSRC, "lc_w4.hip")],
                         capture_output=True, text=True)
    assert res.returncode == 0, res.stderr[-2000:]
    kernels = 0
    for body in re.split(r"\n(?=_ZN\S*:)", (tmp_path / "out.s").read_text()):
        if "9k_w4_rows" not in body.split(":", 1)[0]:
            continue
        kernels += 1
        assert body.count("; wave barrier") >= 4             # two batches a turn, written out
    assert kernels >= 18
