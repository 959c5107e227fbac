"""The int8 linear layer at the largest extents it takes: every launch's grid has less than 2^32 threads, and the parts of a
call are the whole of it.  Host side with stub launchers, under AddressSanitizer + UndefinedBehaviorSanitizer; no GPU is involved."""
import os
import shutil
import subprocess

import pytest

from test_sanitizers import ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_launches_of_the_largest_extents(tmp_path):
    exe = str(tmp_path / "extents_san")
    subprocess.run(["g++", "-std=c++17", *SAN, "-Wall", "-Wextra", os.path.join(ROOT, "paper_2511_12653_amd", "csrc", "fq_linear_api.cpp"),
                    os.path.join(ROOT, "tests", "sanitize", "extents_driver.cpp"), "-o", exe], check=True)
    assert "extents: 0 failures" in _run(exe)
