"""AddressSanitizer + UndefinedBehaviorSanitizer build of the host side of the int8 linear layer and the AdamW step, with stub
launchers that check the layout of the workspace and of the table.  No GPU is involved."""
import os
import shutil
import subprocess

import pytest

from test_sanitizers import ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_operators_host_side_under_asan_and_ubsan(tmp_path):
    exe = str(tmp_path / "operators_san")
    csrc = os.path.join(ROOT, "paper_2511_12653_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", *SAN, "-Wall", "-Wextra", os.path.join(csrc, "fq_linear_api.cpp"),
                    os.path.join(csrc, "fq_adamw_api.cpp"), os.path.join(ROOT, "tests", "sanitize", "operators_driver.cpp"), "-o", exe], check=True)
    assert "0 failures" in _run(exe)
