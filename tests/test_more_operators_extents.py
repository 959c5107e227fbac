"""Layer norm, dropout and the adapters from nothing to their largest extents: grids of less than 2^32 threads, workspaces that hold what goes
into them.  Host side with stub launchers, under AddressSanitizer + UndefinedBehaviorSanitizer; no GPU is involved."""
import os
import shutil
import subprocess

import pytest

from test_sanitizers import ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_launches_of_all_extents(tmp_path):
    exe = str(tmp_path / "more_san")
    csrc = os.path.join(ROOT, "paper_2511_12653_amd", "csrc")
    subprocess.run(["g++", "-std=c++17", *SAN, "-Wall", "-Wextra", *(os.path.join(csrc, "fq_%s_api.cpp" % n) for n in ("norm", "dropout", "adapters")),
                    os.path.join(ROOT, "tests", "sanitize", "more_operators_driver.cpp"), "-o", exe], check=True)
    assert "more operators: 0 failures" in _run(exe)
