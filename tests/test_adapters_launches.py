"""What the adapters' kernels are launched with: LDS for what each of them keeps there, grids and forms that fit the call.  The launcher is the library's own,
compiled for the host alone, with a runtime that only looks; no GPU is involved."""
import os
import shutil
import subprocess

import pytest

from paper_2511_12653_amd import build
from test_sanitizers import ROOT, SAN, _run


@pytest.mark.skipif(shutil.which("g++") is None or shutil.which(build.HIPCC) is None, reason="needs hipcc and g++")
def test_each_kernel_gets_the_lds_that_it_uses(tmp_path):
    csrc = os.path.join(ROOT, "paper_2511_12653_amd", "csrc")
    launcher, exe = str(tmp_path / "launcher.o"), str(tmp_path / "launches")
    subprocess.run([build.HIPCC, "--offload-arch=gfx950", "--cuda-host-only", "-O1", "-std=c++17", "-fPIC", "-c", os.path.join(csrc, "fq_adapters.hip"), "-o", launcher], check=True)
    # (the device code, which the object names, is not there; nothing looks at it)
    subprocess.run(["g++", "-std=c++17", *SAN, "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", "-Wall", "-Wextra", "-Wno-unused-parameter",
                    os.path.join(csrc, "fq_adapters_api.cpp"), os.path.join(ROOT, "tests", "sanitize", "adapters_launch_driver.cpp"), launcher,
                    "-Wl,--unresolved-symbols=ignore-in-object-files", "-o", exe], check=True)
    assert "adapters: 0 failures" in _run(exe)
