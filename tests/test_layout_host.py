"""The layout's entry points where host memory runs out
(tests/native/layout_check.cpp fails their allocations one by one)."""
import os
import shutil
import subprocess

import pytest

from paper_2609_28568_amd import binding

HERE = os.path.dirname(os.path.abspath(__file__))
CSRC = os.path.join(os.path.dirname(HERE), "paper_2609_28568_amd", "csrc")
ROCM = os.environ.get("ROCM_PATH", "/opt/rocm")


def test_failed_allocations_are_reported(tmp_path):
    cxx = shutil.which("g++")
    if not cxx:
        pytest.skip("no g++")
    exe = str(tmp_path / "layout_check")
    subprocess.run([cxx, "-std=c++17", "-O1", "-w", "-D__HIP_PLATFORM_AMD__", f"-I{ROCM}/include",
                    os.path.join(HERE, "native", "layout_check.cpp"), os.path.join(CSRC, "prefix.cpp"),
                    binding.LIB_PATH, f"-L{ROCM}/lib", "-lamdhip64",
                    f"-Wl,-rpath,{os.path.dirname(binding.LIB_PATH)}", f"-Wl,-rpath,{ROCM}/lib", "-o", exe], check=True)
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout + r.stderr
