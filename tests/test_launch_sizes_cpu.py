"""Calls of millions of tokens: every launch holds fewer than 2^32 threads, and together they have a block for each piece of work
(tests/native/launch_sizes.cpp: the built library with launches that are only counted)."""
import os
import shutil
import subprocess

import pytest

from paper_2509_01229_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_launches_of_many_tokens(tmp_path):
    api.lib()
    exe = str(tmp_path / "launch_sizes")
    package = os.path.join(ROOT, "paper_2509_01229_amd")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-isystem", "/opt/rocm/include",
                    "-rdynamic", os.path.join(ROOT, "tests", "native", "launch_sizes.cpp"), "-o", exe, "-L", package, "-l:libliquidgemm.so",
                    "-L/opt/rocm/lib", "-lamdhip64", f"-Wl,-rpath,{package}:/opt/rocm/lib", "-lpthread"], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
    assert "launch_sizes ok" in res.stdout
