"""Calls of several host threads on one stream with one workspace: what a call's first kernel leaves there for its second must not be
overwritten by another call's kernel in between (tests/native/stream_turns.cpp: the built library with launches that only take notes)."""
import os
import shutil
import subprocess

import pytest

from paper_2509_01229_amd import api

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="needs g++")
def test_the_launches_of_a_call_stand_together(tmp_path):
    api.lib()
    exe = str(tmp_path / "stream_turns")
    package = os.path.join(ROOT, "paper_2509_01229_amd")
    subprocess.run(["g++", "-std=c++17", "-O1", "-Wall", "-D__HIP_PLATFORM_AMD__", "-I", os.path.join(ROOT, "include"), "-isystem", "/opt/rocm/include",
                    "-rdynamic", os.path.join(ROOT, "tests", "native", "stream_turns.cpp"), "-o", exe, "-L", package, "-l:libliquidgemm.so",
                    "-L/opt/rocm/lib", "-lamdhip64", f"-Wl,-rpath,{package}:/opt/rocm/lib", "-lpthread"], check=True)
    res = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert res.returncode == 0, res.stdout + res.stderr
    assert "stream_turns ok" in res.stdout
