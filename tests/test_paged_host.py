"""The paged cache's host unit (paged_api.cpp) built with the host compiler
under the address and undefined-behaviour sanitizers: 20,000 attention calls
of random shapes are divided soundly (no GPU, no HIP)."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_01790_amd", "csrc")

pytestmark = pytest.mark.skipif(shutil.which("g++") is None, reason="no host compiler")


def test_division_of_attention_calls(tmp_path):
    exe = str(tmp_path / "paged_driver")
    r = subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-fsanitize=address,undefined",
                        "-fno-sanitize-recover=all", f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                        os.path.join(ROOT, "tests", "host", "paged_driver.cpp"),
                        os.path.join(CSRC, "paged_api.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert "calls checked" in r.stdout
