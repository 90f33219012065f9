"""The lists that the paged calls hand to their launches hold no value that
nobody has set: the host unit with locals that start as a pattern (no GPU)."""

import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_01790_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"

pytestmark = pytest.mark.skipif(not os.path.exists(CLANG), reason="no clang++")


def test_lists_hold_defined_values(tmp_path):
    exe = str(tmp_path / "lists")
    r = subprocess.run([CLANG, "-std=c++17", "-g", "-O1", "-ftrivial-auto-var-init=pattern",
                        f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                        os.path.join(ROOT, "tests", "host", "paged_lists_driver.cpp"),
                        os.path.join(CSRC, "paged_api.cpp"), "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert "8 lists checked" in r.stdout
