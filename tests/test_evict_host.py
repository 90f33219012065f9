"""The host units of reading, accumulated weights and eviction (evict_api.cpp with
paged_api.cpp) built with the host compiler under the address and
undefined-behaviour sanitizers: 20,000 random calls are divided soundly and hand
their launches what they should (no GPU, no HIP)."""

import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_01790_amd", "csrc")
CLANG = "/opt/rocm/llvm/bin/clang++"
FLAGS = {"g++": ["-fsanitize=address,undefined", "-fno-sanitize-recover=all"],
         CLANG: ["-ftrivial-auto-var-init=pattern"]}


@pytest.mark.parametrize("compiler", list(FLAGS))
def test_division_of_calls(tmp_path, compiler):
    if shutil.which(compiler) is None:
        pytest.skip(f"no {compiler}")
    exe = str(tmp_path / "evict_driver")
    r = subprocess.run([compiler, "-std=c++17", "-g", "-O1", *FLAGS[compiler],
                        f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                        os.path.join(ROOT, "tests", "host", "evict_driver.cpp"),
                        os.path.join(CSRC, "paged_api.cpp"), os.path.join(CSRC, "evict_api.cpp"), "-o", exe],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=120)
    assert r.returncode == 0, r.stdout[-2000:] + r.stderr[-2000:]
    assert "calls checked" in r.stdout
