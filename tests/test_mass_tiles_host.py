"""The tiles of added weights: host and kernels share one rule (evict.h), and the
launch refuses a division that no kernel is made for (the built library, no GPU)."""

import os
import subprocess

import pytest

from paper_2606_01790_amd import starkv as sk

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CSRC = os.path.join(ROOT, "paper_2606_01790_amd", "csrc")

pytestmark = pytest.mark.skipif(not os.path.exists(sk.LIB_PATH),
                                reason="libstarkv.so not built")


def test_divisions_without_a_kernel_are_refused(tmp_path):
    exe = str(tmp_path / "mass_tiles_driver")
    r = subprocess.run(["g++", "-std=c++17", "-O1", f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}",
                        os.path.join(ROOT, "tests", "host", "mass_tiles_driver.cpp"), sk.LIB_PATH,
                        f"-Wl,-rpath,{os.path.dirname(sk.LIB_PATH)}", "-Wl,-rpath,/opt/rocm/lib",
                        "-Wl,--allow-shlib-undefined", "-o", exe], capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=60)
    assert r.returncode == 0 and "refused" in r.stdout, r.stdout + r.stderr
