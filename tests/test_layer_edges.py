"""Host side of libsk_layer.so at the ends of its ranges, no GPU."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
SAN = ["-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-static-libasan", "-g", "-O1"]
ENV = dict(os.environ, ASAN_OPTIONS="verify_asan_link_order=0:detect_leaks=1", UBSAN_OPTIONS="print_stacktrace=1")


@pytest.mark.skipif(shutil.which("g++") is None, reason="no host C++ compiler")
def test_plans_at_the_ends_of_their_ranges(tmp_path):
    exe, csrc = str(tmp_path / "layer_edges_driver"), os.path.join(ROOT, "paper_1901_10008_amd", "csrc")
    res = subprocess.run(["g++", "-std=c++17", *SAN, "-I", os.path.join(ROOT, "include"), "-I", csrc, os.path.join(ROOT, "tests", "sanitize", "layer_edges_driver.cpp"),
                          os.path.join(csrc, "layer_plan.cpp"), "-o", exe], capture_output=True, text=True)
    assert res.returncode == 0, res.stderr
    res = subprocess.run([exe], capture_output=True, text=True, env=ENV)
    assert res.returncode == 0 and "layer_edges_driver: ok" in res.stdout, res.stdout + res.stderr
