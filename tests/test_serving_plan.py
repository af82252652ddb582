"""The paged cache's integer logic on the CPU, under the sanitizers: the division of
a batch over workgroups and the bounds of lengths and pages."""
import os
import shutil
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.mark.skipif(shutil.which("g++") is None, reason="g++ not found")
def test_parts_cover_the_batch(tmp_path):
    exe = str(tmp_path / "paged_driver")
    r = subprocess.run(["g++", "-std=c++17", "-g", "-O1", "-Wall", "-Wextra", "-Werror",
                        "-fsanitize=address,undefined", "-fno-sanitize-recover=all", "-I",
                        os.path.join(ROOT, "paper_2504_17577_amd", "csrc"), "-o", exe,
                        os.path.join(ROOT, "tests", "sanitize", "paged_driver.cpp")],
                       capture_output=True, text=True)
    assert r.returncode == 0, r.stderr
    r = subprocess.run([exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "all checks passed" in r.stdout, r.stdout + r.stderr[-4000:]
