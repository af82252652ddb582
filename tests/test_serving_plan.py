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


HIPCC = os.environ.get("HIPCC", "/opt/rocm/bin/hipcc")


@pytest.mark.skipif(os.path.exists("/dev/kfd"), reason="fake-pointer cases run only without a GPU")
@pytest.mark.skipif(not os.path.exists(HIPCC), reason="hipcc not found")
def test_host_code_under_asan_ubsan(tmp_path):
    # host parts instrumented (every sanitizer flag behind -Xarch_host); the
    # device parts are compiled as usual and never run
    flags = ["--offload-arch=gfx950", "-O1", "-g", "-std=c++17", "-fPIC", "-Xarch_host", "-fsanitize=address",
             "-Xarch_host", "-fsanitize=undefined", "-Xarch_host", "-fno-sanitize-recover=all",
             "-Xclang", "-target-feature", "-Xclang", "-packed-fp32-ops", "-I", os.path.join(ROOT, "include")]
    here, csrc = os.path.join(ROOT, "tests", "sanitize"), os.path.join(ROOT, "paper_2504_17577_amd", "csrc")
    objs = [str(tmp_path / f"{n}.o") for n in ("paged", "gemm_epilogue")]
    procs = [subprocess.Popen([HIPCC, *flags, "-c", os.path.join(csrc, f"{n}.hip"), "-o", o], stdout=subprocess.PIPE,
                              stderr=subprocess.PIPE, text=True) for n, o in zip(("paged", "gemm_epilogue"), objs)]
    for p in procs:
        _, err = p.communicate(timeout=900)
        assert p.returncode == 0, err[-4000:]
    drv, exe = str(tmp_path / "driver.o"), str(tmp_path / "driver")
    for cmd in (["gcc", "-std=c11", "-g", "-O1", "-Wall", "-Werror", "-fsanitize=address,undefined",
                 "-fno-sanitize-recover=all", "-I", os.path.join(ROOT, "include"), "-c",
                 os.path.join(here, "serving_driver.c"), "-o", drv],
                [HIPCC, "-Xarch_host", "-fsanitize=address", "-Xarch_host", "-fsanitize=undefined", "-o", exe, drv, *objs]):
        r = subprocess.run(cmd, capture_output=True, text=True)
        assert r.returncode == 0, r.stderr[-4000:]
    env = dict(os.environ, ASAN_OPTIONS="detect_leaks=0:abort_on_error=1", UBSAN_OPTIONS="print_stacktrace=1:halt_on_error=1")
    r = subprocess.run([exe], capture_output=True, text=True, env=env, timeout=300)
    assert r.returncode == 0 and "all checks passed" in r.stdout, r.stdout + r.stderr[-4000:]
