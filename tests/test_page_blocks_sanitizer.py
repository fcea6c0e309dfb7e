"""Gather blocks cut into pages, with sources at the ends of 32 bits, under UndefinedBehaviorSanitizer (CPU)."""
import os
import subprocess

import pytest

from test_host_sanitizers import CLANG, ROOT, SAN, _run

CSRC = os.path.join(ROOT, "paper_2607_28069_amd", "csrc")
SOURCES = [os.path.join(CSRC, f) for f in ("pic_api.cpp", "pic_pages.cpp", "pic_plan.cpp")] + [
    os.path.join(ROOT, "tests", "sanitize", f) for f in ("emulated_launchers.cpp", "page_launchers.cpp", "blocks_driver.cpp")]


def test_blocks_of_any_source(tmp_path):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ in this image")
    exe = str(tmp_path / "blocks_driver")
    r = subprocess.run([CLANG, "-std=c++17", "-O1", "-g", *SAN, "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                        f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", *SOURCES, "-o", exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    r = _run(exe)
    assert r.returncode == 0 and "blocks driver: OK" in r.stdout, (r.stdout + r.stderr)[-3000:]
