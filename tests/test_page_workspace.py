"""Calls over pages write no more of a workspace than the query call names, and nothing of a misaligned one, on the CPU
(tests/sanitize/workspace_driver.cpp, launches emulated by tests/sanitize/page_launchers.cpp)."""
import os
import re
import subprocess

import pytest

from test_host_sanitizers import CLANG, ROOT, SAN, _run

CSRC = os.path.join(ROOT, "paper_2607_28069_amd", "csrc")
SOURCES = [os.path.join(CSRC, f) for f in ("pic_api.cpp", "pic_pages.cpp", "pic_plan.cpp")] + [
    os.path.join(ROOT, "tests", "sanitize", f) for f in ("emulated_launchers.cpp", "page_launchers.cpp", "workspace_driver.cpp")]


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ in this image")
    exe = str(tmp_path_factory.mktemp("workspace") / "workspace_driver")
    r = subprocess.run([CLANG, "-std=c++17", "-O1", "-g", *SAN, "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include",
                        f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}", *SOURCES, "-o", exe], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]
    return exe


@pytest.mark.parametrize("seed", ["1", "2", "3", "4"])
def test_no_more_is_written_than_the_query_names(driver, seed):
    r = _run(driver, seed)
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert int(re.search(r"OK, (\d+) calls", r.stdout).group(1)) >= 5
