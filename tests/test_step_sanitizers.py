"""Shared prefixes, page tables grown on the device and norms with rotation under AddressSanitizer and
UndefinedBehaviorSanitizer (CPU, no GPU): every launching call with garbage tables, starts, lengths and counts over
buffers of the exact documented sizes, the launches emulated (tests/sanitize/step_launchers.cpp).  A planted mistake (a
page buffer one row short) must be caught."""
import os
import subprocess

import pytest

from test_host_sanitizers import CLANG, ROOT, SAN, _run

CSRC = os.path.join(ROOT, "paper_2607_28069_amd", "csrc")
SOURCES = [os.path.join(CSRC, f) for f in ("pic_api.cpp", "pic_pages.cpp", "pic_plan.cpp", "pic_shared.cpp", "pic_grow.cpp",
                                           "pic_tokens.cpp")] + [
    os.path.join(ROOT, "tests", "sanitize", f) for f in ("emulated_launchers.cpp", "page_launchers.cpp", "step_launchers.cpp",
                                                         "step_driver.cpp")]


@pytest.fixture(scope="module")
def driver(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ in this image")
    out = tmp_path_factory.mktemp("step_san")
    flags = ["-std=c++17", "-O1", "-g", "-fno-omit-frame-pointer", *SAN, "-fno-sanitize-recover=all", "-D__HIP_PLATFORM_AMD__",
             "-I/opt/rocm/include", f"-I{os.path.join(ROOT, 'include')}", f"-I{CSRC}"]
    objs = []
    for src in SOURCES:
        obj = str(out / (os.path.basename(src) + ".o"))
        r = subprocess.run([CLANG, *flags, "-c", src, "-o", obj], capture_output=True, text=True, timeout=600)
        assert r.returncode == 0, r.stderr[-3000:]
        objs.append(obj)
    exe = str(out / "step_driver")
    r = subprocess.run([CLANG, *SAN, *objs, "-o", exe], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    return exe


@pytest.mark.parametrize("seed", ["1", "2", "3"])
def test_calls_clean_under_asan_and_ubsan(driver, seed):
    r = _run(driver, seed, "3")
    assert r.returncode == 0, (r.stdout + r.stderr)[-4000:]
    assert "step driver: OK" in r.stdout


def test_planted_short_page_buffer_is_caught(driver):
    r = _run(driver, "--plant")
    assert r.returncode != 0
    assert "AddressSanitizer: heap-buffer-overflow" in r.stderr
