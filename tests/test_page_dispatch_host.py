"""Which way a suffix call over bf16 pages takes with the workspace that the query names (pic_plan.cpp), on the CPU: the
cases that the rounding tests check stay on the way that they name."""
import os
import subprocess

import pytest

import page_cases
from test_host_sanitizers import CLANG, ROOT

SRC = r"""
#include <cstdio>
#include "pic_internal.h"
int main() {
  pic::AttnShape s;
  s.n_layers = 1;
  s.scale_log2 = 1.f;
  int n, ctx;
  while (std::scanf("%d %d %d %d %d %d", &s.n_q_heads, &s.n_kv_heads, &s.head_dim, &s.batch, &n, &ctx) == 6) {
    s.cache_cap = ctx + n;
    const size_t ws = pic::prefill_bf16_workspace(s, n, ctx);
    const pic::SplitPlan p = pic::plan_prefill_splits(s, n, ctx, ws);
    std::puts(pic::few_bf16_better(s, n, ctx, ws) ? "FEW" : p.n_splits == 1 ? "WHOLE" : p.f32_partials ? "F32_SHARES" : "HALF_SHARES");
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ in this image")
    d = tmp_path_factory.mktemp("plan")
    (d / "plan.cpp").write_text(SRC)
    csrc = os.path.join(ROOT, "paper_2607_28069_amd", "csrc")
    r = subprocess.run([CLANG, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{ROOT}/include", f"-I{csrc}",
                        str(d / "plan.cpp"), os.path.join(csrc, "pic_plan.cpp"), "-o", str(d / "plan")], capture_output=True, text=True,
                       timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]

    def run(cases):
        return subprocess.run([str(d / "plan")], input="\n".join(" ".join(map(str, c)) for c in cases), text=True, capture_output=True,
                              check=True, timeout=60).stdout.split()

    return run


@pytest.mark.parametrize("way", ["FEW", "WHOLE", "F32_SHARES", "HALF_SHARES"])
def test_cases_take_the_way_they_name(plan, way):
    cases = getattr(page_cases, way)
    assert plan(cases) == [way] * len(cases)
