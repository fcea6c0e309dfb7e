"""The launch plan of attention over shared prefixes (pic_shared.cpp), on the CPU: the workspace that the query names holds every
part that the launch writes, whatever the sizes."""
import os
import random
import subprocess

import pytest

from test_host_sanitizers import CLANG, ROOT

SRC = r"""
#include <algorithm>
#include <cstdio>
#include "pic_internal.h"
int main() {
  pic::AttnShape s;
  pic::SharedMap m;
  int n, ctx;
  s.scale_log2 = 1.f;
  while (std::scanf("%d %d %d %d %d %d %d %d %d %d", &s.n_layers, &s.n_q_heads, &s.n_kv_heads, &s.head_dim, &s.batch, &m.n_groups,
                    &m.max_group, &m.max_len, &n, &ctx) == 10) {
    m.batch = s.batch;
    m.max_group = std::min(m.max_group, s.batch);
    const pic::SharedPlan p = pic::plan_shared(s, m, n, ctx);
    std::printf("%d %d %d %zu\n", p.prefix_splits, p.own_splits, p.prefix_terms, p.ws_bytes);
  }
}
"""


@pytest.fixture(scope="module")
def plan(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ in this image")
    d = tmp_path_factory.mktemp("shared_plan")
    (d / "plan.cpp").write_text(SRC)
    csrc, san = os.path.join(ROOT, "paper_2607_28069_amd", "csrc"), os.path.join(ROOT, "tests", "sanitize")
    files = [str(d / "plan.cpp")] + [os.path.join(csrc, f) for f in ("pic_shared.cpp", "pic_api.cpp", "pic_pages.cpp", "pic_plan.cpp",
                                                                     "pic_grow.cpp", "pic_tokens.cpp")]
    files += [os.path.join(san, f) for f in ("emulated_launchers.cpp", "page_launchers.cpp", "step_launchers.cpp")]
    r = subprocess.run([CLANG, "-std=c++17", "-O1", "-D__HIP_PLATFORM_AMD__", "-I/opt/rocm/include", f"-I{ROOT}/include", f"-I{csrc}",
                        *files, "-o", str(d / "plan")], capture_output=True, text=True, timeout=600)
    assert r.returncode == 0, r.stderr[-3000:]

    def run(cases):
        """(prefix ranges, own ranges, terms of a probability, workspace bytes) of each (layers, query heads, kv heads, head_dim,
        batch, groups, max_group, max_len, new tokens, max_ctx)."""
        out = subprocess.run([str(d / "plan")], input="\n".join(" ".join(map(str, c)) for c in cases), text=True, capture_output=True,
                             check=True, timeout=60).stdout.split()
        out = [int(x) for x in out]
        return list(zip(out[::4], out[1::4], out[2::4], out[3::4]))

    return run


def written(case, plan):
    layers, hq, _, d, batch, _, _, _, n, _ = case
    return layers * batch * n * hq * (plan[0] + plan[1]) * (d + 2) * 4


def test_workspace_of_huge_batches(plan):
    """Batches of 2^22 requests and more, whose products with 512 workgroups pass 31 bits."""
    cases = [(1, hq, hkv, d, b, g, m, 4096, 1, 8192) for hq, hkv, d in ((1, 1, 64), (4, 1, 128), (16, 8, 64)) for g, m in ((1, 8), (3, 1), (2, 2))
             for b in (1 << 21, (1 << 22) - 1, 1 << 22, (1 << 22) + 5, 1 << 23, (1 << 27) // hq - 1) if b * hq < 1 << 27]
    for c, p in zip(cases, plan(cases)):
        assert p[3] >= written(c, p), (c, p)


def test_workspace_of_any_sizes(plan):
    r = random.Random(1)
    log = lambda lo, hi: int(round(lo * (hi / lo) ** r.random()))  # noqa: E731
    cases = []
    while len(cases) < 4000:
        hkv = r.choice([1, 2, 4, 8, 16])
        c = (r.choice([1, 1, 2, 32]), hkv * r.choice([1, 2, 4, 7, 8]), hkv, r.choice([64, 128]), log(1, 1 << 20), log(1, 300), r.choice([0, log(1, 5000)]),
             r.choice([0, log(1, 1 << 20)]), r.choice([1, log(1, 300)]), log(1, 1 << 20))
        if c[0] * c[1] * c[4] * c[8] < 1 << 27:
            cases.append(c)
    for c, p in zip(cases, plan(cases)):
        assert p[3] >= written(c, p), (c, p)


def test_requests_of_no_group_are_split(plan):
    """Where a batch is larger than its groups, some requests read all of their slots by themselves: no range of these is as long as
    one of the launch's whole time should be (64 tiles of 64 keys), nor is the other requests' prefix left whole."""
    cases = [(1, 32, 8, 128, 4, 1, 2, 32000, 1, 32100), (1, 32, 8, 128, 8, 1, 4, 10368, 1, 10500), (1, 32, 8, 128, 16, 1, 8, 10368, 1, 10500),
             (1, 28, 4, 128, 33, 4, 8, 32000, 1, 32596), (1, 32, 8, 128, 2, 1, 1, 2048, 1, 2100), (2, 32, 8, 64, 6, 1, 3, 8000, 5, 8200)]
    for c, p in zip(cases, plan(cases)):
        assert -(-c[9] // 64) / p[1] <= 64 and c[7] // 64 / p[0] <= 64, (c, p)


def test_parts_of_many_rows(plan):
    """Rows so many that each part costs more than the prefix are given few: most of 4096 requests share nothing here."""
    cases = [(1, 8, 1, 128, 4096, 1, 2, 2048, n, 2100) for n in (1, 8)] + [(1, 8, 1, 128, 4096, 3, 700, 2048, 8, 2100)]
    for c, p in zip(cases, plan(cases)):
        assert p[0] <= 16, (c, p)
