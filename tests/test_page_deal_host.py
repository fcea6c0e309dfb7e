"""How a split suffix prefill over pages deals its key ranges to uneven requests (pic_bounds.h), on the CPU: the
candidate sizes run from the mean to the longest request in n_splits ranges, which always fits; the size
taken is the first whose workgroups and partials fit those of n_splits ranges of every request.  Then the
kernel's block order: every (request, kv head, tile of query rows, range) has one workgroup.  (The kernels'
own arithmetic is compared on the GPU.)"""
import os
import random
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
CLANG = "/opt/rocm/llvm/bin/clang++"
SRC = r"""
#include <cstdio>
#include "pic_bounds.h"
int main() {
  long long total;
  int longest, n_splits, groups;
  while (std::scanf("%lld %d %d %d", &total, &longest, &n_splits, &groups) == 4) {
    const pic::RangeCandidates rc = pic::suffix_range_candidates(total, longest, n_splits, groups);
    for (int i = 0; i < pic::kDecodeDealt; ++i) {
      const int c = rc.at(i);
      // (a reciprocal that is an ulp off, as the hardware's may be)
      for (int ulp = -1; ulp <= 1; ++ulp)
        if (pic::ceil_div24(longest, c, 1.0f / c * (1 + ulp * 1.2e-7f)) != pic::ceil_div(longest, c)) return 1;
      std::printf("%d ", c);
    }
    std::printf("\n");
  }
}
"""
ceil = lambda x, y: -(-x // y)  # noqa: E731


@pytest.fixture(scope="module")
def candidates(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ in this image")
    d = tmp_path_factory.mktemp("deal")
    (d / "deal.cpp").write_text(SRC)
    subprocess.run([CLANG, "-std=c++17", "-O1", f"-I{ROOT}/include", f"-I{ROOT}/paper_2607_28069_amd/csrc",
                    str(d / "deal.cpp"), "-o", str(d / "deal")], check=True, timeout=120)

    def run(rows):
        r = subprocess.run([str(d / "deal")], input="\n".join(" ".join(map(str, x)) for x in rows), text=True,
                           capture_output=True, check=True, timeout=60)
        return [[int(v) for v in line.split()] for line in r.stdout.splitlines()]

    return run


def _cases(rng, count):
    """(n_splits, n_new, rows per token, [(tiles, tokens)] with padding among them)"""
    out = []
    for _ in range(count):
        batch, n_new, rep = rng.randint(2, 64), rng.choice([1, 9, 64, 65, 67, 128, 300]), rng.choice([1, 4, 7])
        top = rng.choice([1, 2, 9, 64, 512, 1 << 24])
        reqs = []
        for _ in range(batch):
            tok = rng.choice([n_new, n_new, rng.randint(0, n_new)])
            reqs.append((rng.randint(1, top) if tok else 0, tok))
        reqs[rng.randrange(batch)] = (top, n_new)
        out.append((rng.choice([2, 3, 5, 8, 31, 32]), n_new, rep, reqs))
    return out


def _sizes(candidates, cases):
    rows = []
    for s, n_new, rep, reqs in cases:
        rows.append((sum(u * ceil(t * rep, 256) for u, t in reqs), max(u for u, _ in reqs), s,
                     len(reqs) * ceil(n_new * rep, 256)))
    return candidates(rows)


def test_candidates_fit_and_ranges_cover(candidates):
    cases = _cases(random.Random(0), 1500)
    for (s, n_new, rep, reqs), cs in zip(cases, _sizes(candidates, cases)):
        m = ceil(n_new * rep, 256)

        def fits(c):
            return (sum(ceil(u, c) * ceil(t * rep, 256) for u, t in reqs) <= s * len(reqs) * m
                    and sum(ceil(u, c) * t for u, t in reqs) <= s * len(reqs) * n_new)

        longest = max(u for u, _ in reqs)
        assert cs == sorted(cs) and cs[0] >= 1 and cs[-1] == ceil(longest, min(s, longest)) and fits(cs[-1])
        size = next(c for c in cs if fits(c))
        assert size >= min(8, cs[-1])
        first, places, blocks = 0, set(), 0
        for u, t in reqs:
            n = ceil(u, size)
            if u:   # equal ranges, each with keys
                assert (n - 1) * ceil(u, n) < u <= n * ceil(u, n) <= n * size
            places.update(range(first, first + n * t))      # (tokens of) partials of its own
            first += n * t
            blocks += n * ceil(t * rep, 256)
        assert len(places) == first <= s * len(reqs) * n_new and blocks <= s * len(reqs) * m


def test_every_range_has_one_workgroup(candidates):
    """The kernel's block order, over 8 XCDs, in a grid sized for n_splits ranges of every request."""
    cases = [x for x in _cases(random.Random(1), 400) if max(u for u, _ in x[3]) <= 512 and len(x[3]) <= 12]
    assert len(cases) > 30
    for (s, n_new, rep, reqs), cs in zip(cases, _sizes(candidates, cases)):
        heads, m = 3, ceil(n_new * rep, 256)
        n_wg = m * s * len(reqs) * heads
        size = next(c for c in cs if sum(ceil(u, c) * ceil(t * rep, 256) for u, t in reqs) <= s * len(reqs) * m
                    and sum(ceil(u, c) * t for u, t in reqs) <= s * len(reqs) * n_new)
        n, mt = [ceil(u, size) for u, _ in reqs], [ceil(t * rep, 256) for _, t in reqs]
        wgs = [a * b * heads for a, b in zip(n, mt)]
        total = sum(wgs)
        per = ceil(total, 8)
        seen = set()
        for w in range(ceil(n_wg, 8) * 8):
            at, in_b, b = w // 8, (w % 8) * per + w // 8, 0
            if at >= per or in_b >= total:
                continue
            while in_b >= wgs[b]:
                in_b -= wgs[b]
                b += 1
            key = (b, in_b // (mt[b] * n[b]), mt[b] - 1 - in_b % mt[b], in_b // mt[b] % n[b])
            assert key not in seen and key[1] < heads and key[2] >= 0
            seen.add(key)
        assert len(seen) == total
