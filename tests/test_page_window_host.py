"""Where the kernels over pages find their rows and their work, on the CPU, with the functions that they call
(pic_bounds.h): the windows on the page table, walked as the decode, few-rows, float32 and prefill kernels walk them,
name page_row's rows and never reach past a register's 64 lanes; and a dealt launch has one workgroup for every
(request, kv head, key range, tile of query rows)."""
import os
import subprocess

import pytest

from test_host_sanitizers import CLANG, ROOT, SAN

SRC = r"""
#include <algorithm>
#include <cstdio>
#include <random>
#include <set>
#include <tuple>
#include <vector>
#include "pic_bounds.h"
using namespace pic;
std::mt19937_64 rng(1);
int64_t rnd(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }
#define NEED(c) do { if (!(c)) { std::printf("line %d: %s\n", __LINE__, #c); std::exit(1); } } while (0)

struct Walk {   // the two registers of a wave
  PageMap m;
  int b;
  int32_t step;
  PageWindow win;
  int32_t cur[64], next[64];
  int32_t entry(int32_t i) const { return m.table[(int64_t)b * m.cap + clamp_entry(i, m)]; }
  Walk(const PageMap& map, int req, int32_t st, int32_t first) : m(map), b(req), step(st), win{first} {
    for (int j = 0; j < 64; ++j) cur[j] = entry(win.at + j), next[j] = entry(win.at + step + j);
  }
  void ask(int32_t i) {
    if (!win.moves(i, step)) return;
    std::copy(next, next + 64, cur);
    for (int j = 0; j < 64; ++j) next[j] = entry(win.at + step + j);
  }
  int64_t row(int32_t slot) const {
    const int32_t lane = win.lane(slot >> m.shift);
    NEED(lane >= 0 && lane < 64);
    return ((int64_t)clamp_page(cur[lane], m) << m.shift) + (slot & ((1 << m.shift) - 1));
  }
};

void windows() {
  for (int it = 0; it < 400; ++it) {
    PageMap m;
    m.shift = (int)rnd(4, 10);
    m.n_pages = (int)rnd(1, 50);
    m.cap = (int)rnd(1, it % 3 ? 40 : 900);
    std::vector<int32_t> table(2 * (size_t)m.cap);
    for (auto& t : table) t = rnd(0, 9) ? (int32_t)rnd(0, m.n_pages - 1) : (int32_t)rnd(INT32_MIN, INT32_MAX);
    m.table = table.data();
    const int b = (int)rnd(0, 1), slots = m.cap << m.shift;
    // decode and few rows: tiles of 32 keys in two blocks of 16, from a multiple of 32
    {
      const int c0 = (int)rnd(0, (slots - 1) / 32) * 32, c1 = (int)rnd(c0 + 1, std::min(slots, c0 + (it % 5 ? 3000 : 100000)));
      Walk w(m, b, 64, c0 >> m.shift);
      for (int k0 = c0; k0 < c1; k0 += 32)
        for (int mb = 0; mb < 2; ++mb) {
          const int slot16 = std::min(k0 + 16 * mb, (c1 - 1) & ~15);
          w.ask(slot16 >> m.shift);
          for (int key = slot16; key < std::min(slot16 + 16, c1); ++key) NEED(w.row(slot16) + (key - slot16) == page_row(m, b, key));
        }
    }
    // float32: wave v of W takes every W-th tile of 16
    for (int W : {4, 8})
      for (int v = 0; v < W; ++v) {
        Walk w(m, b, 64, (v * 16) >> m.shift);
        for (int t = v; t * 16 < slots; t += W) {
          w.ask((t * 16) >> m.shift);
          for (int i = 0; i < 16; ++i) NEED(w.row(t * 16) + i == page_row(m, b, t * 16 + i));
        }
      }
    // prefill: 64-key tiles, one after another and two past the last; wave v moves `rows` rows at rows (8 i + v)
    for (int rows : {4, 8})
      for (int v = 0; v < 8; ++v) {
        const int t0 = (int)rnd(0, (slots - 1) / 64), steps = 64 / (rows * 8);
        Walk w(m, b, 56, (t0 * 64 + rows * v) >> m.shift);
        for (int T = t0; T * 64 < slots + 128; ++T) {
          w.ask((T * 64 + rows * v) >> m.shift);
          for (int i = 0; i < steps; ++i) {
            const int slot = T * 64 + rows * (8 * i + v);
            const int64_t r = w.row(slot);
            for (int k = 0; k < rows && slot + k < slots; ++k) NEED(r + k == page_row(m, b, slot + k));
          }
        }
      }
  }
}

void blocks() {
  for (int it = 0; it < 3000; ++it) {
    const int batch = (int)rnd(2, 64), heads = (int)rnd(1, 8), xcds = 8;
    std::vector<int> n(batch), tok(batch), m(batch), wgs(batch);
    int total = 0;
    for (int b = 0; b < batch; ++b) {
      tok[b] = rnd(0, 3) ? (int)rnd(1, 300) : 0;
      n[b] = tok[b] ? (int)rnd(1, it % 4 ? 5 : 40) : 0;
      m[b] = tok[b] ? (int)rnd(1, 4) : 0;
      total += wgs[b] = n[b] * m[b] * heads;
    }
    const int grid = (total + (int)rnd(0, 30) + xcds - 1) / xcds * xcds;
    std::set<std::tuple<int, int, int, int>> seen;
    auto of = [](const std::vector<int>& v) { return [&v](int b) { NEED(b < (int)v.size()); return v[b]; }; };
    for (int w = 0; w < grid; ++w) {
      DealtBlock x;
      if (!dealt_block(w, xcds, total, of(wgs), of(n), of(m), of(tok), x)) continue;
      NEED(x.b >= 0 && x.b < batch && x.g >= 0 && x.g < heads && x.split >= 0 && x.split < n[x.b] && x.mt >= 0 && x.mt < m[x.b]);
      int first = 0;
      for (int b = 0; b < x.b; ++b) first += n[b] * tok[b];
      NEED(x.first == first && x.ranges == n[x.b] && x.row_tiles == m[x.b]);
      NEED(seen.insert({x.b, x.g, x.split, x.mt}).second);
    }
    NEED((int)seen.size() == total);
  }
}

int main() {
  windows();
  blocks();
  std::printf("OK\n");
}
"""


@pytest.fixture(scope="module")
def walker(tmp_path_factory):
    if not os.path.exists(CLANG):
        pytest.skip("no clang++ in this image")
    d = tmp_path_factory.mktemp("window")
    (d / "window.cpp").write_text(SRC)
    r = subprocess.run([CLANG, "-std=c++17", "-O1", *SAN, "-fno-sanitize-recover=all", f"-I{ROOT}/include",
                        f"-I{ROOT}/paper_2607_28069_amd/csrc", str(d / "window.cpp"), "-o", str(d / "window")], capture_output=True,
                       text=True, timeout=300)
    assert r.returncode == 0, r.stderr[-3000:]
    return str(d / "window")


def test_windows_and_dealt_workgroups(walker):
    r = subprocess.run([walker], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.strip() == "OK", (r.stdout + r.stderr)[-3000:]
