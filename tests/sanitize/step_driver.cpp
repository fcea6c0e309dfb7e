// Sanitizer driver for shared prefixes, page tables grown on the device, and norms with rotation (see sanitize_driver.cpp):
// every launching call with garbage tables, starts, lengths and token counts over buffers of the exact documented sizes,
// and grown tables against pic_page_grow.
//
// usage: step_driver [seed] [rounds]      prints "step driver: OK" and exits 0
//        step_driver --plant              page buffers one row short: must end in an ASan report
#include <algorithm>
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <memory>
#include <random>
#include <vector>

#include "pic.h"

namespace pic {
namespace emu {
extern long launches;
}
}  // namespace pic

namespace {

std::mt19937_64 rng;
int64_t rnd(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }

struct Buf {
  void* p = nullptr;
  explicit Buf(size_t bytes) {
    if (posix_memalign(&p, 16, bytes == 0 ? 1 : bytes) != 0) std::abort();
    std::memset(p, 0, bytes == 0 ? 1 : bytes);
  }
  ~Buf() { std::free(p); }
  Buf(const Buf&) = delete;
  Buf& operator=(const Buf&) = delete;
  int32_t& operator[](int64_t i) { return static_cast<int32_t*>(p)[i]; }
  int32_t* ints() { return static_cast<int32_t*>(p); }
};

int failures = 0;
#define EXPECT(cond)                                                                                    \
  do {                                                                                                  \
    if (!(cond)) {                                                                                      \
      std::fprintf(stderr, "FAILED %s:%d: %s (%s)\n", __FILE__, __LINE__, #cond, pic_last_error());     \
      ++failures;                                                                                       \
    }                                                                                                   \
  } while (0)

int32_t garbage(int32_t scale) {
  switch (rnd(0, 5)) {
    case 0: return (int32_t)rnd(INT32_MIN, INT32_MAX);
    case 1: return -(int32_t)rnd(1, 1 << 20);
    case 2: return (int32_t)rnd(0, 2 * (int64_t)scale + 8);
    default: return (int32_t)rnd(0, scale > 0 ? scale - 1 : 0);
  }
}

pic_model model_of(int L, int hq, int hkv, int D, bool f32) {
  pic_model m;
  std::memset(&m, 0, sizeof(m));
  m.n_layers = L;
  m.n_q_heads = hq;
  m.n_kv_heads = hkv;
  m.head_dim = D;
  m.dtype = f32 ? PIC_F32 : PIC_BF16;
  m.rope_theta = 1e4;
  m.rope_pairing = (int)rnd(0, 1);
  m.rope_tables = rnd(0, 1) ? L : 1;
  return m;
}

void fuzz_attention(bool plant) {
  for (int it = 0; it < 60; ++it) {
    const bool f32 = !plant && rnd(0, 7) == 0, decode = rnd(0, 1);
    const int D = rnd(0, 1) ? 64 : 128, hkv = (int)rnd(1, 3), hq = hkv * (int)rnd(1, it % 9 == 0 ? 70 : 5), L = (int)rnd(1, 2);
    const pic_model m = model_of(L, hq, hkv, D, f32);
    const size_t rb = (size_t)D * (f32 ? 4 : 2);
    const int batch = (int)rnd(1, it % 4 ? 5 : 30), n = decode ? 1 : (int)rnd(1, 40);
    const int32_t max_len = (int32_t)rnd(n, it % 5 == 0 ? 2600 : 300), step = decode ? (int32_t)rnd(0, std::min(max_len - 1, 9)) : 0;
    const int32_t max_base = max_len - n - step;
    pic_pages pg;
    pg.page_tokens = 16 << rnd(0, 3);
    pg.n_pages = (int32_t)rnd(1, 12);
    pg.table_cap = (max_len + pg.page_tokens - 1) / pg.page_tokens + (int32_t)rnd(0, 2);
    const pic_shared sh = {(int32_t)rnd(1, batch + 2), (int32_t)rnd(0, batch + 1), (int32_t)rnd(0, pg.table_cap * pg.page_tokens)};
    const size_t rows = (size_t)L * hkv * pg.n_pages * pg.page_tokens, toks = (size_t)L * batch * n;
    Buf pk(rows * rb - (plant ? rb : 0)), pv(rows * rb), q(toks * hq * rb), k(toks * hkv * rb), v(toks * hkv * rb), out(toks * hq * rb);
    Buf table((size_t)batch * pg.table_cap * 4), lens(batch * 4), nv(batch * 4), start((sh.n_groups + 1) * 4), shared(sh.n_groups * 4);
    for (int i = 0; i < batch * pg.table_cap; ++i) table[i] = plant ? pg.n_pages - 1 : garbage(pg.n_pages);
    for (int b = 0; b < batch; ++b) {
      lens[b] = plant ? max_base : garbage(max_base + 1);
      nv[b] = garbage(n + 1);
    }
    const bool tidy = rnd(0, 1);
    for (int i = 0; i <= sh.n_groups; ++i) start[i] = tidy ? (int32_t)rnd(0, batch) : garbage(batch);
    if (tidy) std::sort(start.ints(), start.ints() + sh.n_groups + 1);
    for (int i = 0; i < sh.n_groups; ++i) shared[i] = garbage(sh.max_len + 1);
    const int32_t* starts = sh.n_groups == 1 && rnd(0, 1) ? nullptr : start.ints();
    size_t need = pic_page_shared_workspace_bytes(&m, &sh, batch, n, max_base + step);
    EXPECT(f32 || need > 0);
    if (f32) need = decode ? 0 : pic_prefill_workspace_bytes(&m, batch, n, max_base);
    Buf ws(need);
    const int32_t* nvp = rnd(0, 1) ? nv.ints() : nullptr;
    auto call = [&](size_t ws_n) {
      return decode ? pic_page_shared_decode_attn(&m, &pg, &sh, q.p, k.p, v.p, pk.p, pv.p, table.ints(), batch, starts, shared.ints(),
                                                  lens.ints(), step, max_base, 0.f, out.p, ws.p, ws_n, nullptr)
                    : pic_page_shared_suffix_attn(&m, &pg, &sh, q.p, k.p, v.p, pk.p, pv.p, table.ints(), batch, starts, shared.ints(),
                                                  lens.ints(), max_base, nvp, n, 0.f, out.p, ws.p, ws_n, nullptr);
    };
    const long before = pic::emu::launches;
    if (!f32) EXPECT(call(need - 1) == PIC_ERR_WORKSPACE && pic::emu::launches == before);
    EXPECT(call(need) == PIC_OK && pic::emu::launches > before);
  }
}

void fuzz_grow() {
  for (int it = 0; it < 200; ++it) {
    pic_pages pg = {(int32_t)rnd(0, 20), 16 << rnd(0, 2), (int32_t)rnd(0, 6)};
    const int32_t batch = (int32_t)rnd(0, 6), n = (int32_t)rnd(0, 40), offset = (int32_t)rnd(0, 3);
    Buf refs(pg.n_pages * 4), table(batch * pg.table_cap * 4), lens(batch * 4), nv(batch * 4), pairs(batch * 8), ready(batch * 4), result(12);
    const bool wild = it % 3 == 0;
    for (int i = 0; i < pg.n_pages; ++i) refs[i] = (int32_t)rnd(0, wild ? 3 : 0);
    for (int i = 0; i < batch * pg.table_cap; ++i) {
      table[i] = pg.n_pages && rnd(0, 2) ? (int32_t)rnd(0, pg.n_pages - 1) : -1;
      if (wild) table[i] = garbage(pg.n_pages);
      else if (table[i] >= 0) ++refs[table[i]];
    }
    for (int b = 0; b < batch; ++b) {
      lens[b] = rnd(0, 3) && !wild ? (int32_t)rnd(0, 50) : garbage(60);
      nv[b] = garbage(n + 1);
    }
    const int32_t* nvp = rnd(0, 1) ? nv.ints() : nullptr;
    std::vector<int32_t> r(refs.ints(), refs.ints() + pg.n_pages), t(table.ints(), table.ints() + batch * pg.table_cap), from(batch), to(batch);
    bool past = false;   // a length past what the host's call can be asked for
    for (int b = 0; b < batch; ++b) {
      const int64_t f = lens[b] < 0 ? 0 : (int64_t)lens[b] + offset;
      const int64_t e = lens[b] < 0 ? 0 : f + (nvp ? std::min(std::max(nv[b], 0), n) : n);
      past = past || e > INT32_MAX;
      from[b] = (int32_t)std::min<int64_t>(f, INT32_MAX);
      to[b] = (int32_t)std::min<int64_t>(e, INT32_MAX);
    }
    const size_t need = pic_page_grow_workspace_bytes(&pg, batch, n);
    Buf ws(need);
    EXPECT(pic_page_grow_async(&pg, batch, refs.ints(), table.ints(), lens.ints(), offset, nvp, n, pairs.ints(), ready.ints(),
                               result.ints(), ws.p, need - 1, nullptr) == PIC_ERR_WORKSPACE);
    EXPECT(pic_page_grow_async(&pg, batch, refs.ints(), table.ints(), lens.ints(), offset, nvp, n, pairs.ints(), ready.ints(),
                               result.ints(), ws.p, need, nullptr) == PIC_OK);
    std::vector<int32_t> want(2 * (size_t)batch + 2, -1);
    int32_t n_pairs = 0;
    const pic_status st = pic_page_grow(&pg, batch, r.data(), t.data(), from.data(), to.data(), want.data(), batch, &n_pairs);
    if (past) continue;
    EXPECT(result[0] == st);
    EXPECT(std::equal(r.begin(), r.end(), refs.ints()) && std::equal(t.begin(), t.end(), table.ints()));
    EXPECT(st != PIC_OK || (result[1] == n_pairs && std::equal(pairs.ints(), pairs.ints() + 2 * n_pairs, want.begin())));
    for (int b = 0; b < batch; ++b) EXPECT(ready[b] == (st == PIC_OK && lens[b] >= 0 ? lens[b] : -1));
    // copies of whatever is listed
    const pic_model m = model_of((int)rnd(1, 2), 2, 1, 64, rnd(0, 1));
    const size_t bytes = (size_t)m.n_layers * pg.n_pages * pg.page_tokens * 64 * (m.dtype == PIC_F32 ? 4 : 2);
    Buf k(bytes), v(bytes), listed(batch * 8);
    for (int i = 0; i < 2 * batch; ++i) listed[i] = garbage(pg.n_pages);
    EXPECT(pic_page_copy_async(&m, &pg, k.p, v.p, listed.ints(), batch, nullptr) == PIC_OK);
  }
}

void fuzz_norm() {
  for (int it = 0; it < 150; ++it) {
    const bool f32 = rnd(0, 1);
    const int D = rnd(0, 1) ? 64 : 128, hkv = (int)rnd(1, 3), hq = hkv * (int)rnd(1, 5), L = (int)rnd(1, 3), es = f32 ? 4 : 2;
    const pic_model m = model_of(L, hq, hkv, D, f32);
    const int batch = (int)rnd(1, 6), n = (int)rnd(1, it % 5 ? 20 : 700);
    const int32_t max_base = (int32_t)rnd(0, 300), offset = (int32_t)rnd(0, 5), mad = max_base + offset + n - 1;
    const int64_t toks = (int64_t)L * batch * n, pad = 16 / es * rnd(0, 3);
    const int64_t sq = hq * D + pad, sk = hkv * D + pad;
    // (rows end where the last token's heads do)
    Buf q(((toks - 1) * sq + hq * D) * es), k(((toks - 1) * sk + hkv * D) * es), v(((toks - 1) * sk + hkv * D) * es);
    Buf qo(toks * hq * D * es), ko(toks * hkv * D * es), vo(toks * hkv * D * es), w(L * D * 4), lens(batch * 4), nv(batch * 4);
    for (int b = 0; b < batch; ++b) {
      lens[b] = garbage(max_base + 1);
      nv[b] = garbage(n + 1);
    }
    Buf table(pic_rope_table_bytes(&m, mad));
    pic_qk_norm how = {static_cast<const float*>(w.p), rnd(0, 1) ? static_cast<const float*>(w.p) : nullptr, 1e-6f,
                       16 * (int32_t)rnd(0, D / 16), (int32_t)rnd(0, 1), 1.f};
    EXPECT(pic_qk_norm_rope(&m, &how, rnd(0, 3) ? q.p : nullptr, sq, rnd(0, 3) ? k.p : nullptr, sk, rnd(0, 1) ? v.p : nullptr, sk, batch,
                            rnd(0, 3) ? lens.ints() : nullptr, max_base, offset, rnd(0, 1) ? nv.ints() : nullptr, n,
                            rnd(0, 3) ? table.p : nullptr, mad, qo.p, ko.p, vo.p, nullptr) == PIC_OK);
  }
}

}  // namespace

int main(int argc, char** argv) {
  if (argc > 1 && std::strcmp(argv[1], "--plant") == 0) {
    rng.seed(1);
    fuzz_attention(true);
    return 0;
  }
  rng.seed(argc > 1 ? std::strtoull(argv[1], nullptr, 10) : 1);
  const int rounds = argc > 2 ? std::atoi(argv[2]) : 2;
  for (int r = 0; r < rounds; ++r) {
    fuzz_attention(false);
    fuzz_grow();
    fuzz_norm();
  }
  if (failures) return 1;
  std::printf("step driver: OK\n");
  return 0;
}
