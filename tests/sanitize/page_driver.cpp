// Sanitizer driver for the paged-cache calls (see sanitize_driver.cpp): fuzzed bookkeeping on host
// arrays of the exact sizes, and every launching call with garbage page tables, lengths and token
// counts over buffers of the exact documented sizes.
//
// usage: page_driver [seed] [rounds]      prints "page driver: OK" and exits 0
//        page_driver --plant              page buffers one row short: must end in an ASan report
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

void fuzz_books() {
  for (int it = 0; it < 200; ++it) {
    pic_pages pg = {(int32_t)rnd(0, 20), 16 << rnd(0, 2), (int32_t)rnd(0, 6)};
    const int32_t batch = (int32_t)rnd(0, 5);
    std::vector<int32_t> refs(pg.n_pages), table((size_t)batch * pg.table_cap, -1), len(batch, 0), to(batch), pairs(2 * batch);
    const bool wild = it % 4 == 0;   // tables and counts that no call left behind
    for (int k = 0; k < 20; ++k) {
      if (wild && !table.empty()) table[rnd(0, (int64_t)table.size() - 1)] = garbage(pg.n_pages);
      if (wild && !refs.empty()) refs[rnd(0, (int64_t)refs.size() - 1)] = (int32_t)rnd(0, 2);
      const int32_t b = batch ? (int32_t)rnd(wild ? -1 : 0, batch - (wild ? 0 : 1)) : 0;
      int32_t n = -1, used = -1;
      switch (rnd(0, 4)) {
        case 0: {
          for (int i = 0; i < batch; ++i) to[i] = len[i] + (int32_t)rnd(wild ? -3 : 0, 40);
          const std::vector<int32_t> r0 = refs, t0 = table;
          const pic_status st = pic_page_grow(&pg, batch, refs.data(), table.data(), len.data(), to.data(), pairs.data(),
                                              (int32_t)rnd(0, batch), &n);
          if (st == PIC_OK) len = to;
          else EXPECT(refs == r0 && table == t0);
          if (wild) for (auto& x : len) x = x < 0 ? 0 : x;
          break;
        }
        case 1: {
          const int32_t d = batch ? (int32_t)rnd(0, batch - 1) : 0, keep = (int32_t)rnd(0, 50);
          const bool ok = b >= 0 && b < batch;
          const pic_status st = pic_page_fork(&pg, batch, refs.data(), table.data(), b, ok ? std::min(keep, len[b]) : keep, d);
          if (st == PIC_OK) len[d] = std::min(keep, len[b]);
          break;
        }
        case 2: {
          const int32_t keep = (int32_t)rnd(0, 40);
          const pic_status st = pic_page_free(&pg, batch, refs.data(), table.data(), b, keep);
          if (st == PIC_OK) len[b] = std::min(len[b], keep);
          else EXPECT(wild || batch == 0);
          break;
        }
        case 3: {
          const int32_t cap = (int32_t)rnd(0, pg.n_pages / 2);
          std::vector<int32_t> moves(2 * (size_t)cap);
          const pic_status st = pic_page_compact(&pg, batch, refs.data(), table.data(), moves.data(), cap, &n, &used);
          EXPECT(wild || st == PIC_OK || (st == PIC_ERR_CAPACITY && n > cap));
          break;
        }
        default: {
          std::vector<pic_block> blocks(rnd(0, 5));
          for (auto& x : blocks)
            x = {(int32_t)rnd(-1, batch), (int32_t)rnd(0, 100), wild ? garbage(100) : (int32_t)rnd(0, 60), (int32_t)rnd(0, 65), 3};
          std::vector<pic_block> out(rnd(0, 12));
          pic_page_blocks(&pg, batch, table.data(), blocks.data(), (int32_t)blocks.size(), out.data(), (int32_t)out.size(), &n);
        }
      }
    }
  }
}

void fuzz_calls(bool plant) {
  for (int it = 0; it < 60; ++it) {
    const bool f32 = rnd(0, 3) == 0, rope = !f32 && rnd(0, 1);
    const int D = rnd(0, 1) ? 64 : 128, hkv = (int)rnd(1, 3), hq = hkv * (int)rnd(1, it % 9 == 0 ? 20 : 5), L = (int)rnd(1, 2);
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
    const size_t rb = (size_t)D * (f32 ? 4 : 2);
    const bool decode = rnd(0, 1), deal = decode && it % 6 == 0;
    const int batch = (int)rnd(deal ? 2 : 1, 4), n = decode ? 1 : (int)rnd(1, 40);
    const int32_t max_len = deal ? 8200 : (int32_t)rnd(n, it % 5 == 0 ? 2600 : 300), step = decode ? (int32_t)rnd(0, std::min(max_len - 1, 9)) : 0;
    const int32_t max_base = max_len - n - step;
    pic_pages pg;
    pg.page_tokens = 16 << rnd(0, 3);
    pg.n_pages = (int32_t)rnd(1, 12);
    pg.table_cap = (max_len + pg.page_tokens - 1) / pg.page_tokens + (int32_t)rnd(0, 2);
    const size_t rows = (size_t)L * hkv * pg.n_pages * pg.page_tokens, toks = (size_t)L * batch * n;
    Buf pk(rows * rb - (plant ? rb : 0)), pv(rows * rb), q(toks * hq * rb), k(toks * hkv * rb), v(toks * hkv * rb), out(toks * hq * rb);
    std::unique_ptr<int32_t[]> table(new int32_t[(size_t)batch * pg.table_cap]), lens(new int32_t[batch]), nv(new int32_t[batch]);
    for (int i = 0; i < batch * pg.table_cap; ++i) table[i] = plant ? pg.n_pages - 1 : garbage(pg.n_pages);
    for (int b = 0; b < batch; ++b) {
      lens[b] = plant ? max_base : garbage(max_base + 1);
      nv[b] = garbage(n + 1);
    }
    const int32_t mad = max_len - 1;
    Buf rt(pic_rope_table_bytes(&m, mad));
    const int32_t splits = deal ? 8 : (int32_t)rnd(0, 5);
    const size_t ws_n = decode ? pic_decode_workspace_bytes(&m, batch, max_len, splits) : pic_prefill_workspace_bytes(&m, batch, n, max_base);
    Buf ws(ws_n);
    void* wp = ws_n ? ws.p : nullptr;
    const int32_t* nvp = rnd(0, 1) ? nv.get() : nullptr;
    const long before = pic::emu::launches;
    pic_status st;
    if (decode) {
      st = rope ? pic_page_decode_attn_rope(&m, &pg, q.p, k.p, v.p, pk.p, pv.p, table.get(), batch, lens.get(), step, max_base, rt.p,
                                            mad, 0.f, splits, out.p, wp, ws_n, nullptr)
                : pic_page_decode_attn(&m, &pg, q.p, k.p, v.p, pk.p, pv.p, table.get(), batch, lens.get(), step, max_base, 0.f,
                                       splits, out.p, wp, ws_n, nullptr);
    } else {
      st = rope ? pic_page_suffix_attn_rope(&m, &pg, q.p, k.p, v.p, pk.p, pv.p, table.get(), batch, lens.get(), max_base, nvp, n,
                                            rt.p, mad, 0.f, out.p, wp, ws_n, nullptr)
                : pic_page_suffix_attn(&m, &pg, q.p, k.p, v.p, pk.p, pv.p, table.get(), batch, lens.get(), max_base, nvp, n, 0.f,
                                       out.p, wp, ws_n, nullptr);
    }
    EXPECT(st == PIC_OK && pic::emu::launches > before);
    // a call whose table is too small for its lengths, and copies that overlap, launch nothing
    const long quiet = pic::emu::launches;
    pic_pages small = pg;
    small.table_cap = (max_len - 1) / pg.page_tokens;
    EXPECT(pic_page_decode_attn(&m, &small, q.p, k.p, v.p, pk.p, pv.p, table.get(), batch, lens.get(), 0, max_len - 1, 0.f, 1, out.p,
                                nullptr, 0, nullptr) == PIC_ERR_CAPACITY);
    std::vector<int32_t> pairs;
    for (int i = 0; i < pg.n_pages; ++i) {
      pairs.push_back(garbage(pg.n_pages));
      pairs.push_back(garbage(pg.n_pages));
    }
    bool good = true;
    for (size_t i = 0; i < pairs.size(); ++i) {
      good = good && pairs[i] >= 0 && pairs[i] < pg.n_pages;
      for (size_t j = 1; j < pairs.size(); j += 2) good = good && (i == j || pairs[i] != pairs[j]);
    }
    EXPECT((pic_page_copy(&m, &pg, pk.p, pv.p, pairs.data(), pg.n_pages, nullptr) == PIC_OK) == good);
    EXPECT(good || pic::emu::launches == quiet);
    if (pg.n_pages >= 2) {
      const int32_t one[2] = {pg.n_pages - 1, 0};
      EXPECT(pic_page_copy(&m, &pg, pk.p, pv.p, one, 1, nullptr) == PIC_OK);
    }
  }
}

}  // namespace

int main(int argc, char** argv) {
  if (argc > 1 && std::strcmp(argv[1], "--plant") == 0) {
    rng.seed(1);
    fuzz_calls(true);
    return 0;
  }
  rng.seed(argc > 1 ? std::strtoull(argv[1], nullptr, 10) : 1);
  const int rounds = argc > 2 ? std::atoi(argv[2]) : 2;
  for (int r = 0; r < rounds; ++r) {
    fuzz_books();
    fuzz_calls(false);
  }
  if (failures) return 1;
  std::printf("page driver: OK\n");
  return 0;
}
