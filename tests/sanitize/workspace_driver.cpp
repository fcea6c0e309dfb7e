// What calls over pages write of their workspace: at most the bytes that the query call names, whatever larger buffer
// they bring (calls whose query is 0 may overlap and share one), and nothing of a misaligned one.  The launches are
// emulated (page_launchers.cpp); run under AddressSanitizer and UndefinedBehaviorSanitizer.
//
// usage: workspace_driver [seed]      prints "workspace driver: OK, <n> calls of query 0" and exits 0
#include <cstdint>
#include <cstdio>
#include <cstdlib>
#include <cstring>
#include <random>
#include <vector>

#include "pic.h"

namespace {

std::mt19937_64 rng;
int64_t rnd(int64_t lo, int64_t hi) { return std::uniform_int_distribution<int64_t>(lo, hi)(rng); }
int failures = 0, none = 0;

struct Buf {
  uint8_t* p = nullptr;
  size_t n;
  explicit Buf(size_t bytes) : n(bytes) {
    if (posix_memalign((void**)&p, 16, bytes + 16) != 0) std::abort();
    std::memset(p, 0xA5, bytes + 16);
  }
  ~Buf() { std::free(p); }
  Buf(const Buf&) = delete;
  Buf& operator=(const Buf&) = delete;
  bool untouched(size_t from) const {
    for (size_t i = from; i < n; ++i)
      if (p[i] != 0xA5) return false;
    return true;
  }
};

void one(bool decode) {
  static const int shapes[][3] = {{32, 8, 128}, {28, 4, 128}, {8, 2, 64}, {32, 8, 64}, {16, 1, 64}, {4, 4, 128}};
  const int* sh = shapes[rnd(0, 5)];
  pic_model m;
  std::memset(&m, 0, sizeof(m));
  m.n_layers = 1;
  m.n_q_heads = sh[0];
  m.n_kv_heads = sh[1];
  m.head_dim = sh[2];
  m.dtype = PIC_BF16;
  m.rope_theta = 1e4;
  const int batch = (int)rnd(1, rnd(0, 2) ? 4 : 24), n = decode ? 1 : (int)rnd(1, rnd(0, 2) ? 8 : 70);
  const int32_t max_base = (int32_t)rnd(0, 3000), splits = (int32_t)rnd(0, 1);
  pic_pages pg = {8, 64, (max_base + n + 63) / 64};
  const size_t rb = (size_t)m.head_dim * 2, toks = (size_t)batch * n;
  Buf pages(2 * (size_t)m.n_kv_heads * 8 * 64 * rb), q(toks * m.n_q_heads * rb), kv(toks * m.n_kv_heads * rb), out(toks * m.n_q_heads * rb);
  std::vector<int32_t> table((size_t)batch * pg.table_cap), lens(batch);
  for (auto& t : table) t = (int32_t)rnd(0, 7);
  for (auto& b : lens) b = (int32_t)rnd(0, max_base);
  lens[0] = max_base;
  const size_t named = decode ? pic_decode_workspace_bytes(&m, batch, max_base + 1, splits) : pic_prefill_workspace_bytes(&m, batch, n, max_base);
  none += named == 0;
  uint8_t *pk = pages.p, *pv = pages.p + pages.n / 2;
  auto call = [&](void* ws, size_t bytes) {
    return decode ? pic_page_decode_attn(&m, &pg, q.p, kv.p, kv.p, pk, pv, table.data(), batch, lens.data(), 0, max_base, 0.f, splits, out.p,
                                         ws, bytes, nullptr)
                  : pic_page_suffix_attn(&m, &pg, q.p, kv.p, kv.p, pk, pv, table.data(), batch, lens.data(), max_base, nullptr, n, 0.f, out.p,
                                         ws, bytes, nullptr);
  };
  {
    Buf ws(named + (32 << 20));
    const pic_status st = call(ws.p, ws.n);
    if (st != PIC_OK || !ws.untouched(named)) {
      std::fprintf(stderr, "%s, %d/%d heads of %d, %d requests x %d tokens after %d: status %d, %zu bytes named, more written: %d\n",
                   decode ? "decode" : "suffix", sh[0], sh[1], sh[2], batch, n, max_base, st, named, !ws.untouched(named));
      ++failures;
    }
  }
  {
    Buf ws(named + (8 << 20));
    const pic_status st = call(ws.p + 8, ws.n);
    if ((st != PIC_OK && st != PIC_ERR_MISALIGNED) || (named == 0 && st != PIC_OK) || !ws.untouched(0)) {
      std::fprintf(stderr, "%s, %d/%d heads of %d, %d requests x %d tokens after %d: misaligned, status %d, %zu bytes named, written: %d\n",
                   decode ? "decode" : "suffix", sh[0], sh[1], sh[2], batch, n, max_base, st, named, !ws.untouched(0));
      ++failures;
    }
  }
}

}  // namespace

int main(int argc, char** argv) {
  rng.seed(argc > 1 ? std::strtoull(argv[1], nullptr, 10) : 1);
  for (int i = 0; i < 40; ++i) one(i % 4 == 0);
  if (failures) return 1;
  std::printf("workspace driver: OK, %d calls of query 0\n", none);
  return 0;
}
