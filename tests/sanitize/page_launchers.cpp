// CPU emulation of the launches over paged caches, for the sanitizer build of the host library (see
// emulated_launchers.cpp): the grids, ranges and partial slots of page_copy.hip, page_decode.hip,
// page_few.hip and the pages modes of prefill_bf16.hip and attn_f32.hip, every row found with the
// kernels' own clamping helpers and touched in host memory.
#include <algorithm>
#include <cstring>
#include <vector>

#include "pic_internal.h"

namespace pic {
namespace emu {
extern long launches;
}

namespace {

void rd(const void* base, int64_t row, int64_t bytes) {
  const volatile uint8_t* p = static_cast<const uint8_t*>(base) + row * bytes;
  (void)p[0];
  (void)p[bytes - 1];
}
void wr(void* base, int64_t row, int64_t bytes) {
  uint8_t* p = static_cast<uint8_t*>(base) + row * bytes;
  p[0] = 0;
  p[bytes - 1] = 0;
}

// One request, layer and kv head of a call.
struct Stream {
  const PageAttnArgs& a;
  int64_t es;   // element bytes
  int l, b, g, n_tok, ctx;

  Stream(const PageAttnArgs& args, int64_t elem, int l_, int b_, int g_) : a(args), es(elem), l(l_), b(b_), g(g_) {
    n_tok = page_new_tokens(a.base_len, a.n_valid, b, a.n_new);
    ctx = n_tok > 0 ? clamp_len(a.base_len[b], a.max_base) + a.offset : 0;
  }
  int64_t rb() const { return a.s.head_dim * es; }
  int64_t row0() const { return ((int64_t)l * a.s.n_kv_heads + g) * a.s.cache_cap; }
  int64_t new_row(int i) const { return (((int64_t)l * a.s.batch + b) * a.n_new + i) * a.s.n_kv_heads + g; }
  int64_t q_row(int i, int h) const { return (((int64_t)l * a.s.batch + b) * a.n_new + i) * a.s.n_q_heads + h; }
  void turn(int pos) const {
    if (a.table) rd(a.table + l * a.table_stride, std::min(pos, a.max_abs_delta), (int64_t)a.s.head_dim / 2 * 8);
  }
  void key(int slot) const {   // a slot the request sees
    if (slot >= ctx) {
      rd(a.k_new, new_row(slot - ctx), rb());
      rd(a.v_new, new_row(slot - ctx), rb());
      turn(slot);
    } else {
      rd(a.pages_k, row0() + page_row(a.map, b, slot), rb());
      rd(a.pages_v, row0() + page_row(a.map, b, slot), rb());
    }
  }
  void entries(int slot) const {   // the window of 128 table entries a wave holds from its first slot on
    for (int j = 0; j < 128; ++j)
      (void)*const_cast<const volatile int32_t*>(a.map.table + (int64_t)b * a.map.cap + clamp_entry((slot >> a.map.shift) + j, a.map));
  }
  void keys(int c0, int c1) const {
    if (c0 >= c1) return;
    entries(c0);
    for (int s = c0; s < c1; ++s) key(s);
  }
  void store(int i) const {
    const int64_t row = page_store_row(a.map, b, ctx + i);
    if (row < 0) return;
    wr(a.pages_k, row0() + row, rb());
    wr(a.pages_v, row0() + row, rb());
  }
};

}  // namespace

hipError_t launch_page_copy(void* pages_k, void* pages_v, int64_t n_streams, int64_t n_pages, int64_t page_bytes,
                            const int32_t* pairs, int32_t n_pairs, hipStream_t) {
  ++emu::launches;
  for (int64_t st = 0; st < n_streams; ++st)
    for (int32_t i = 0; i < n_pairs; ++i)
      for (void* p : {pages_k, pages_v}) {
        uint8_t* base = static_cast<uint8_t*>(p) + st * n_pages * page_bytes;
        std::memcpy(base + pairs[2 * i + 1] * page_bytes, base + pairs[2 * i] * page_bytes, page_bytes);
      }
  return hipSuccess;
}

hipError_t launch_attn_f32_pages(const PageAttnArgs& a) {
  ++emu::launches;
  for (int l = 0; l < a.s.n_layers; ++l)
    for (int b = 0; b < a.s.batch; ++b)
      for (int g = 0; g < a.s.n_kv_heads; ++g) {
        const Stream s(a, 4, l, b, g);
        if (s.n_tok == 0) continue;
        s.keys(0, s.ctx + s.n_tok);
        const int n_rep = a.s.n_q_heads / a.s.n_kv_heads;
        for (int i = 0; i < s.n_tok; ++i) {
          s.store(i);
          for (int h = 0; h < n_rep; ++h) {
            rd(a.q, s.q_row(i, g * n_rep + h), s.rb());
            wr(a.out, s.q_row(i, g * n_rep + h), s.rb());
          }
        }
      }
  return hipSuccess;
}

hipError_t launch_decode_bf16_pages(const PageAttnArgs& a) {
  ++emu::launches;
  const AttnShape& s = a.s;
  const int32_t max_len = a.max_base + a.offset + 1;
  const int64_t rows_all = (int64_t)s.n_layers * s.batch * s.n_q_heads * a.n_splits;
  float* ws_o = static_cast<float*>(a.workspace);
  float* ws_ml = ws_o ? ws_o + rows_all * s.head_dim : nullptr;
  int64_t dealt_chunk = 0;   // equal ranges are of the request's own keys
  std::vector<int32_t> mine(s.batch, a.n_splits), first(s.batch + 1, 0);
  if (decode_dealt(a.n_splits, s.batch, max_len)) {
    std::vector<int32_t> u(s.batch);
    int32_t total = 0, longest = 0;
    for (int b = 0; b < s.batch; ++b) {
      u[b] = a.base_len[b] < 0 ? 0 : decode_units(clamp_len(a.base_len[b], a.max_base) + a.offset + 1);
      total += u[b];
      longest = std::max(longest, u[b]);
    }
    if (longest == 0) return hipSuccess;
    const RangeCandidates rc = decode_range_candidates(total, longest, a.n_splits, s.batch);
    int32_t c = 0;
    for (int i = 0; i < kDecodeDealt; ++i) {
      c = rc.at(i);
      int64_t sum = 0;
      for (int b = 0; b < s.batch; ++b) sum += ceil_div(u[b], c);
      if (sum <= (int64_t)a.n_splits * s.batch) break;
      if (i == kDecodeDealt - 1) return hipErrorInvalidValue;   // the last candidate always fits
    }
    dealt_chunk = c * kDecodeUnit;
    for (int b = 0; b < s.batch; ++b) mine[b] = ceil_div(u[b], c);
  }
  for (int b = 0; b < s.batch; ++b) first[b + 1] = first[b] + mine[b];
  const int n_rep = s.n_q_heads / s.n_kv_heads;
  for (int l = 0; l < s.n_layers; ++l)
    for (int b = 0; b < s.batch; ++b)
      for (int g = 0; g < s.n_kv_heads; ++g) {
        const Stream st(a, 2, l, b, g);
        if (st.n_tok == 0) continue;
        st.turn(st.ctx);
        const int64_t chunk =
            dealt_chunk ? dealt_chunk : (int64_t)decode_units(ceil_div(st.ctx + 1, a.n_splits)) * kDecodeUnit;
        for (int split = 0; split < mine[b]; ++split) {
          const int n_vis = st.ctx + 1;
          const int wc0 = (int)std::min((int64_t)split * chunk, (int64_t)n_vis);
          const int wc1 = (int)std::min((int64_t)wc0 + chunk, (int64_t)n_vis);
          st.keys(wc0, wc1);
          if (st.ctx >= wc0 && st.ctx < wc1) st.store(0);
          for (int h = g * n_rep; h < (g + 1) * n_rep; ++h) {
            rd(a.q, st.q_row(0, h), st.rb());
            if (mine[b] == 1) {
              wr(a.out, st.q_row(0, h), st.rb());
            } else {
              const int64_t slot = ((int64_t)l * s.batch * a.n_splits + first[b]) * s.n_q_heads + (int64_t)h * mine[b] + split;
              wr(ws_o, slot, (int64_t)s.head_dim * 4);
              wr(ws_ml, slot, 8);
            }
          }
        }
        if (mine[b] > 1)
          for (int h = g * n_rep; h < (g + 1) * n_rep; ++h) wr(a.out, st.q_row(0, h), st.rb());
      }
  return hipSuccess;
}

namespace {
// A bf16 suffix call: request b's keys in splits_of(b) equal ranges, whole units of `unit` each.
template <typename S, typename F, typename G>
hipError_t walk_suffix(const PageAttnArgs& a, S splits_of, int unit, F partial, G combined) {
  ++emu::launches;
  const AttnShape& s = a.s;
  const int n_rep = s.n_q_heads / s.n_kv_heads;
  for (int l = 0; l < s.n_layers; ++l)
    for (int b = 0; b < s.batch; ++b)
      for (int g = 0; g < s.n_kv_heads; ++g) {
        const Stream st(a, 2, l, b, g);
        if (st.n_tok == 0) continue;
        const int n_vis = st.ctx + st.n_tok;
        const int splits = splits_of(b);
        if (splits < 1) return hipErrorInvalidValue;
        const int64_t chunk = (int64_t)ceil_div(ceil_div(n_vis, unit), splits) * unit;
        for (int sp = 0; sp < splits; ++sp) {
          const int wc0 = (int)std::min(sp * chunk, (int64_t)n_vis), wc1 = (int)std::min(wc0 + chunk, (int64_t)n_vis);
          st.keys(wc0, wc1);
          for (int i = 0; i < st.n_tok; ++i)
            for (int h = g * n_rep; h < (g + 1) * n_rep; ++h) partial(l, b, i, h, st, sp);
        }
        for (int i = 0; i < st.n_tok; ++i) {
          st.store(i);
          st.turn(st.ctx + i);
          for (int h = g * n_rep; h < (g + 1) * n_rep; ++h) {
            rd(a.q, st.q_row(i, h), st.rb());
            combined(l, b, i, h, st);
            wr(a.out, st.q_row(i, h), st.rb());
          }
        }
      }
  return hipSuccess;
}
}  // namespace

hipError_t launch_few_bf16_pages(const PageAttnArgs& a) {
  const AttnShape& s = a.s;
  const int n = few_bf16_splits(s, a.n_new, a.max_base, a.workspace ? a.ws_bytes : 0);
  const int64_t rows = (int64_t)s.n_layers * s.batch * a.n_new * s.n_q_heads;
  float* ws_o = static_cast<float*>(a.workspace);
  float* ws_ml = n > 1 ? ws_o + rows * n * s.head_dim : nullptr;
  return walk_suffix(a, [&](int) { return n; }, kDecodeUnit, [&](int, int, int i, int h, const Stream& st, int sp) {
    if (n == 1) return;
    wr(ws_o, st.q_row(i, h) * n + sp, (int64_t)s.head_dim * 4);
    wr(ws_ml, st.q_row(i, h) * n + sp, 8);
  }, [](int, int, int, int, const Stream&) {});
}

hipError_t launch_prefill_bf16_pages(const PageAttnArgs& a) {
  const AttnShape& s = a.s;
  const SplitPlan p = plan_prefill_splits(s, a.n_new, a.max_base, a.workspace ? a.ws_bytes : 0);
  const int64_t rows = (int64_t)s.n_layers * s.batch * a.n_new * s.n_q_heads;
  const int64_t part = (int64_t)s.head_dim * (p.f32_partials ? 4 : 2);
  uint8_t* ws_o = static_cast<uint8_t*>(a.workspace);
  std::vector<int32_t> n(s.batch, p.n_splits), first(s.batch, 0);
  bool dealt = suffix_dealt(p.n_splits, s.batch);
  if (dealt) {
    const int n_rep = s.n_q_heads / s.n_kv_heads;
    std::vector<int32_t> u(s.batch, 0), t(s.batch), m(s.batch);
    int64_t total = 0;
    int32_t longest = 0, c = 0;
    for (int b = 0; b < s.batch; ++b) {
      t[b] = page_new_tokens(a.base_len, a.n_valid, b, a.n_new);
      m[b] = ceil_div(t[b] * n_rep, kPrefillRowsPerWG);
      if (t[b] > 0) u[b] = ceil_div(clamp_len(a.base_len[b], a.max_base) + t[b], kPrefillKeys);
      total += (int64_t)u[b] * m[b];
      longest = std::max(longest, u[b]);
    }
    if (longest == 0) {
      ++emu::launches;
      return hipSuccess;
    }
    const RangeCandidates rc = suffix_range_candidates(total, longest, p.n_splits, s.batch * p.m_tiles);
    for (int i = 0; i < kDecodeDealt; ++i) {
      c = rc.at(i);
      int64_t wgs = 0, parts = 0;
      for (int b = 0; b < s.batch; ++b) {
        n[b] = ceil_div(u[b], c);
        wgs += (int64_t)n[b] * m[b];
        parts += (int64_t)n[b] * t[b];
      }
      if (wgs <= (int64_t)p.n_splits * s.batch * p.m_tiles && parts <= (int64_t)p.n_splits * s.batch * a.n_new) break;
      if (i == kDecodeDealt - 1) return hipErrorInvalidValue;   // the last candidate always fits
    }
    dealt = suffix_deal_pays(c, rc.top);
    if (!dealt) n.assign(s.batch, p.n_splits);
    for (int b = 1; b < s.batch; ++b) first[b] = first[b - 1] + n[b - 1] * t[b - 1];
  }
  // a row's partial of range sp
  auto slot = [&](int l, int b, int i, int h, const Stream& st, int sp) {
    if (!dealt) return sp * rows + st.q_row(i, h);
    return ((int64_t)l * p.n_splits * s.batch * a.n_new + first[b] + (int64_t)sp * st.n_tok + i) * s.n_q_heads + h;
  };
  return walk_suffix(a, [&](int b) { return n[b]; }, kPrefillKeys,
                     [&](int l, int b, int i, int h, const Stream& st, int sp) {
    if (n[b] == 1) return;
    wr(ws_o, slot(l, b, i, h, st, sp), part);
    wr(ws_o + p.n_splits * rows * part, slot(l, b, i, h, st, sp), 8);
  }, [&](int l, int b, int i, int h, const Stream& st) {
    for (int sp = 0; n[b] > 1 && sp < n[b]; ++sp) rd(ws_o, slot(l, b, i, h, st, sp), part);
  });
}

}  // namespace pic
