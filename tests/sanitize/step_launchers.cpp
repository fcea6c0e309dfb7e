// CPU emulation of the launches of page_shared.hip, page_grow.hip and qk_norm.hip, for the sanitizer build of the host library
// (see emulated_launchers.cpp): every row, table entry, partial and workspace entry that a kernel addresses, found with its
// own clamping helpers and touched in host memory.
#include <algorithm>
#include <cstring>
#include <vector>

#include "pic_internal.h"

namespace pic {
namespace emu {
extern long launches;
}

namespace {

void rd(const void* base, int64_t at, int64_t bytes) {
  const volatile uint8_t* p = static_cast<const uint8_t*>(base) + at;
  (void)p[0];
  (void)p[bytes - 1];
}
void wr(void* base, int64_t at, int64_t bytes) {
  uint8_t* p = static_cast<uint8_t*>(base) + at;
  p[0] = 0;
  p[bytes - 1] = 0;
}

}  // namespace

hipError_t launch_shared_bf16_pages(const PageAttnArgs& a, const SharedMap& m, const SharedPlan& plan) {
  ++emu::launches;
  const AttnShape& s = a.s;
  const int n_rep = s.n_q_heads / s.n_kv_heads, parts = plan.prefix_splits + plan.own_splits;
  const int64_t rb = (int64_t)s.head_dim * 2;
  float* ws_ml = static_cast<float*>(a.workspace) + (size_t)s.n_layers * s.batch * a.n_new * s.n_q_heads * parts * s.head_dim;
  for (int l = 0; l < s.n_layers; ++l)
    for (int64_t block = 0; block < plan.prefix_blocks + plan.own_blocks; ++block) {
      const bool prefix = block < plan.prefix_blocks;
      const int64_t at = prefix ? block : block - plan.prefix_blocks;
      const int ROWS = prefix ? 64 * plan.row_blocks : 64;
      const int row_tiles = prefix ? plan.prefix_row_tiles : plan.own_row_tiles, splits = prefix ? plan.prefix_splits : plan.own_splits;
      const int rt = at / 8 % row_tiles;
      const int64_t range = at / 8 / row_tiles * 8 + at % 8;
      const int split = range % splits, g = range / splits % s.n_kv_heads, owner = (int)(range / splits / s.n_kv_heads), row0 = rt * ROWS;
      if (owner >= (prefix ? m.n_groups : s.batch)) continue;
      int b0 = owner, n_rows, k0, k1, ctx = INT32_MAX, n_tok = 0, gi = owner;
      if (prefix) {
        b0 = m.first(owner);
        n_rows = std::min(m.requests(owner) * a.n_new * n_rep - row0, ROWS);
        if (n_rows <= 0) continue;
        const int tiles = m.slots(owner) / kSharedKeys, per = ceil_div(tiles, splits);
        k0 = std::min(split * per, tiles) * kSharedKeys;
        k1 = std::min(split * per + per, tiles) * kSharedKeys;
      } else {
        n_tok = page_new_tokens(a.base_len, a.n_valid, b0, a.n_new);
        n_rows = std::min(n_tok * n_rep - row0, ROWS);
        if (n_rows <= 0) continue;
        ctx = clamp_len(a.base_len[b0], a.max_base) + a.offset;
        gi = m.group_of(b0);
        const int from = gi < 0 ? 0 : shared_part(m.slots(gi), ctx), end = ctx + n_tok;
        const int tiles = ceil_div(end - from, kSharedKeys), per = ceil_div(tiles, splits);
        k0 = from + std::min(split * per, tiles) * kSharedKeys;
        k1 = std::min(from + std::min(split * per + per, tiles) * kSharedKeys, end);
      }
      for (int r = row0; r < row0 + n_rows; ++r) {
        const int per_request = prefix ? a.n_new * n_rep : INT32_MAX;
        const int b = b0 + r / per_request, in_b = r % per_request, tok = in_b / n_rep;
        const int64_t row = (((int64_t)l * s.batch + b) * a.n_new + tok) * s.n_q_heads + g * n_rep + (in_b - tok * n_rep);
        int lim;
        if (!prefix) lim = std::min(k1, ctx + tok + 1);
        else if (tok >= page_new_tokens(a.base_len, a.n_valid, b, a.n_new)) lim = -1;
        else lim = std::min(k1, shared_part(k1, clamp_len(a.base_len[b], a.max_base) + a.offset));
        if (lim < 0) continue;
        rd(a.q, row * rb, rb);
        const int first = prefix ? split : gi < 0 && split == 0 ? 0 : plan.prefix_splits + split;
        for (int p = first; p <= (prefix ? split : plan.prefix_splits + split); ++p) {
          wr(a.workspace, (row * parts + p) * s.head_dim * 4, s.head_dim * 4);
          wr(ws_ml, (row * parts + p) * 8, 8);
        }
      }
      const int k_end = prefix ? k1 : std::min(k1, ctx + (row0 + n_rows - 1) / n_rep + 1), tab = std::min(b0, s.batch - 1);
      const int64_t stream0 = ((int64_t)l * s.n_kv_heads + g) * s.cache_cap;
      for (int wave = 0; wave < 4; ++wave) {
        const int win = std::min(k0 + 16 * wave, std::max(k_end - 1, 0) & ~15) >> a.map.shift;
        for (int j = 0; j < 128; ++j) rd(a.map.table, ((int64_t)tab * a.map.cap + clamp_entry(win + j, a.map)) * 4, 4);
      }
      for (int key = k0; key < k_end; ++key)
        for (int kv = 0; kv < 2; ++kv) {
          if (key < ctx) rd(kv ? a.pages_v : a.pages_k, (stream0 + page_row(a.map, tab, key)) * rb, rb);
          else rd(kv ? a.v_new : a.k_new, ((((int64_t)l * s.batch + tab) * a.n_new + key - ctx) * s.n_kv_heads + g) * rb, rb);
        }
      if (!prefix && row0 == 0)
        for (int i = std::max(k0 - ctx, 0); i < std::min(k1 - ctx, n_tok); ++i) {
          const int64_t row = page_store_row(a.map, b0, ctx + i);
          if (row < 0) continue;
          wr(a.pages_k, (stream0 + row) * rb, rb);
          wr(a.pages_v, (stream0 + row) * rb, rb);
          rd(a.k_new, ((((int64_t)l * s.batch + b0) * a.n_new + i) * s.n_kv_heads + g) * rb, rb);
        }
    }
  // the combine
  for (int64_t row = 0; row < (int64_t)s.n_layers * s.batch * a.n_new * s.n_q_heads; ++row) {
    const int b = (int)(row / ((int64_t)a.n_new * s.n_q_heads) % s.batch), tok = (int)(row / s.n_q_heads % a.n_new);
    for (int p = 0; p < parts; ++p) {
      rd(a.workspace, (row * parts + p) * s.head_dim * 4, s.head_dim * 4);
      rd(ws_ml, (row * parts + p) * 8, 8);
    }
    if (tok < page_new_tokens(a.base_len, a.n_valid, b, a.n_new)) wr(a.out, row * rb, rb);
  }
  return hipSuccess;
}

hipError_t launch_qk_norm(pic_dtype dt, int head_dim, bool, int n_layers, QkNormArgs a, hipStream_t) {
  ++emu::launches;
  const int64_t es = dt == PIC_F32 ? 4 : 2, rb = head_dim * es;
  for (int l = 0; l < n_layers; ++l)
    for (int b = 0; b < a.batch; ++b)
      for (int i = 0; i < a.n_new; ++i) {
        int n_tok = a.n_new;
        int64_t pos = a.offset + i;
        if (a.base_len) {
          n_tok = page_new_tokens(a.base_len, a.n_valid, b, a.n_new);
          pos += clamp_len(a.base_len[b], a.max_base);
        } else if (a.n_valid) {
          n_tok = clamp_len(a.n_valid[b], a.n_new);
        }
        if (i >= n_tok) continue;
        const int64_t tok = ((int64_t)l * a.batch + b) * a.n_new + i;
        if (a.table) rd(a.table + l * a.table_stride, pos * (head_dim / 2) * 8, head_dim / 2 * 8);
        auto rows = [&](const void* in, void* out, int64_t stride, int heads, const float* w) {
          for (int h = 0; in && h < heads; ++h) {
            rd(in, (tok * stride + (int64_t)h * head_dim) * es, rb);
            wr(out, (tok * heads + h) * rb, rb);
            if (w) rd(w, (int64_t)l * head_dim * 4, head_dim * 4);
          }
        };
        rows(a.q, a.q_out, a.q_stride, a.n_q_heads, a.q_weight);
        rows(a.k, a.k_out, a.k_stride, a.n_kv_heads, a.k_weight);
        rows(a.v, a.v_out, a.v_stride, a.n_kv_heads, nullptr);
      }
  return hipSuccess;
}

// The kernel's steps one entry after another, its arrays in the same places of the workspace.
hipError_t launch_page_grow(const PageGrowArgs& a, hipStream_t) {
  ++emu::launches;
  const int32_t P = 1 << a.shift;
  const int64_t cap = page_grow_entries(P, a.table_cap, a.batch, a.n_new);
  int32_t *first = a.workspace, *shared = first + a.batch + 1, *at = shared + cap, *take = at + cap, *lowest = take + cap;
  bool bad_cap = false, bad_entry = false;
  int32_t entries = 0;
  std::vector<int32_t> req, place;
  std::vector<bool> partly;
  for (int b = 0; b < a.batch; ++b) {
    first[b] = entries;
    const int64_t from = (int64_t)a.base_len[b] + a.offset, to = from + page_new_tokens(a.base_len, a.n_valid, b, a.n_new);
    if (to <= from) continue;
    const int64_t end = (to + P - 1) >> a.shift;
    if (end > a.table_cap) {
      bad_cap = true;
      continue;
    }
    for (int64_t i = from >> a.shift; i < end; ++i) {
      req.push_back(b);
      place.push_back((int32_t)i);
      partly.push_back(i == from >> a.shift && (from & (P - 1)) != 0);
    }
    entries = (int32_t)req.size();
  }
  first[a.batch] = entries;
  int32_t n_shared = 0, takes = 0, copies = 0;
  for (int e = 0; !bad_cap && e < entries; ++e) {
    const int32_t page = a.page_table[(int64_t)req[e] * a.table_cap + place[e]];
    take[e] = 0;
    if (page == -1 && !partly[e]) take[e] = 1;
    else if (page < 0 || page >= a.n_pages || a.refs[page] < 1) bad_entry = true;
    else if (a.refs[page] > 1) {
      shared[n_shared] = page;
      at[n_shared++] = e;
    }
  }
  bool fits = !bad_cap && !bad_entry;
  const bool known = fits;
  if (fits) {
    for (int i = 0; i < n_shared; ++i)
      if (a.refs[shared[i]] - std::count(shared, shared + i, shared[i]) > 1) take[at[i]] = partly[at[i]] ? 3 : 1;
    for (int e = 0; e < entries; ++e) takes += take[e] != 0;
    int32_t found = 0;
    for (int32_t p = 0; p < a.n_pages && found < takes; ++p)
      if (a.refs[p] == 0) lowest[found++] = p;
    fits = found >= takes;
  }
  int32_t k = 0;
  for (int e = 0; fits && e < entries; ++e) {
    if (take[e] == 0) continue;
    int32_t* entry = a.page_table + (int64_t)req[e] * a.table_cap + place[e];
    if (*entry >= 0) --a.refs[*entry];
    if (take[e] == 3) {
      a.pairs[2 * copies] = *entry;
      a.pairs[2 * copies++ + 1] = lowest[k];
    }
    a.refs[lowest[k]] = 1;
    *entry = lowest[k++];
  }
  for (int64_t i = 2 * (int64_t)copies; i < 2 * (int64_t)a.batch; ++i) a.pairs[i] = -1;
  for (int b = 0; b < a.batch; ++b) a.ready[b] = fits && a.base_len[b] >= 0 ? a.base_len[b] : -1;
  a.result[0] = fits ? PIC_OK : bad_cap || known ? PIC_ERR_CAPACITY : PIC_ERR_RANGE;
  a.result[1] = copies;
  a.result[2] = known ? takes : 0;
  return hipSuccess;
}

hipError_t launch_page_copy_listed(void* pages_k, void* pages_v, int64_t n_streams, int64_t n_pages, int64_t page_bytes,
                                   const int32_t* pairs, int32_t cap, hipStream_t) {
  ++emu::launches;
  for (int32_t i = 0; i < cap; ++i) {
    const int32_t x = pairs[2 * i], y = pairs[2 * i + 1];
    if (x < 0 || x >= n_pages || y < 0 || y >= n_pages) continue;
    for (int64_t st = 0; st < n_streams; ++st)
      for (void* p : {pages_k, pages_v}) {
        rd(p, (st * n_pages + x) * page_bytes, page_bytes);
        wr(p, (st * n_pages + y) * page_bytes, page_bytes);
      }
  }
  return hipSuccess;
}

}  // namespace pic
