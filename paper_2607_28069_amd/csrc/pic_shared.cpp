// C ABI of libpic, attention of new tokens over pages for batches that share prefixes: checks, launch planning, dispatch.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "pic.h"
#include "pic_check.h"
#include "pic_internal.h"

namespace pic {

namespace {

int64_t ceil_of(int64_t n, int64_t d) { return (n + d - 1) / d; }

// The time of a launch, in tiles of 64 keys of a workgroup that has a compute unit to itself (about 1.2 us).  512 workgroups
// run at once, the prefixes' before the requests' own; two on a compute unit slow each other down, and a workgroup's
// start (lengths, page numbers, first tile) costs about 3 tiles.  Requests of no group are the last of the batch, at worst.
struct LaunchCost {
  int64_t prefix_units, own_units, lone_units;   // workgroups per key range; lone: those of requests of no group, among own
  int64_t own_tiles, lone_tiles;                 // of a request of a group, and of one of none
  double both, join;                             // a tile where compute units hold two; a part's share of the combine

  double operator()(int64_t prefix_tiles, int64_t prefix_splits, int64_t own_splits) const {
    constexpr double kStart = 3.0;
    const int64_t P = prefix_units * prefix_splits;
    const int64_t rest = P % 512;
    double t = (double)prefix_tiles * ((double)(P / 512) * both + (rest == 0 ? 0.0 : rest <= 256 ? 1.0 : both)) + kStart * (double)((P + 511) / 512);
    const int64_t beside = P < 512 ? 512 - P : 0, O = own_units * own_splits;
    const double own = (double)ceil_of(own_tiles, own_splits) + kStart;
    if (O <= beside) t = std::max(t, own);
    else t += own * (double)((std::max<int64_t>(0, O - beside * (int64_t)(t / own)) + 511) / 512);
    if (lone_units > 0) {   // (the last ones to start: as short ranges leave their places, or after all else)
      const int64_t lone = lone_units * own_splits;
      const double each = (double)ceil_of(lone_tiles, own_splits) + kStart;
      if (lone <= beside) t = std::max(t, own * (double)std::max<int64_t>(0, O - beside) / (double)beside + each);
      else t += each * (double)ceil_of(lone, 512);
    }
    return t + join * (double)(prefix_splits + own_splits);
  }
};

// Workgroups of requests' own ranges, at most, where some requests are in no group: most of them then find nothing to do.
constexpr int64_t kLoneBlocks = 4096;

}  // namespace

// Key ranges of a launch: as many as cover some or all compute units, or up to twice, whichever the estimate above puts first
// (few where a prefix is short and its rows many, as each range writes a part of every row, which the combine reads), requests'
// own ranges filling what is left.  Measured, us by ranges of the prefix (head_dim 128, 8 kv heads):
// 64 requests over 16K + 300 own (16 workgroups a range) 12: 54.6, 16: 47.8, 24: 52.3, 32: 58.1; 16 over 10K (8) 20: 21.3, 28:
// 19.1, 40: 22.0; 16 x 24 tokens over 10K (96) 2: 143, 4: 92, 5: 86, 8: 107; 4 groups of up to 32K (16) 16: 68, 24: 62, 28: 57,
// 32: 63 (at head_dim 64, or with 64 rows at most, such a share of the second place on every compute unit loses 1 to 2 us); 12 x 5
// tokens at head_dim 64 (48) 5: 35, 8: 29, 11: 33; 32 over 2K (8) 31: 17.9, 16: 18.0, 8: 19.8; 4 x 4 tokens over 2K (8) 31: 15.3, 16:
// 12.8; 16 over 2K (8) 31: 14.5, 16: 12.7.
SharedPlan plan_shared(const AttnShape& s, const SharedMap& m, int32_t n_new, int32_t max_ctx) {
  SharedPlan p;
  const int64_t n_rep = s.n_q_heads / s.n_kv_heads;
  const int64_t own_rows = n_new * n_rep, group_rows = m.max_group * own_rows;
  p.row_blocks = group_rows > 64 ? 2 : 1;
  // Probabilities in two bfloat16 terms wherever the calls that this one takes the place of keep 16 bits (pic_page_decode_attn;
  // pic_page_suffix_attn up to 32 rows), whatever max_group is.  One term of 8 bits / two, us: 64 requests over 16K 43.9 / 48.7, 4
  // groups of up to 32K 51.5 / 56.2, 12 x 5 tokens at head_dim 64 24.4 / 29.2, errors against 64 bits 0.0024 / 0.0017, 0.0015 /
  // 0.0011, 0.0017 / 0.0012 (those of the output's own rounding).  Past that products bound the call: 16 x 24 tokens over 10K
  // 78.7 / 103.6, 0.0024 / 0.0017, the first as in a prefill.
  p.prefix_terms = group_rows > 64 && own_rows > 32 ? 1 : 2;
  p.prefix_row_tiles = (int32_t)ceil_of(group_rows, 64 * p.row_blocks);
  p.own_row_tiles = (int32_t)ceil_of(own_rows, 64);
  const int64_t prefix_tiles = std::min(m.max_len, max_ctx) / kSharedKeys;
  const int64_t all_tiles = ceil_of((int64_t)max_ctx + n_new, kSharedKeys), own_tiles = all_tiles - prefix_tiles;
  // Requests that no group has room for: all of their slots are their own, and are split as such (4 requests of 32K, 2 of them
  // a group, 581 us with one range each, 70 so; 8 of 10K, 4 a group, 102 -> 43; 33 of 32K, 4 groups of 8, 660 -> 161;
  // pic_page_decode_attn 69, 45, 452).  How much less than max_len a group shares is not known here.
  const int64_t lone = std::max<int64_t>(0, s.batch - (int64_t)m.n_groups * m.max_group);
  const int64_t heads = (int64_t)s.n_kv_heads * s.n_layers;
  const int64_t prefix_units = m.n_groups * heads * p.prefix_row_tiles, own_units = s.batch * heads * p.own_row_tiles;
  const int64_t rows = (int64_t)s.n_layers * s.batch * n_new * s.n_q_heads, part_bytes = rows * (s.head_dim + 2) * (int64_t)sizeof(float);
  // (groups are rarely of one size: of the row tiles that the grid has room for, about as many as the batch fills)
  const int64_t row_tiles = std::min<int64_t>((int64_t)m.n_groups * p.prefix_row_tiles,
                                              s.batch * own_rows / (64 * p.row_blocks) + m.n_groups);
  LaunchCost cost;
  cost.prefix_units = heads * row_tiles;
  cost.own_units = own_units;
  cost.lone_units = lone * heads * p.own_row_tiles;
  cost.own_tiles = own_tiles;
  cost.lone_tiles = all_tiles;
  // (bound by the loads, which one workgroup with tiles of half the size does not keep busy, or by products)
  cost.both = p.row_blocks == 2 ? 1.7 : s.head_dim == 64 ? 1.3 : 2.0;
  cost.join = (double)part_bytes * 2.0 / 5.8e6;   // (written and read, 4.8 TB/s)
  double best = 1e30;
  auto consider = [&](int64_t n, double least) {   // n key ranges of the prefix
    int64_t tiles = 0;
    if (prefix_tiles > 0 && prefix_units > 0) {
      tiles = ceil_of(prefix_tiles, std::min({n, prefix_tiles, (int64_t)kSharedMaxSplits}));
      n = ceil_of(prefix_tiles, tiles);
    } else {
      n = 0;
    }
    const int64_t left = 512 - std::min<int64_t>(512, cost.prefix_units * n);
    const int64_t beside = std::max<int64_t>(1, std::min({left / own_units, (own_tiles + 1) / 2, (int64_t)kSharedMaxSplits}));
    const int64_t most = lone > 0 ? std::min({kLoneBlocks / own_units, (all_tiles + 1) / 2, (int64_t)kSharedMaxSplits}) : 0;
    for (int64_t o = beside;; o = std::min(2 * o, most)) {
      const double c = cost(tiles, n, o);
      if (c < least * best) {
        best = c;
        p.prefix_splits = (int32_t)n;
        p.own_splits = (int32_t)o;
      }
      if (o >= most) break;
    }
  };
  for (const int64_t fill : {32, 64, 96, 128, 192, 256, 384, 448, 512}) {
    if (fill < 384 && m.n_groups > 1) continue;   // (nor of one length: longer ones need company)
    if (fill == 448 && (p.row_blocks == 1 || s.head_dim == 64)) continue;
    consider(std::max<int64_t>(1, fill / std::max<int64_t>(1, cost.prefix_units)), 1.0);
  }
  // Far fewer ranges where the estimate, which is off by a quarter at times, leaves no doubt: rows so many that their parts cost more
  // than the prefix.  4096 requests of 100 slots and 2 of them over 2K, 8 heads on 1 of 128: 305 -> 113 us, with 8 tokens each 1900
  // -> 223; 62 over 349 slots 20.2 -> 14.8; 2 and 4 groups of uneven prefixes 23 to 29 -> 19 to 24; at worst 22.9 -> 24.8.
  for (const int64_t n : {16, 8, 4, 2, 1})
    if (n * cost.prefix_units <= 512) consider(n, 0.75);
  auto blocks = [](int64_t ranges, int64_t row_tiles) { return ceil_of(ranges, 8) * 8 * row_tiles; };   // (whole rounds of the XCDs)
  p.prefix_blocks = blocks((int64_t)m.n_groups * s.n_kv_heads * p.prefix_splits, p.prefix_row_tiles);
  p.own_blocks = blocks((int64_t)s.batch * s.n_kv_heads * p.own_splits, p.own_row_tiles);
  // Rows that the last-level cache (256 MB) will not hold until the next call leave it to others (8 requests x 33K in 4
  // groups 60 -> 55 us, 64 requests of up to 2K of their own 72 -> 63; below, 16 over 10K 19.5 -> 21.2).
  const double tiles_read = (double)m.n_groups * prefix_tiles + (double)(s.batch - lone) * own_tiles + (double)lone * all_tiles;
  p.stream = p.prefix_row_tiles <= 1 && heads * s.head_dim * 4.0 * tiles_read * kSharedKeys > 256e6;
  // Room for every call of these groups with no more requests, tokens and slots, so that a buffer for the largest serves all.
  // Parts of prefixes: max(1, 512 / prefix_units) ranges of R = heads * batch * own_rows rows, where prefix_units / heads is at
  // least 1, batch * own_rows / 128, or n_groups * max_group * own_rows / 128.  Of requests: max(1, 512 / own_units), with some in
  // no group kLoneBlocks / own_units, where own_units / heads is at least batch, or batch * own_rows / 64.
  const int64_t grouped = (int64_t)m.n_groups * m.max_group;
  int64_t most = 0;
  if (prefix_tiles > 0 && grouped > 0)
    most = std::max(rows, std::min({65536 * ceil_of(s.batch, grouped), (int64_t)512 * s.batch * own_rows, rows * std::min<int64_t>(prefix_tiles, kSharedMaxSplits)}));
  most += std::max(rows, std::min((lone > 0 ? kLoneBlocks : 512) * std::min<int64_t>(64, own_rows), rows * std::min<int64_t>((all_tiles + 1) / 2, kSharedMaxSplits)));
  p.ws_bytes = (size_t)most * (s.head_dim + 2) * sizeof(float);
  return p;
}

}  // namespace pic

using namespace pic;

namespace {

// Slots of a request that attention reads: positions rounded up to a workgroup's tile stay in 31 bits.
constexpr int64_t kMaxSlots = int64_t(1) << 30;

pic_status check_shared(const pic_shared* sh) {
  if (sh == nullptr) return fail(PIC_ERR_INVALID_ARG, "shared is NULL");
  if (sh->n_groups < 1 || sh->max_group < 0 || sh->max_len < 0)
    return fail(PIC_ERR_INVALID_ARG, "n_groups < 1, or max_group or max_len < 0");
  return PIC_OK;
}

// The sizes of a call whose new tokens come after `max_ctx` slots at most, and its plan.
pic_status check_sizes(const pic_model* m, const pic_shared* sh, int32_t batch, int32_t n_new, int64_t max_ctx, SharedMap* groups,
                       SharedPlan* plan) {
  if (batch < 0 || n_new < 0 || max_ctx < 0) return fail(PIC_ERR_INVALID_ARG, "negative size");
  if (max_ctx + n_new > kMaxSlots) return fail(PIC_ERR_CAPACITY, "%lld slots per request (at most 2^30)", (long long)max_ctx + n_new);
  if (sh->n_groups >= 1 << 24) return fail(PIC_ERR_UNSUPPORTED, "too many groups");
  if ((double)batch * m->n_q_heads * n_new * std::max(m->n_layers, 1) >= (double)(1 << 27)) return fail(PIC_ERR_UNSUPPORTED, "too many query rows");
  if ((int64_t)n_new * m->n_kv_heads >= (int64_t(1) << 24)) return fail(PIC_ERR_UNSUPPORTED, "too many new tokens per request");
  if (m->n_layers > 65535) return fail(PIC_ERR_UNSUPPORTED, "more than 65535 layers");
  groups->n_groups = sh->n_groups;
  groups->max_group = std::min(sh->max_group, batch);
  groups->max_len = sh->max_len;
  groups->batch = batch;
  if (batch == 0 || n_new == 0 || m->n_layers == 0 || m->dtype != PIC_BF16) return PIC_OK;
  *plan = plan_shared(shape_of(m, batch, 0, 0.f), *groups, n_new, (int32_t)max_ctx);
  if (plan->prefix_blocks + plan->own_blocks >= (int64_t(1) << 24)) return fail(PIC_ERR_UNSUPPORTED, "too many workgroups");
  return PIC_OK;
}

pic_status shared_attn(const pic_model* model, const pic_pages* pages, const pic_shared* shared, const void* q, const void* k_new,
                       const void* v_new, void* pages_k, void* pages_v, const int32_t* page_table, int32_t batch,
                       const int32_t* group_start, const int32_t* shared_len, const int32_t* base_len, int32_t max_base,
                       int32_t offset, const int32_t* n_valid, int32_t n_new, float scale, bool decode, void* out, void* workspace,
                       size_t ws_bytes, void* stream) {
  PIC_CHECK(check_model(model));
  PIC_CHECK(check_pages(pages));
  PIC_CHECK(check_shared(shared));
  if (max_base < 0 || offset < 0) return fail(PIC_ERR_INVALID_ARG, "negative size");
  if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(PIC_ERR_INVALID_ARG, "scale must be finite and >= 0");
  SharedMap groups;
  SharedPlan plan;
  PIC_CHECK(check_sizes(model, shared, batch, n_new, (int64_t)max_base + offset, &groups, &plan));
  const int64_t max_len = (int64_t)max_base + offset + n_new;
  if (std::max<int64_t>(max_len, shared->max_len) > (int64_t)pages->table_cap * pages->page_tokens)
    return fail(PIC_ERR_CAPACITY, "%lld slots per request exceed a page table of %d pages of %d tokens",
                (long long)std::max<int64_t>(max_len, shared->max_len), pages->table_cap, pages->page_tokens);
  if (batch == 0 || n_new == 0 || model->n_layers == 0) return ok();
  if (pages->n_pages == 0) return fail(PIC_ERR_RANGE, "no pages");
  PIC_CHECK(check_ptr(q, "q"));
  PIC_CHECK(check_ptr(k_new, decode ? "k_new" : "k_suf"));
  PIC_CHECK(check_ptr(v_new, decode ? "v_new" : "v_suf"));
  PIC_CHECK(check_ptr(pages_k, "pages_k"));
  PIC_CHECK(check_ptr(pages_v, "pages_v"));
  PIC_CHECK(check_ptr(out, "out"));
  if (!page_table) return fail(PIC_ERR_INVALID_ARG, "page_table is NULL");
  if (!base_len) return fail(PIC_ERR_INVALID_ARG, decode ? "base_len is NULL" : "ctx_len is NULL");
  if (!shared_len) return fail(PIC_ERR_INVALID_ARG, "shared_len is NULL");
  if (!group_start && shared->n_groups != 1) return fail(PIC_ERR_INVALID_ARG, "group_start is NULL, and there are %d groups", shared->n_groups);
  // Request by request: a long suffix is bound by the float32 matrix rate, whatever is read.  (A decode is not: 16 requests over 10K
  // take 210 us, where the shared bytes and the products are 18 each.)
  if (model->dtype == PIC_F32) {
    return decode ? pic_page_decode_attn(model, pages, q, k_new, v_new, pages_k, pages_v, page_table, batch, base_len, offset, max_base,
                                         scale, 0, out, workspace, ws_bytes, stream)
                  : pic_page_suffix_attn(model, pages, q, k_new, v_new, pages_k, pages_v, page_table, batch, base_len, max_base,
                                         n_valid, n_new, scale, out, workspace, ws_bytes, stream);
  }
  if (!workspace || ws_bytes < plan.ws_bytes)
    return fail(PIC_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu", plan.ws_bytes, workspace ? ws_bytes : (size_t)0);
  PIC_CHECK(check_ptr(workspace, "workspace"));
  groups.start = group_start;
  groups.len = shared_len;
  PageAttnArgs a;
  a.s = shape_of(model, batch, pages->n_pages * pages->page_tokens, scale);
  a.map.table = page_table;
  a.map.cap = pages->table_cap;
  a.map.n_pages = pages->n_pages;
  a.map.shift = __builtin_ctz((unsigned)pages->page_tokens);
  a.q = q;
  a.k_new = k_new;
  a.v_new = v_new;
  a.pages_k = pages_k;
  a.pages_v = pages_v;
  a.base_len = base_len;
  a.n_valid = n_valid;
  a.max_base = max_base;
  a.offset = offset;
  a.n_new = n_new;
  a.out = out;
  a.workspace = workspace;
  a.ws_bytes = plan.ws_bytes;
  a.stream = (hipStream_t)stream;
  return hip_status(launch_shared_bf16_pages(a, groups, plan), decode ? "shared decode launch" : "shared suffix launch");
}

}  // namespace

PIC_API size_t pic_page_shared_workspace_bytes(const pic_model* model, const pic_shared* shared, int32_t batch, int32_t n_new,
                                               int32_t max_ctx) {
  SharedMap groups;
  SharedPlan plan;
  if (check_model(model) != PIC_OK || check_shared(shared) != PIC_OK) return 0;
  if (check_sizes(model, shared, batch, n_new, max_ctx, &groups, &plan) != PIC_OK) return 0;
  return plan.ws_bytes;
}

PIC_API pic_status pic_page_shared_suffix_attn(const pic_model* model, const pic_pages* pages, const pic_shared* shared, const void* q,
                                               const void* k_suf, const void* v_suf, void* pages_k, void* pages_v,
                                               const int32_t* page_table, int32_t batch, const int32_t* group_start,
                                               const int32_t* shared_len, const int32_t* ctx_len, int32_t max_ctx,
                                               const int32_t* n_valid, int32_t n_suffix, float scale, void* out, void* workspace,
                                               size_t ws_bytes, void* stream) {
  return shared_attn(model, pages, shared, q, k_suf, v_suf, pages_k, pages_v, page_table, batch, group_start, shared_len, ctx_len,
                     max_ctx, 0, n_valid, n_suffix, scale, false, out, workspace, ws_bytes, stream);
}

PIC_API pic_status pic_page_shared_decode_attn(const pic_model* model, const pic_pages* pages, const pic_shared* shared, const void* q,
                                               const void* k_new, const void* v_new, void* pages_k, void* pages_v,
                                               const int32_t* page_table, int32_t batch, const int32_t* group_start,
                                               const int32_t* shared_len, const int32_t* base_len, int32_t step,
                                               int32_t max_base_len, float scale, void* out, void* workspace, size_t ws_bytes,
                                               void* stream) {
  return shared_attn(model, pages, shared, q, k_new, v_new, pages_k, pages_v, page_table, batch, group_start, shared_len, base_len,
                     max_base_len, step, nullptr, 1, scale, true, out, workspace, ws_bytes, stream);
}
