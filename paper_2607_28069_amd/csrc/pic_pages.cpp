// C ABI of libpic, paged caches: page bookkeeping on the host, page copies, and attention of new
// tokens over pages.  Every check runs before anything is enqueued; a failing call launches nothing.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <vector>

#include "pic.h"
#include "pic_check.h"
#include "pic_internal.h"

namespace pic {

pic_status check_pages(const pic_pages* pg) {
  if (pg == nullptr) return fail(PIC_ERR_INVALID_ARG, "pages is NULL");
  if (pg->n_pages < 0 || pg->table_cap < 0) return fail(PIC_ERR_INVALID_ARG, "n_pages or table_cap < 0");
  const int32_t p = pg->page_tokens;
  if (p < 16 || p > 1024 || (p & (p - 1)) != 0)
    return fail(PIC_ERR_UNSUPPORTED, "page_tokens %d (a power of two from 16 to 1024)", p);
  if ((int64_t)pg->n_pages * p > INT32_MAX)
    return fail(PIC_ERR_UNSUPPORTED, "%d pages of %d tokens: more than INT32_MAX rows", pg->n_pages, p);
  return PIC_OK;
}

}  // namespace pic

using namespace pic;

namespace {

// Slots of a request that attention reads: positions rounded up to a workgroup's tile stay in 31 bits.
constexpr int64_t kMaxSlots = int64_t(1) << 30;

int page_shift(int32_t page_tokens) { return __builtin_ctz((unsigned)page_tokens); }

// Host arrays of the bookkeeping calls.
pic_status check_table(const pic_pages* pg, int32_t batch, const void* refs, const void* page_table) {
  PIC_CHECK(check_pages(pg));
  if (batch < 0) return fail(PIC_ERR_INVALID_ARG, "batch < 0");
  if (!refs && pg->n_pages > 0) return fail(PIC_ERR_INVALID_ARG, "refs is NULL");
  if (!page_table && (int64_t)batch * pg->table_cap > 0) return fail(PIC_ERR_INVALID_ARG, "page_table is NULL");
  return PIC_OK;
}

pic_status check_request(int32_t request, int32_t batch, const char* name) {
  if (request < 0 || request >= batch) return fail(PIC_ERR_RANGE, "%s %d out of [0, %d)", name, request, batch);
  return PIC_OK;
}

int32_t pages_of(const pic_pages* pg, int32_t tokens) { return (int32_t)(((int64_t)tokens + pg->page_tokens - 1) / pg->page_tokens); }

pic_status bad_entry(int32_t b, int32_t i, int32_t page) {
  return fail(PIC_ERR_RANGE, "page table entry %d of request %d is %d: no page in use", i, b, page);
}

// Runs f, which may ask for host memory.
template <typename F>
pic_status with_memory(F f) {
  try {
    return f();
  } catch (const std::bad_alloc&) {
    return fail(PIC_ERR_CAPACITY, "out of host memory");
  }
}

}  // namespace

// ---------------------------------------------------------------------------------------------
// 5a. page bookkeeping
// ---------------------------------------------------------------------------------------------

PIC_API pic_status pic_page_grow(const pic_pages* pages, int32_t batch, int32_t* refs, int32_t* page_table,
                                 const int32_t* len, const int32_t* new_len, int32_t* pairs, int32_t pair_cap,
                                 int32_t* n_pairs) {
  PIC_CHECK(check_table(pages, batch, refs, page_table));
  if (!n_pairs) return fail(PIC_ERR_INVALID_ARG, "n_pairs is NULL");
  if (batch > 0 && (!len || !new_len)) return fail(PIC_ERR_INVALID_ARG, "len or new_len is NULL");
  if (pair_cap < 0 || (pair_cap > 0 && !pairs)) return fail(PIC_ERR_INVALID_ARG, "pairs is NULL, or pair_cap < 0");
  return with_memory([&]() -> pic_status {
    // what changes, first worked out on the side: entries that take a page, and the page each lets go of (-1: none)
    struct Take {
      int32_t b, i, old;
      bool copy;
    };
    std::vector<Take> takes;
    std::vector<int32_t> free_pages;
    int64_t most = 0;
    for (int32_t b = 0; b < batch; ++b) {
      if (len[b] < 0) return fail(PIC_ERR_INVALID_ARG, "len[%d] < 0", b);
      if (new_len[b] <= len[b]) continue;
      if (pages_of(pages, new_len[b]) > pages->table_cap)
        return fail(PIC_ERR_CAPACITY, "request %d needs %d pages, its table has room for %d", b, pages_of(pages, new_len[b]),
                    pages->table_cap);
      most += pages_of(pages, new_len[b]) - len[b] / pages->page_tokens;
    }
    takes.reserve(most);   // (nothing below asks for memory)
    free_pages.reserve(std::min(most, (int64_t)pages->n_pages));
    int32_t copies = 0;
    pic_status st = PIC_OK;
    for (int32_t b = 0; b < batch && st == PIC_OK; ++b) {
      if (new_len[b] <= len[b]) continue;
      const int32_t* row = page_table + (int64_t)b * pages->table_cap;
      for (int32_t i = len[b] / pages->page_tokens; i < pages_of(pages, new_len[b]); ++i) {
        const bool partly = i == len[b] / pages->page_tokens && len[b] % pages->page_tokens != 0;
        const int32_t page = row[i];
        if (page == -1 && !partly) {
          takes.push_back({b, i, -1, false});
          continue;
        }
        if (page < 0 || page >= pages->n_pages || refs[page] < 1) {
          st = bad_entry(b, i, page);
          break;
        }
        if (refs[page] == 1) continue;
        --refs[page];   // (so that the last of several sharers keeps it; undone below on failure)
        takes.push_back({b, i, page, partly});
        copies += partly;
      }
    }
    if (st == PIC_OK) {
      for (int32_t p = 0; p < pages->n_pages && free_pages.size() < takes.size(); ++p)
        if (refs[p] == 0) free_pages.push_back(p);
      if (free_pages.size() < takes.size())
        st = fail(PIC_ERR_CAPACITY, "%zu pages needed, %zu free", takes.size(), free_pages.size());
      else if (copies > pair_cap)
        st = fail(PIC_ERR_CAPACITY, "%d pairs needed, room for %d", copies, pair_cap);
    }
    if (st != PIC_OK) {
      for (const Take& t : takes)
        if (t.old >= 0) ++refs[t.old];
      return st;
    }
    int32_t n = 0;
    for (size_t k = 0; k < takes.size(); ++k) {
      const Take& t = takes[k];
      refs[free_pages[k]] = 1;
      page_table[(int64_t)t.b * pages->table_cap + t.i] = free_pages[k];
      if (t.copy) {
        pairs[2 * n] = t.old;
        pairs[2 * n + 1] = free_pages[k];
        ++n;
      }
    }
    *n_pairs = n;
    return ok();
  });
}

PIC_API pic_status pic_page_fork(const pic_pages* pages, int32_t batch, int32_t* refs, int32_t* page_table, int32_t src,
                                 int32_t len, int32_t dst) {
  PIC_CHECK(check_table(pages, batch, refs, page_table));
  PIC_CHECK(check_request(src, batch, "src"));
  PIC_CHECK(check_request(dst, batch, "dst"));
  if (src == dst) return fail(PIC_ERR_INVALID_ARG, "request %d cannot fork onto itself", src);
  if (len < 0) return fail(PIC_ERR_INVALID_ARG, "len < 0");
  const int32_t n = pages_of(pages, len);
  if (n > pages->table_cap) return fail(PIC_ERR_CAPACITY, "%d pages, the table has room for %d", n, pages->table_cap);
  const int32_t* from = page_table + (int64_t)src * pages->table_cap;
  int32_t* to = page_table + (int64_t)dst * pages->table_cap;
  for (int32_t i = 0; i < pages->table_cap; ++i)
    if (to[i] != -1) return fail(PIC_ERR_INVALID_ARG, "request %d still holds pages", dst);
  for (int32_t i = 0; i < n; ++i)
    if (from[i] < 0 || from[i] >= pages->n_pages || refs[from[i]] < 1) return bad_entry(src, i, from[i]);
  for (int32_t i = 0; i < n; ++i) {
    to[i] = from[i];
    ++refs[from[i]];
  }
  return ok();
}

PIC_API pic_status pic_page_free(const pic_pages* pages, int32_t batch, int32_t* refs, int32_t* page_table, int32_t request,
                                 int32_t keep_len) {
  PIC_CHECK(check_table(pages, batch, refs, page_table));
  PIC_CHECK(check_request(request, batch, "request"));
  if (keep_len < 0) return fail(PIC_ERR_INVALID_ARG, "keep_len < 0");
  int32_t* row = page_table + (int64_t)request * pages->table_cap;
  const int32_t first = pages_of(pages, keep_len);
  for (int32_t i = first; i < pages->table_cap; ++i)
    if (row[i] != -1 && (row[i] < 0 || row[i] >= pages->n_pages || refs[row[i]] < 1)) return bad_entry(request, i, row[i]);
  for (int32_t i = first; i < pages->table_cap; ++i) {
    if (row[i] != -1) --refs[row[i]];
    row[i] = -1;
  }
  return ok();
}

PIC_API pic_status pic_page_compact(const pic_pages* pages, int32_t batch, int32_t* refs, int32_t* page_table, int32_t* pairs,
                                    int32_t pair_cap, int32_t* n_pairs, int32_t* n_used) {
  PIC_CHECK(check_table(pages, batch, refs, page_table));
  if (!n_pairs || !n_used) return fail(PIC_ERR_INVALID_ARG, "n_pairs or n_used is NULL");
  if (pair_cap < 0 || (pair_cap > 0 && !pairs)) return fail(PIC_ERR_INVALID_ARG, "pairs is NULL, or pair_cap < 0");
  return with_memory([&]() -> pic_status {
    const int64_t entries = (int64_t)batch * pages->table_cap;
    std::vector<int32_t> held(pages->n_pages), to(pages->n_pages);   // references in the table; new number of each page
    for (int64_t i = 0; i < entries; ++i) {
      const int32_t p = page_table[i];
      if (p == -1) continue;
      if (p < 0 || p >= pages->n_pages || refs[p] < 1)
        return bad_entry((int32_t)(i / pages->table_cap), (int32_t)(i % pages->table_cap), p);
      ++held[p];
    }
    int32_t used = 0;
    for (int32_t p = 0; p < pages->n_pages; ++p) {
      if (refs[p] != held[p])
        return fail(PIC_ERR_INVALID_ARG, "page %d has %d references, %d in this table", p, refs[p], held[p]);
      used += refs[p] > 0;
    }
    // pages in use at or past `used` move down to the free pages below it, in order
    int32_t moves = 0;
    for (int32_t p = 0; p < used; ++p) moves += refs[p] == 0;
    if (moves > pair_cap) {
      *n_pairs = moves;
      return fail(PIC_ERR_CAPACITY, "%d pairs needed, room for %d", moves, pair_cap);
    }
    int32_t hole = 0, n = 0;
    for (int32_t p = 0; p < pages->n_pages; ++p) {
      to[p] = p;
      if (p < used || held[p] == 0) continue;
      while (held[hole] != 0) ++hole;
      pairs[2 * n] = p;
      pairs[2 * n + 1] = hole;
      ++n;
      to[p] = hole++;
    }
    for (int64_t i = 0; i < entries; ++i)
      if (page_table[i] != -1) page_table[i] = to[page_table[i]];
    for (int32_t k = 0; k < n; ++k) {
      refs[pairs[2 * k + 1]] = refs[pairs[2 * k]];
      refs[pairs[2 * k]] = 0;
    }
    *n_pairs = n;
    *n_used = used;
    return ok();
  });
}

PIC_API pic_status pic_page_blocks(const pic_pages* pages, int32_t batch, const int32_t* page_table, const pic_block* blocks,
                                   int32_t n_blocks, pic_block* out, int32_t out_cap, int32_t* n_out) {
  PIC_CHECK(check_pages(pages));
  if (batch < 0 || n_blocks < 0 || out_cap < 0) return fail(PIC_ERR_INVALID_ARG, "negative size");
  if (!n_out) return fail(PIC_ERR_INVALID_ARG, "n_out is NULL");
  if (!page_table && (int64_t)batch * pages->table_cap > 0) return fail(PIC_ERR_INVALID_ARG, "page_table is NULL");
  if (n_blocks > 0 && !blocks) return fail(PIC_ERR_INVALID_ARG, "blocks is NULL");
  const int32_t P = pages->page_tokens;
  // counted and checked first, so that a failing call writes no block
  int64_t need = 0;
  for (int32_t k = 0; k < n_blocks; ++k) {
    const pic_block& b = blocks[k];
    if (!map_block_ok(b, batch, (int32_t)std::min((int64_t)pages->table_cap * P, (int64_t)INT32_MAX)))
      return fail(PIC_ERR_RANGE, "block %d (request %d, slots from %d, %d tokens) lies outside the page table", k, b.request,
                  b.dst_slot, b.n_tokens);
    for (int32_t i = b.dst_slot / P; i <= (b.dst_slot + b.n_tokens - 1) / P; ++i) {
      const int32_t page = page_table[(int64_t)b.request * pages->table_cap + i];
      if (page < 0 || page >= pages->n_pages)
        return fail(PIC_ERR_RANGE, "page table entry %d of request %d is %d: no page", i, b.request, page);
      ++need;
    }
  }
  if (need > INT32_MAX) return fail(PIC_ERR_CAPACITY, "too many blocks");
  *n_out = (int32_t)need;
  if (need > out_cap) return fail(PIC_ERR_CAPACITY, "%lld blocks needed, room for %d", (long long)need, out_cap);
  if (need > 0 && !out) return fail(PIC_ERR_INVALID_ARG, "out is NULL");
  int32_t n = 0;
  for (int32_t k = 0; k < n_blocks; ++k) {
    const pic_block& b = blocks[k];
    for (int32_t t = 0; t < b.n_tokens;) {
      const int32_t slot = b.dst_slot + t, in_page = slot % P;
      pic_block& o = out[n++];
      o.request = 0;
      o.src_token = (int32_t)((uint32_t)b.src_token + (uint32_t)t);   // (past INT32_MAX: negative, so in no pool)
      o.dst_slot = page_table[(int64_t)b.request * pages->table_cap + slot / P] * P + in_page;
      o.n_tokens = std::min(b.n_tokens - t, P - in_page);
      o.delta = b.delta;
      t += o.n_tokens;
    }
  }
  return ok();
}

// ---------------------------------------------------------------------------------------------
// 5b. page copies
// ---------------------------------------------------------------------------------------------

namespace {

// All copies are as if at once: no page is written twice, or both read and written.
pic_status check_pairs(const int32_t* pairs, int32_t n_pairs, int32_t n_pages) {
  for (int32_t i = 0; i < 2 * n_pairs; ++i)
    if (pairs[i] < 0 || pairs[i] >= n_pages)
      return fail(PIC_ERR_RANGE, "pair %d: page %d out of [0, %d)", i / 2, pairs[i], n_pages);
  return with_memory([&]() -> pic_status {
    constexpr int32_t kFew = 256;
    int32_t few[kFew];
    std::vector<int32_t> many;
    int32_t* dst = few;
    if (n_pairs > kFew) {
      many.resize(n_pairs);
      dst = many.data();
    }
    for (int32_t i = 0; i < n_pairs; ++i) dst[i] = pairs[2 * i + 1];
    std::sort(dst, dst + n_pairs);
    for (int32_t i = 1; i < n_pairs; ++i)
      if (dst[i] == dst[i - 1]) return fail(PIC_ERR_INVALID_ARG, "page %d is written twice", dst[i]);
    for (int32_t i = 0; i < n_pairs; ++i)
      if (std::binary_search(dst, dst + n_pairs, pairs[2 * i]))
        return fail(PIC_ERR_INVALID_ARG, "page %d is both read and written", pairs[2 * i]);
    return PIC_OK;
  });
}

}  // namespace

PIC_API pic_status pic_page_copy(const pic_model* model, const pic_pages* pages, void* pages_k, void* pages_v,
                                 const int32_t* pairs, int32_t n_pairs, void* stream) {
  PIC_CHECK(check_model(model));
  PIC_CHECK(check_pages(pages));
  if (n_pairs < 0 || n_pairs > pages->n_pages) return fail(PIC_ERR_INVALID_ARG, "%d pairs of %d pages", n_pairs, pages->n_pages);
  if (n_pairs == 0) return ok();
  if (!pairs) return fail(PIC_ERR_INVALID_ARG, "pairs is NULL");
  PIC_CHECK(check_pairs(pairs, n_pairs, pages->n_pages));
  if (model->n_layers == 0) return ok();
  PIC_CHECK(check_ptr(pages_k, "pages_k"));
  PIC_CHECK(check_ptr(pages_v, "pages_v"));
  const int64_t page_bytes = (int64_t)pages->page_tokens * model->head_dim * (model->dtype == PIC_F32 ? 4 : 2);
  return hip_status(launch_page_copy(pages_k, pages_v, (int64_t)model->n_layers * model->n_kv_heads, pages->n_pages, page_bytes,
                                     pairs, n_pairs, (hipStream_t)stream),
                    "page copy launch");
}

// ---------------------------------------------------------------------------------------------
// 5c, 5d. attention of new tokens over pages
// ---------------------------------------------------------------------------------------------

namespace {

// decode: one token per request at base_len + offset, split over the context; else n_new tokens
// from base_len on.  `what` names the lengths' argument.
pic_status page_attn(const pic_model* model, const pic_pages* pages, const void* q, const void* k_new, const void* v_new,
                     void* pages_k, void* pages_v, const int32_t* page_table, int32_t batch, const int32_t* base_len,
                     int32_t max_base, int32_t offset, const int32_t* n_valid, int32_t n_new, bool rope, const void* table,
                     int32_t max_abs_delta, float scale, bool decode, int32_t n_splits, void* out, void* workspace,
                     size_t ws_bytes, void* stream) {
  PIC_CHECK(check_model(model));
  PIC_CHECK(check_pages(pages));
  if (rope && model->dtype != PIC_BF16)
    return fail(PIC_ERR_UNSUPPORTED, "fused RoPE is built for bf16 caches");
  if (batch < 0 || max_base < 0 || offset < 0 || n_new < 0 || n_splits < 0)
    return fail(PIC_ERR_INVALID_ARG, "negative size");
  if (!(scale >= 0.f) || !std::isfinite(scale)) return fail(PIC_ERR_INVALID_ARG, "scale must be finite and >= 0");
  const int64_t max_len = (int64_t)max_base + offset + n_new;
  if (max_len > kMaxSlots) return fail(PIC_ERR_CAPACITY, "%lld slots per request (at most 2^30)", (long long)max_len);
  if (max_len > (int64_t)pages->table_cap * pages->page_tokens)
    return fail(PIC_ERR_CAPACITY, "%lld slots per request exceed a page table of %d pages of %d tokens", (long long)max_len,
                pages->table_cap, pages->page_tokens);
  if (rope && (max_abs_delta < 0 || max_abs_delta > kMaxAbsDelta || max_len - 1 > max_abs_delta))
    return fail(PIC_ERR_RANGE, "position %lld needs a table with max_abs_delta >= that, got %d", (long long)(max_len - 1),
                max_abs_delta);
  if ((int64_t)batch * model->n_q_heads * n_new > INT32_MAX ||
      (int64_t)n_new * (model->n_q_heads / model->n_kv_heads) >= (int64_t(1) << 27))
    return fail(PIC_ERR_UNSUPPORTED, "too many query rows");
  if (model->n_layers > 65535) return fail(PIC_ERR_UNSUPPORTED, "more than 65535 layers");
  const int64_t rows = (int64_t)pages->n_pages * pages->page_tokens;
  if (model->dtype == PIC_BF16 && !decode) PIC_CHECK(check_rows32(0, (int64_t)n_new * model->n_kv_heads, rows));
  if (batch == 0 || n_new == 0 || model->n_layers == 0) return ok();
  if (pages->n_pages == 0) return fail(PIC_ERR_RANGE, "no pages");
  PIC_CHECK(check_ptr(q, "q"));
  PIC_CHECK(check_ptr(k_new, decode ? "k_new" : "k_suf"));
  PIC_CHECK(check_ptr(v_new, decode ? "v_new" : "v_suf"));
  PIC_CHECK(check_ptr(pages_k, "pages_k"));
  PIC_CHECK(check_ptr(pages_v, "pages_v"));
  if (rope) PIC_CHECK(check_ptr(table, "table"));
  PIC_CHECK(check_ptr(out, "out"));
  if (!page_table) return fail(PIC_ERR_INVALID_ARG, "page_table is NULL");
  if (!base_len) return fail(PIC_ERR_INVALID_ARG, decode ? "base_len is NULL" : "ctx_len is NULL");
  PageAttnArgs a;
  a.s = shape_of(model, batch, (int32_t)rows, scale);
  a.map.table = page_table;
  a.map.cap = pages->table_cap;
  a.map.n_pages = pages->n_pages;
  a.map.shift = page_shift(pages->page_tokens);
  if (model->dtype == PIC_BF16) {
    if (decode) PIC_CHECK(plan_decode_call(model, a.s, (int32_t)max_len, false, &n_splits, &workspace, &ws_bytes));
    else PIC_CHECK(check_prefill_workspace(model, batch, n_new, max_base, workspace, &ws_bytes));
  }
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
  a.table = static_cast<const float2*>(table);
  a.table_stride = n_tables(model) > 1 ? (int64_t)(max_abs_delta + 1) * (model->head_dim / 2) : 0;
  a.max_abs_delta = max_abs_delta;
  a.interleaved = model->rope_pairing == PIC_ROPE_INTERLEAVED;
  a.out = out;
  a.workspace = workspace;
  a.ws_bytes = ws_bytes;
  a.n_splits = n_splits;
  a.stream = (hipStream_t)stream;
  const bool few = few_bf16_better(a.s, n_new, max_base, workspace ? ws_bytes : 0);
  const hipError_t e = model->dtype == PIC_F32 ? launch_attn_f32_pages(a)
                       : decode                ? launch_decode_bf16_pages(a)
                       : few                   ? launch_few_bf16_pages(a)
                                               : launch_prefill_bf16_pages(a);
  return hip_status(e, decode ? "page decode launch" : "page suffix launch");
}

}  // namespace

PIC_API pic_status pic_page_suffix_attn(const pic_model* model, const pic_pages* pages, const void* q, const void* k_suf,
                                        const void* v_suf, void* pages_k, void* pages_v, const int32_t* page_table,
                                        int32_t batch, const int32_t* ctx_len, int32_t max_ctx, const int32_t* n_valid,
                                        int32_t n_suffix, float scale, void* out, void* workspace, size_t ws_bytes,
                                        void* stream) {
  return page_attn(model, pages, q, k_suf, v_suf, pages_k, pages_v, page_table, batch, ctx_len, max_ctx, 0, n_valid, n_suffix,
                   false, nullptr, 0, scale, false, 0, out, workspace, ws_bytes, stream);
}

PIC_API pic_status pic_page_suffix_attn_rope(const pic_model* model, const pic_pages* pages, const void* q, const void* k_suf,
                                             const void* v_suf, void* pages_k, void* pages_v, const int32_t* page_table,
                                             int32_t batch, const int32_t* ctx_len, int32_t max_ctx, const int32_t* n_valid,
                                             int32_t n_suffix, const void* table, int32_t max_abs_delta, float scale,
                                             void* out, void* workspace, size_t ws_bytes, void* stream) {
  return page_attn(model, pages, q, k_suf, v_suf, pages_k, pages_v, page_table, batch, ctx_len, max_ctx, 0, n_valid, n_suffix,
                   true, table, max_abs_delta, scale, false, 0, out, workspace, ws_bytes, stream);
}

PIC_API pic_status pic_page_decode_attn(const pic_model* model, const pic_pages* pages, const void* q, const void* k_new,
                                        const void* v_new, void* pages_k, void* pages_v, const int32_t* page_table,
                                        int32_t batch, const int32_t* base_len, int32_t step, int32_t max_base_len,
                                        float scale, int32_t n_splits, void* out, void* workspace, size_t ws_bytes,
                                        void* stream) {
  return page_attn(model, pages, q, k_new, v_new, pages_k, pages_v, page_table, batch, base_len, max_base_len, step, nullptr, 1,
                   false, nullptr, 0, scale, true, n_splits, out, workspace, ws_bytes, stream);
}

PIC_API pic_status pic_page_decode_attn_rope(const pic_model* model, const pic_pages* pages, const void* q, const void* k_new,
                                             const void* v_new, void* pages_k, void* pages_v, const int32_t* page_table,
                                             int32_t batch, const int32_t* base_len, int32_t step, int32_t max_base_len,
                                             const void* table, int32_t max_abs_delta, float scale, int32_t n_splits,
                                             void* out, void* workspace, size_t ws_bytes, void* stream) {
  return page_attn(model, pages, q, k_new, v_new, pages_k, pages_v, page_table, batch, base_len, max_base_len, step, nullptr, 1,
                   true, table, max_abs_delta, scale, true, n_splits, out, workspace, ws_bytes, stream);
}
