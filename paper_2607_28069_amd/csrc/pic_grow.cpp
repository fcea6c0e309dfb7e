// C ABI of libpic, page bookkeeping on the device: tables grown from the requests' lengths, and copies of listed pages.
#include <hip/hip_runtime.h>

#include "pic.h"
#include "pic_check.h"
#include "pic_internal.h"

using namespace pic;

namespace {

pic_status check_grow(const pic_pages* pg, int32_t batch, int32_t n_new) {
  PIC_CHECK(check_pages(pg));
  if (batch < 0 || n_new < 0) return fail(PIC_ERR_INVALID_ARG, "negative size");
  if (page_grow_entries(pg->page_tokens, pg->table_cap, batch, n_new) > (int64_t(1) << 28))
    return fail(PIC_ERR_UNSUPPORTED, "too many table entries in one call");
  return PIC_OK;
}

size_t grow_bytes(const pic_pages* pg, int32_t batch, int32_t n_new) {
  const int64_t entries = page_grow_entries(pg->page_tokens, pg->table_cap, batch, n_new);
  return (size_t)(batch + 1 + 3 * entries + std::min<int64_t>(entries, pg->n_pages)) * sizeof(int32_t);
}

}  // namespace

PIC_API size_t pic_page_grow_workspace_bytes(const pic_pages* pages, int32_t batch, int32_t n_new) {
  return check_grow(pages, batch, n_new) == PIC_OK ? grow_bytes(pages, batch, n_new) : 0;
}

PIC_API pic_status pic_page_grow_async(const pic_pages* pages, int32_t batch, int32_t* refs, int32_t* page_table,
                                       const int32_t* base_len, int32_t offset, const int32_t* n_valid, int32_t n_new,
                                       int32_t* pairs, int32_t* ready, int32_t* result, void* workspace, size_t ws_bytes,
                                       void* stream) {
  PIC_CHECK(check_grow(pages, batch, n_new));
  if (offset < 0) return fail(PIC_ERR_INVALID_ARG, "offset < 0");
  PIC_CHECK(check_ptr(result, "result"));
  if (batch > 0) {
    if (pages->n_pages > 0) PIC_CHECK(check_ptr(refs, "refs"));
    if (pages->table_cap > 0) PIC_CHECK(check_ptr(page_table, "page_table"));
    if (!base_len) return fail(PIC_ERR_INVALID_ARG, "base_len is NULL");
    PIC_CHECK(check_ptr(pairs, "pairs"));
    PIC_CHECK(check_ptr(ready, "ready"));
  }
  const size_t need = grow_bytes(pages, batch, n_new);
  if (!workspace || ws_bytes < need)
    return fail(PIC_ERR_WORKSPACE, "workspace needs %zu bytes, got %zu", need, workspace ? ws_bytes : (size_t)0);
  PIC_CHECK(check_ptr(workspace, "workspace"));
  PageGrowArgs a;
  a.refs = refs;
  a.page_table = page_table;
  a.base_len = base_len;
  a.n_valid = n_valid;
  a.pairs = pairs;
  a.ready = ready;
  a.result = result;
  a.workspace = static_cast<int32_t*>(workspace);
  a.n_pages = batch > 0 ? pages->n_pages : 0;   // (without requests no page is looked at)
  a.table_cap = pages->table_cap;
  a.shift = __builtin_ctz((unsigned)pages->page_tokens);
  a.batch = batch;
  a.n_new = n_new;
  a.offset = offset;
  return hip_status(launch_page_grow(a, (hipStream_t)stream), "page grow launch");
}

PIC_API pic_status pic_page_copy_async(const pic_model* model, const pic_pages* pages, void* pages_k, void* pages_v,
                                       const int32_t* pairs, int32_t pair_cap, void* stream) {
  PIC_CHECK(check_model(model));
  PIC_CHECK(check_grow(pages, 0, 0));
  if (pair_cap < 0) return fail(PIC_ERR_INVALID_ARG, "pair_cap < 0");
  if (pair_cap == 0 || model->n_layers == 0 || pages->n_pages == 0) return ok();
  PIC_CHECK(check_ptr(pages_k, "pages_k"));
  PIC_CHECK(check_ptr(pages_v, "pages_v"));
  PIC_CHECK(check_ptr(pairs, "pairs"));
  const int64_t page_bytes = (int64_t)pages->page_tokens * model->head_dim * (model->dtype == PIC_F32 ? 4 : 2);
  return hip_status(launch_page_copy_listed(pages_k, pages_v, (int64_t)model->n_layers * model->n_kv_heads, pages->n_pages,
                                            page_bytes, pairs, pair_cap, (hipStream_t)stream),
                    "page copy launch");
}
