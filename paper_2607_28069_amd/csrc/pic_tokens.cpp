// C ABI of libpic, new tokens before their attention: norms of queries and keys with the rotation, and the
// frequencies of a rotation stretched for long contexts.
#include <hip/hip_runtime.h>

#include <algorithm>
#include <cmath>

#include "pic.h"
#include "pic_check.h"
#include "pic_internal.h"

using namespace pic;

namespace {

// rope_dim as given (0: the whole head), or an error
pic_status check_rope_dim(int32_t head_dim, int32_t* rope_dim) {
  if (*rope_dim == 0) *rope_dim = head_dim;
  if (*rope_dim < 0 || *rope_dim > head_dim || *rope_dim % 16 != 0)
    return fail(PIC_ERR_UNSUPPORTED, "rope_dim %d of %d (a multiple of 16)", *rope_dim, head_dim);
  return PIC_OK;
}

// One of q, k and v: rows of n_heads heads, `stride` elements from token to token (0: dense).
pic_status check_rows(const pic_model* m, const void* in, int64_t* stride, int32_t n_heads, const void* out, const char* name) {
  const int64_t dense = (int64_t)n_heads * m->head_dim;
  if (*stride == 0) *stride = dense;
  if (*stride < dense) return fail(PIC_ERR_INVALID_ARG, "%s: %lld elements from token to token, %lld in a row", name,
                                   (long long)*stride, (long long)dense);
  if (*stride % (m->dtype == PIC_F32 ? 4 : 8) != 0) return fail(PIC_ERR_MISALIGNED, "%s: rows are not 16-byte aligned", name);
  PIC_CHECK(check_ptr(in, name));
  PIC_CHECK(check_ptr(out, name));
  if (in == out && *stride != dense) return fail(PIC_ERR_INVALID_ARG, "%s: in place only where the rows are dense", name);
  return PIC_OK;
}

}  // namespace

PIC_API pic_status pic_rope_yarn_freq(int32_t head_dim, int32_t rope_dim, double theta, double factor,
                                      double original_max_position, double beta_fast, double beta_slow, double* inv_freq,
                                      double* attention_factor) {
  if (head_dim != 64 && head_dim != 128) return fail(PIC_ERR_INVALID_ARG, "head_dim %d (supported: 64, 128)", head_dim);
  PIC_CHECK(check_rope_dim(head_dim, &rope_dim));
  if (!inv_freq || !attention_factor) return fail(PIC_ERR_INVALID_ARG, "inv_freq or attention_factor is NULL");
  if (!(theta > 1.0) || !(factor >= 1.0) || !(original_max_position > 0.0) || !(beta_slow > 0.0) || !(beta_fast > beta_slow) ||
      !std::isfinite(theta) || !std::isfinite(factor) || !std::isfinite(original_max_position) || !std::isfinite(beta_fast))
    return fail(PIC_ERR_INVALID_ARG, "inconsistent frequency-scaling parameters");
  const double pi = 3.14159265358979323846;
  // the pair (a real number) that turns `turns` times over the original positions
  auto pair_of = [&](double turns) { return rope_dim * std::log(original_max_position / (turns * 2 * pi)) / (2 * std::log(theta)); };
  const double low = std::max(std::floor(pair_of(beta_fast)), 0.0);
  const double high = std::min(std::ceil(pair_of(beta_slow)), rope_dim - 1.0);
  const double span = std::max(high - low, 1e-3);
  for (int i = 0; i < head_dim / 2; ++i) {
    inv_freq[i] = 0.0;
    if (i >= rope_dim / 2) continue;
    const double f = std::pow(theta, -2.0 * i / rope_dim);
    const double ramp = std::min(std::max((i - low) / span, 0.0), 1.0);   // 0: kept, 1: divided by factor
    inv_freq[i] = f / factor * ramp + f * (1 - ramp);
  }
  *attention_factor = 0.1 * std::log(factor) + 1.0;
  return ok();
}

PIC_API pic_status pic_qk_norm_rope(const pic_model* model, const pic_qk_norm* how, const void* q, int64_t q_stride,
                                    const void* k, int64_t k_stride, const void* v, int64_t v_stride, int32_t batch,
                                    const int32_t* base_len, int32_t max_base_len, int32_t offset, const int32_t* n_valid,
                                    int32_t n_new, const void* table, int32_t max_abs_delta, void* q_out, void* k_out,
                                    void* v_out, void* stream) {
  PIC_CHECK(check_model(model));
  if (!how) return fail(PIC_ERR_INVALID_ARG, "how is NULL");
  if (batch < 0 || n_new < 0 || max_base_len < 0 || offset < 0) return fail(PIC_ERR_INVALID_ARG, "negative size");
  if (!(how->eps >= 0.f) || !std::isfinite(how->eps)) return fail(PIC_ERR_INVALID_ARG, "eps must be finite and >= 0");
  if (!std::isfinite(how->rope_scale)) return fail(PIC_ERR_INVALID_ARG, "rope_scale must be finite");
  if (how->rope_order != PIC_ROPE_ORDER_KEEP && how->rope_order != PIC_ROPE_ORDER_PAIRS)
    return fail(PIC_ERR_INVALID_ARG, "rope_order %d", how->rope_order);
  int32_t rope_dim = how->rope_dim;
  PIC_CHECK(check_rope_dim(model->head_dim, &rope_dim));
  if (table) {
    if (max_abs_delta < 0 || max_abs_delta > kMaxAbsDelta)
      return fail(PIC_ERR_RANGE, "max_abs_delta %d outside [0, %d]", max_abs_delta, kMaxAbsDelta);
    const int64_t last = (int64_t)(base_len ? max_base_len : 0) + offset + n_new - 1;
    if (last > max_abs_delta)
      return fail(PIC_ERR_RANGE, "position %lld needs a table with max_abs_delta >= that, got %d", (long long)last, max_abs_delta);
    PIC_CHECK(check_ptr(table, "table"));
  }
  if (model->n_layers > 65535) return fail(PIC_ERR_UNSUPPORTED, "more than 65535 layers");
  QkNormArgs a;
  // (items of kQkNormHeads heads of a token; a grid holds fewer than 2^32 threads)
  const int64_t rows = (int64_t)batch * n_new, tokens = rows < (int64_t(1) << 28) ? model->n_layers * rows : rows;
  auto chunks = [](const void* x, int64_t heads) { return x ? (heads + kQkNormHeads - 1) / kQkNormHeads : 0; };
  const int64_t heads = chunks(q, model->n_q_heads) + chunks(k, model->n_kv_heads) + chunks(v, model->n_kv_heads);
  if (tokens >= (int64_t(1) << 28) || heads >= (int64_t(1) << 28) || tokens * heads * 16 >= (int64_t(1) << 32))
    return fail(PIC_ERR_UNSUPPORTED, "too many tokens in one call");
  if (tokens == 0 || heads == 0) return ok();
  if (!aligned16(how->q_weight)) return fail(PIC_ERR_MISALIGNED, "q_weight is not 16-byte aligned");
  if (!aligned16(how->k_weight)) return fail(PIC_ERR_MISALIGNED, "k_weight is not 16-byte aligned");
  if (q) PIC_CHECK(check_rows(model, q, &q_stride, model->n_q_heads, q_out, "q"));
  if (k) PIC_CHECK(check_rows(model, k, &k_stride, model->n_kv_heads, k_out, "k"));
  if (v) PIC_CHECK(check_rows(model, v, &v_stride, model->n_kv_heads, v_out, "v"));
  a.q = q;
  a.k = k;
  a.v = v;
  a.q_out = q_out;
  a.k_out = k_out;
  a.v_out = v_out;
  a.q_stride = q_stride;
  a.k_stride = k_stride;
  a.v_stride = v_stride;
  a.q_weight = how->q_weight;
  a.k_weight = how->k_weight;
  a.base_len = base_len;
  a.n_valid = n_valid;
  a.table = static_cast<const float2*>(table);
  a.table_stride = n_tables(model) > 1 ? (int64_t)(max_abs_delta + 1) * (model->head_dim / 2) : 0;
  a.batch = batch;
  a.n_new = n_new;
  a.n_q_heads = model->n_q_heads;
  a.n_kv_heads = model->n_kv_heads;
  a.max_base = max_base_len;
  a.offset = offset;
  a.rope_dim = rope_dim;
  a.eps = how->eps;
  a.rope_scale = how->rope_scale == 0.f ? 1.f : how->rope_scale;
  a.pairs_order = how->rope_order == PIC_ROPE_ORDER_PAIRS;
  return hip_status(launch_qk_norm(model->dtype, model->head_dim, model->rope_pairing == PIC_ROPE_INTERLEAVED, model->n_layers, a,
                                   (hipStream_t)stream),
                    "qk norm launch");
}
