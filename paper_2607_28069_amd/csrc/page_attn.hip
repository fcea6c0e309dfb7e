// Attention of new tokens over a paged cache, for every type and shape: the new rows are stored into
// their pages by one launch, then one wave takes one query row and walks the slots it sees, 64 at a
// time with a running maximum and sum.
#include <type_traits>

#include "pic_bounds.h"
#include "pic_internal.h"

namespace pic {
namespace {

template <typename T>
__device__ __forceinline__ float to_f32(T x) {
  if constexpr (std::is_same_v<T, float>) return x;
  else return bf16_to_f32(x);
}
template <typename T>
__device__ __forceinline__ T from_f32(float x) {
  if constexpr (std::is_same_v<T, float>) return x;
  else return (T)(pack_bf16x2(x, 0.f) & 0xFFFFu);
}

// Element d of a row, turned to position p where there is a table (and rounded as when stored).
template <typename T, int HD>
__device__ __forceinline__ T turned(const T* row, int d, const PageAttnArgs& a, int l, int p) {
  if (a.table == nullptr) return row[d];
  const int i = a.interleaved ? d >> 1 : d & (HD / 2 - 1);
  const int dx = a.interleaved ? 2 * i : i, dy = a.interleaved ? 2 * i + 1 : i + HD / 2;
  const float2 cs = a.table[l * a.table_stride + (int64_t)min(p, a.max_abs_delta) * (HD / 2) + i];
  const float x = to_f32(row[dx]), y = to_f32(row[dy]);
  return from_f32<T>(d == dx ? fmaf(x, cs.x, -(y * cs.y)) : fmaf(x, cs.y, y * cs.x));
}

// rows (l, b, i, g) of the new tokens, one wave each
template <typename T, int HD>
__global__ void __launch_bounds__(64) page_append_kernel(PageAttnArgs a, int64_t n_rows) {
  const AttnShape& s = a.s;
  for (int64_t r = blockIdx.x; r < n_rows; r += gridDim.x) {
    const int g = (int)(r % s.n_kv_heads), i = (int)(r / s.n_kv_heads % a.n_new);
    const int64_t lb = r / s.n_kv_heads / a.n_new;
    const int b = (int)(lb % s.batch), l = (int)(lb / s.batch);
    if (i >= page_new_tokens(a.base_len, a.n_valid, b, a.n_new)) continue;
    const int p = clamp_len(a.base_len[b], a.max_base) + a.offset + i;
    const int64_t row = page_store_row(a.map, b, p);
    if (row < 0) continue;
    const int64_t dst = (((int64_t)l * s.n_kv_heads + g) * s.cache_cap + row) * HD;
    for (int d = threadIdx.x; d < HD; d += 64) {
      static_cast<T*>(a.pages_k)[dst + d] = turned<T, HD>(static_cast<const T*>(a.k_new) + r * HD, d, a, l, p);
      static_cast<T*>(a.pages_v)[dst + d] = static_cast<const T*>(a.v_new)[r * HD + d];
    }
  }
}

// rows (l, b, i, h) of the queries, one wave each
template <typename T, int HD>
__global__ void __launch_bounds__(64) page_attn_kernel(PageAttnArgs a, int64_t n_rows) {
  __shared__ float qs[HD], ps[64];
  __shared__ int64_t rows[64];
  const AttnShape& s = a.s;
  const int lane = threadIdx.x;
  for (int64_t r = blockIdx.x; r < n_rows; r += gridDim.x) {
    const int h = (int)(r % s.n_q_heads), i = (int)(r / s.n_q_heads % a.n_new);
    const int64_t lb = r / s.n_q_heads / a.n_new;
    const int b = (int)(lb % s.batch), l = (int)(lb / s.batch);
    if (i >= page_new_tokens(a.base_len, a.n_valid, b, a.n_new)) continue;
    const int p = clamp_len(a.base_len[b], a.max_base) + a.offset + i;
    const int64_t stream = (((int64_t)l * s.n_kv_heads + h / (s.n_q_heads / s.n_kv_heads)) * s.cache_cap) * HD;
    const T* K = static_cast<const T*>(a.pages_k) + stream;
    const T* V = static_cast<const T*>(a.pages_v) + stream;
    for (int d = lane; d < HD; d += 64) qs[d] = to_f32(turned<T, HD>(static_cast<const T*>(a.q) + r * HD, d, a, l, p));
    __syncthreads();
    float m = -INFINITY, den = 0.f, o[HD / 64] = {};
    for (int k0 = 0; k0 <= p; k0 += 64) {
      const int key = k0 + lane;
      const int64_t row = page_row(a.map, b, min(key, p));
      float x = 0.f;
      for (int d = 0; d < HD; ++d) x = fmaf(qs[d], to_f32(K[row * HD + d]), x);
      x = key <= p ? x * s.scale_log2 : -INFINITY;
      float mx = x;
      for (int w = 32; w > 0; w >>= 1) mx = fmaxf(mx, __shfl_xor(mx, w, 64));
      const float m_new = fmaxf(m, mx), keep = __builtin_amdgcn_exp2f(m - m_new), e = __builtin_amdgcn_exp2f(x - m_new);
      m = m_new;
      float sum = e;
      for (int w = 32; w > 0; w >>= 1) sum += __shfl_xor(sum, w, 64);
      den = den * keep + sum;
      __syncthreads();
      ps[lane] = e;
      rows[lane] = row;
      __syncthreads();
      const int n = min(64, p - k0 + 1);
      for (int c = 0; c < HD / 64; ++c) {
        float acc = o[c] * keep;
        for (int j = 0; j < n; ++j) acc = fmaf(ps[j], to_f32(V[rows[j] * HD + 64 * c + lane]), acc);
        o[c] = acc;
      }
    }
    for (int c = 0; c < HD / 64; ++c) static_cast<T*>(a.out)[r * HD + 64 * c + lane] = from_f32<T>(o[c] / den);
    __syncthreads();
  }
}

template <typename T, int HD>
hipError_t launch_as(const PageAttnArgs& a) {
  const int64_t tokens = (int64_t)a.s.n_layers * a.s.batch * a.n_new;
  const int64_t kv = tokens * a.s.n_kv_heads, q = tokens * a.s.n_q_heads, most = int64_t(1) << 22;
  hipLaunchKernelGGL((page_append_kernel<T, HD>), dim3((unsigned)(kv < most ? kv : most)), dim3(64), 0, a.stream, a, kv);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  hipLaunchKernelGGL((page_attn_kernel<T, HD>), dim3((unsigned)(q < most ? q : most)), dim3(64), 0, a.stream, a, q);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_page_attn(pic_dtype dt, const PageAttnArgs& a) {
  if (dt == PIC_F32) return a.s.head_dim == 64 ? launch_as<float, 64>(a) : launch_as<float, 128>(a);
  return a.s.head_dim == 64 ? launch_as<bf16_t, 64>(a) : launch_as<bf16_t, 128>(a);
}

}  // namespace pic
