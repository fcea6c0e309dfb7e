// Norms of queries and keys for each head with the position rotation in the same pass: what stands between a layer's
// projections and its attention.
//
//   y = x w / sqrt(mean(x^2) + eps)             over the D elements of a head, w per layer
//   z = scale R(p) y on the first rope_dim elements, y on the others       p = the token's slot
//
// in float32 from the load to the one rounding of the store (the rotation in the form of the re-rotation kernel).  Per
// head some 10 flops an element: the bytes are the whole cost, each row read once and written once.
//
// A lane holds two 16-byte pieces of a row, so that both members of every turned pair are its own: piece j of either
// half of the turned part (halves), or 32 bytes in one piece (interleaved); D / 2 / VEC lanes hold a row, and their
// sums of squares meet in 2 to 4 DPP additions.  Those lanes take kQkNormHeads = 2 heads of one token, neighbouring lanes
// neighbouring heads, with all their loads on their way at once: weights and the token's row of the rotary table are
// asked for once for 2 rows.  Values only move: from a slice of the projection's rows to the dense rows that the
// attention calls take.
//
// Measured with 1 / 2 / 4 heads: 7 tokens of 28 + 2 x 4 heads 3.1 / 3.4 / 4.2 us, 16 x 131 tokens of 32 + 2 x 8 heads, half
// of them padding, 11.9 / 11.2 / 11.8 us, 64 x 1024 tokens of 32 + 2 x 8 heads 328 / 296 / 291 us (5.4 TB/s).  A workgroup
// walking over its tokens' heads with the weights in registers, the table's row asked for once a head's norm was done,
// took 4.1, 13.5 and 311 us.  Loads and stores that pass the caches by took 320 us for the long call: the next kernel's
// reads would miss as well.
#include <type_traits>

#include "pic_bounds.h"
#include "pic_internal.h"

namespace pic {
namespace {

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

template <typename T>
struct Piece;   // 16 bytes of T
template <>
struct Piece<float> {
  static constexpr int N = 4;
  static __device__ __forceinline__ void widen(u32x4 v, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) x[i] = __uint_as_float(v[i]);
  }
  static __device__ __forceinline__ u32x4 round(const float* x) {
    return u32x4{__float_as_uint(x[0]), __float_as_uint(x[1]), __float_as_uint(x[2]), __float_as_uint(x[3])};
  }
};
template <>
struct Piece<bf16_t> {
  static constexpr int N = 8;
  static __device__ __forceinline__ void widen(u32x4 v, float* x) {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      x[2 * i] = __uint_as_float(v[i] << 16);
      x[2 * i + 1] = __uint_as_float(v[i] & 0xFFFF0000u);
    }
  }
  static __device__ __forceinline__ u32x4 round(const float* x) {
    return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]), pack_bf16x2(x[6], x[7])};
  }
};

// The sum of x over the aligned N lanes (4, 8 or 16) around this one.
template <int N>
__device__ __forceinline__ float sum_of(float x) {
  auto add = [&](auto ctrl) {
    x += __uint_as_float(__builtin_amdgcn_update_dpp(0, __float_as_uint(x), decltype(ctrl)::value, 0xF, 0xF, false));
  };
  add(std::integral_constant<int, 0xB1>{});                          // quad_perm 1 0 3 2
  add(std::integral_constant<int, 0x4E>{});                          // quad_perm 2 3 0 1
  if constexpr (N >= 8) add(std::integral_constant<int, 0x141>{});   // row_half_mirror
  if constexpr (N >= 16) add(std::integral_constant<int, 0x140>{});  // row_mirror
  return x;
}

constexpr int kHeads = kQkNormHeads;

// grid: lanes of (token, chunk of heads) in order, 256 threads
template <typename T, int HD, bool kInterleaved>
__global__ void __launch_bounds__(256) qk_norm_kernel(QkNormArgs a, uint32_t q_chunks, uint32_t k_chunks, uint32_t chunks, uint32_t items) {
  constexpr int VEC = Piece<T>::N, LPR = HD / 2 / VEC;
  const uint32_t item = (blockIdx.x * 256 + threadIdx.x) / LPR;
  if (item >= items) return;
  const uint32_t tok = item / chunks, chunk = item - tok * chunks;
  const uint32_t lb = tok / (uint32_t)a.n_new, l = lb / (uint32_t)a.batch;
  const int i = tok - lb * a.n_new, b = lb - l * a.batch;
  // which heads
  const bool is_q = chunk < q_chunks, is_v = chunk >= q_chunks + k_chunks;
  const int h0 = is_q ? chunk : is_v ? chunk - q_chunks - k_chunks : chunk - q_chunks;
  const int heads = is_q ? a.n_q_heads : a.n_kv_heads, apart = (heads + kHeads - 1) / kHeads;   // heads h0, h0 + apart, ...
  int n_tok = a.n_new;
  int64_t pos = a.offset + i;
  if (a.base_len) {
    n_tok = page_new_tokens(a.base_len, a.n_valid, b, a.n_new);
    pos += clamp_len(a.base_len[b], a.max_base);
  } else if (a.n_valid) {
    n_tok = clamp_len(a.n_valid[b], a.n_new);
  }
  if (i >= n_tok) return;   // padding
  const int j = threadIdx.x % LPR, turning = a.rope_dim / 2 / VEC;   // lanes [0, turning) hold turned pairs
  int in1, in2, out1, out2;   // elements of this lane's pieces
  if constexpr (kInterleaved) {
    in1 = out1 = 2 * j * VEC;
    in2 = out2 = in1 + VEC;
  } else {
    const int rest = (HD - a.rope_dim) / 2;
    in1 = j < turning ? j * VEC : a.rope_dim + (j - turning) * VEC;
    in2 = in1 + (j < turning ? a.rope_dim / 2 : rest);
    out1 = a.pairs_order && !is_v ? j * VEC : in1;
    out2 = a.pairs_order && !is_v ? HD / 2 + j * VEC : in2;
  }
  const T* in = static_cast<const T*>(is_q ? a.q : is_v ? a.v : a.k) + (int64_t)tok * (is_q ? a.q_stride : is_v ? a.v_stride : a.k_stride) + h0 * HD;
  T* out = static_cast<T*>(is_q ? a.q_out : is_v ? a.v_out : a.k_out) + ((int64_t)tok * heads + h0) * HD;
  u32x4 x1[kHeads], x2[kHeads];
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    const T* row = in + (h0 + u * apart < heads ? u * apart : 0) * HD;
    x1[u] = *reinterpret_cast<const u32x4*>(row + in1);
    x2[u] = *reinterpret_cast<const u32x4*>(row + in2);
  }
  const bool turned = a.table && !is_v && j < turning;
  float c[VEC], s[VEC];
  if (turned) {
    const float2* cs = a.table + (int64_t)l * a.table_stride + pos * (HD / 2) + j * VEC;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      c[e] = cs[e].x * a.rope_scale;
      s[e] = cs[e].y * a.rope_scale;
    }
  }
  const float* weight = is_q ? a.q_weight : is_v ? nullptr : a.k_weight;
  float w[2 * VEC];
  if (weight) {
    weight += (int64_t)l * HD;
#pragma unroll
    for (int e = 0; e < VEC; ++e) {
      w[e] = weight[in1 + e];
      w[VEC + e] = weight[in2 + e];
    }
  }
#pragma unroll
  for (int u = 0; u < kHeads; ++u) {
    if (h0 + u * apart >= heads) break;   // (the lanes of a row leave together)
    if (!is_v) {
      float x[2 * VEC];
      Piece<T>::widen(x1[u], x);
      Piece<T>::widen(x2[u], x + VEC);
      if (weight) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) ss = fmaf(x[e], x[e], ss);
        const float r = 1.f / sqrtf(sum_of<LPR>(ss) * (1.f / HD) + a.eps);
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) x[e] = x[e] * r * w[e];
      }
      if (turned) {
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          float& x0 = kInterleaved ? x[2 * e] : x[e];
          float& y0 = kInterleaved ? x[2 * e + 1] : x[VEC + e];
          const float p = x0, q = y0;
          x0 = fmaf(p, c[e], -(q * s[e]));
          y0 = fmaf(p, s[e], q * c[e]);
        }
      }
      x1[u] = Piece<T>::round(x);
      x2[u] = Piece<T>::round(x + VEC);
    }
    *reinterpret_cast<u32x4*>(out + u * apart * HD + out1) = x1[u];
    *reinterpret_cast<u32x4*>(out + u * apart * HD + out2) = x2[u];
  }
}

template <typename T, int HD>
hipError_t launch_as(const QkNormArgs& a, bool interleaved, int n_layers, hipStream_t stream) {
  auto chunks = [](const void* x, int heads) { return x ? (uint32_t)(heads + kHeads - 1) / kHeads : 0u; };
  const uint32_t qc = chunks(a.q, a.n_q_heads), kc = chunks(a.k, a.n_kv_heads), all = qc + kc + chunks(a.v, a.n_kv_heads);
  const int64_t tokens = (int64_t)n_layers * a.batch * a.n_new, items = tokens * all;
  constexpr int kPer = 256 / (HD / 2 / Piece<T>::N);
  const auto kernel = interleaved ? qk_norm_kernel<T, HD, true> : qk_norm_kernel<T, HD, false>;
  hipLaunchKernelGGL(kernel, dim3((unsigned)((items + kPer - 1) / kPer)), dim3(256), 0, stream, a, qc, kc, all, (uint32_t)items);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm(pic_dtype dt, int head_dim, bool interleaved, int n_layers, QkNormArgs a, hipStream_t stream) {
  if (dt == PIC_F32)
    return head_dim == 64 ? launch_as<float, 64>(a, interleaved, n_layers, stream) : launch_as<float, 128>(a, interleaved, n_layers, stream);
  return head_dim == 64 ? launch_as<bf16_t, 64>(a, interleaved, n_layers, stream) : launch_as<bf16_t, 128>(a, interleaved, n_layers, stream);
}

}  // namespace pic
