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
// sums of squares meet in 2 to 4 DPP additions.  A workgroup takes a few neighbouring tokens of one request with
// all their heads: weights stay in registers (a lane's pieces are the same in every row), and a token's row of
// the rotary table is read from the caches by all heads but one.  Values only move: from a slice of the
// projection's rows to the dense rows that the attention calls take.
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

// grid (B * ceil(n_new / tokens), L), 256 threads
template <typename T, int HD, bool kInterleaved>
__global__ void __launch_bounds__(256) qk_norm_kernel(QkNormArgs a) {
  constexpr int VEC = Piece<T>::N, LPR = HD / 2 / VEC, RPP = 256 / LPR, kAhead = 4;
  const int per_request = (a.n_new + a.tokens - 1) / a.tokens;
  const int b = blockIdx.x / per_request, i0 = (blockIdx.x - b * per_request) * a.tokens, l = blockIdx.y;
  // (uniform) the used tokens of this request, and the position of its first
  int n_tok = a.n_new;
  int64_t pos0 = a.offset;
  if (a.base_len) {
    n_tok = page_new_tokens(a.base_len, a.n_valid, b, a.n_new);
    pos0 += clamp_len(a.base_len[b], a.max_base);
  } else if (a.n_valid) {
    n_tok = clamp_len(a.n_valid[b], a.n_new);
  }
  const int n_here = min(n_tok - i0, a.tokens);
  if (n_here <= 0) return;
  const int j = threadIdx.x % LPR, turning = a.rope_dim / 2 / VEC;   // lanes [0, turning) hold turned pairs
  const bool turned = a.table && j < turning;
  int in1, in2, out1, out2;   // elements of this lane's pieces
  if constexpr (kInterleaved) {
    in1 = out1 = 2 * j * VEC;
    in2 = out2 = in1 + VEC;
  } else {
    const int rest = (HD - a.rope_dim) / 2;
    in1 = j < turning ? j * VEC : a.rope_dim + (j - turning) * VEC;
    in2 = in1 + (j < turning ? a.rope_dim / 2 : rest);
    out1 = a.pairs_order ? j * VEC : in1;
    out2 = a.pairs_order ? HD / 2 + j * VEC : in2;
  }
  // weights of the queries and of the keys at this lane's elements
  float w[2][2 * VEC];
#pragma unroll
  for (int x = 0; x < 2; ++x) {
    const float* from = x ? a.k_weight : a.q_weight;
    if (from) {
      from += (int64_t)l * HD;
#pragma unroll
      for (int e = 0; e < VEC; ++e) {
        w[x][e] = from[in1 + e];
        w[x][VEC + e] = from[in2 + e];
      }
    }
  }
  const float2* table = a.table + (int64_t)l * a.table_stride;
  const int64_t tok0 = ((int64_t)l * a.batch + b) * a.n_new + i0;
  const int qh = a.q ? a.n_q_heads : 0, kh = a.k ? a.n_kv_heads : 0, heads = qh + kh + (a.v ? a.n_kv_heads : 0);
  // rows of these tokens, head by head: this thread's are threadIdx.x / LPR, + RPP, ...
  int t = 0, h = threadIdx.x / LPR;
  auto settle = [&]() {
    while (h >= heads && t < n_here) {
      h -= heads;
      ++t;
    }
  };
  settle();
  while (t < n_here) {
    int row_t[kAhead], row_h[kAhead];
    u32x4 x1[kAhead], x2[kAhead];
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      row_t[u] = t;
      row_h[u] = h;
      if (t < n_here) {
        const int64_t tok = tok0 + t;
        const T* row = h < qh        ? static_cast<const T*>(a.q) + tok * a.q_stride + h * HD
                       : h < qh + kh ? static_cast<const T*>(a.k) + tok * a.k_stride + (h - qh) * HD
                                     : static_cast<const T*>(a.v) + tok * a.v_stride + (h - qh - kh) * HD;
        x1[u] = *reinterpret_cast<const u32x4*>(row + in1);
        x2[u] = *reinterpret_cast<const u32x4*>(row + in2);
        h += RPP;
        settle();
      }
    }
#pragma unroll
    for (int u = 0; u < kAhead; ++u) {
      if (row_t[u] >= n_here) break;   // (the lanes of a row leave together)
      const int64_t tok = tok0 + row_t[u];
      const int rh = row_h[u];
      if (rh >= qh + kh) {
        T* row = static_cast<T*>(a.v_out) + (tok * a.n_kv_heads + (rh - qh - kh)) * HD;
        *reinterpret_cast<u32x4*>(row + in1) = x1[u];
        *reinterpret_cast<u32x4*>(row + in2) = x2[u];
        continue;
      }
      float x[2 * VEC];
      Piece<T>::widen(x1[u], x);
      Piece<T>::widen(x2[u], x + VEC);
      const bool is_k = rh >= qh;
      if (is_k ? a.k_weight != nullptr : a.q_weight != nullptr) {
        float ss = 0.f;
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) ss = fmaf(x[e], x[e], ss);
        const float r = 1.f / sqrtf(sum_of<LPR>(ss) * (1.f / HD) + a.eps);
#pragma unroll
        for (int e = 0; e < 2 * VEC; ++e) x[e] = x[e] * r * (is_k ? w[1][e] : w[0][e]);
      }
      if (turned) {
        const float2* cs = table + (pos0 + i0 + row_t[u]) * (HD / 2) + j * VEC;
#pragma unroll
        for (int e = 0; e < VEC; ++e) {
          const float c = cs[e].x * a.rope_scale, s = cs[e].y * a.rope_scale;
          float& x0 = kInterleaved ? x[2 * e] : x[e];
          float& y0 = kInterleaved ? x[2 * e + 1] : x[VEC + e];
          const float p = x0, q = y0;
          x0 = fmaf(p, c, -(q * s));
          y0 = fmaf(p, s, q * c);
        }
      }
      T* row = is_k ? static_cast<T*>(a.k_out) + (tok * a.n_kv_heads + (rh - qh)) * HD
                    : static_cast<T*>(a.q_out) + (tok * a.n_q_heads + rh) * HD;
      *reinterpret_cast<u32x4*>(row + out1) = Piece<T>::round(x);
      *reinterpret_cast<u32x4*>(row + out2) = Piece<T>::round(x + VEC);
    }
  }
}

template <typename T, int HD>
hipError_t launch_as(const QkNormArgs& a, bool interleaved, dim3 grid, hipStream_t stream) {
  if (interleaved)
    hipLaunchKernelGGL((qk_norm_kernel<T, HD, true>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((qk_norm_kernel<T, HD, false>), grid, dim3(256), 0, stream, a);
  return hipGetLastError();
}

}  // namespace

hipError_t launch_qk_norm(pic_dtype dt, int head_dim, bool interleaved, int n_layers, QkNormArgs a, hipStream_t stream) {
  const int64_t per = (a.n_new + a.tokens - 1) / a.tokens;
  const dim3 grid((unsigned)(per * a.batch), n_layers);
  if (dt == PIC_F32)
    return head_dim == 64 ? launch_as<float, 64>(a, interleaved, grid, stream) : launch_as<float, 128>(a, interleaved, grid, stream);
  return head_dim == 64 ? launch_as<bf16_t, 64>(a, interleaved, grid, stream) : launch_as<bf16_t, 128>(a, interleaved, grid, stream);
}

}  // namespace pic
