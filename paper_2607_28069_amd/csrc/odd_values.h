// What is not finite in the bf16 attention kernels' sums over values of a paged cache.  A probability, or the
// weight of a partial sum, may be 0 in 32 bits where the softmax's is not, and a probability's second term has
// either sign: an infinity would become NaN.  So where a sum came out not finite (any_odd: an addition each), what is
// not finite in it is added up without weights.
#pragma once

#include "pic_internal.h"

namespace pic {
namespace {

template <int N>
__device__ __forceinline__ bool any_odd(const float (&o)[N]) {
  float sum = 0.f;
#pragma unroll
  for (int e = 0; e < N; ++e) sum += fabsf(o[e]);
  return !(sum < INFINITY);   // (or too large a sum: nothing is found then)
}
// o: joined from n partial sums, x(i, e) element e of the i-th
template <int N, typename X>
__device__ __forceinline__ void odd_partials(float (&o)[N], int n, X x) {
  if (!any_odd(o)) return;
  float sum[N] = {};
  for (int i = 0; i < n; ++i)
#pragma unroll
    for (int e = 0; e < N; ++e) {
      const float v = x(i, e);
      if (!(fabsf(v) < INFINITY)) sum[e] += v;
    }
#pragma unroll
  for (int e = 0; e < N; ++e)
    if (!(fabsf(sum[e]) < INFINITY)) o[e] = sum[e];
}
// The values of a row's 8 head dims that are not finite, into sum.
__device__ __forceinline__ void add_odd(uint4 row8, float (&sum)[8]) {
  const uint32_t w[4] = {row8.x, row8.y, row8.z, row8.w};
#pragma unroll
  for (int e = 0; e < 8; ++e) {
    const float v = __builtin_bit_cast(float, e & 1 ? w[e >> 1] & 0xFFFF0000u : w[e >> 1] << 16);
    if (!(fabsf(v) < INFINITY)) sum[e] += v;
  }
}
// By a whole wave: the sum of those of head dims 8 c .. + 7, c = lane % KC, over keys [k0, k1) (row(key): where a key's
// values lie); 0 where all are finite.  Eight rows a lane are on their way at once; keys past the last are that one
// again, which changes no such sum.
template <int KC, typename Row>
__device__ __forceinline__ void odd_values(Row row, int k0, int k1, float (&sum)[8]) {
  constexpr int kAhead = 8, kStep = 64 / KC;
  const int lane = threadIdx.x & 63;
  for (int key0 = k0 + lane / KC; key0 < k1; key0 += kAhead * kStep) {
    const bf16_t* at[kAhead];
    uint4 x[kAhead];
#pragma unroll
    for (int i = 0; i < kAhead; ++i) at[i] = row(min(key0 + i * kStep, k1 - 1)) + 8 * (lane % KC);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) x[i] = *reinterpret_cast<const uint4*>(at[i]);
#pragma unroll
    for (int i = 0; i < kAhead; ++i) add_odd(x[i], sum);
  }
#pragma unroll
  for (int off = KC; off < 64; off <<= 1)
#pragma unroll
    for (int e = 0; e < 8; ++e) sum[e] += __shfl_xor(sum[e], off, 64);
}

}  // namespace
}  // namespace pic
