// What the bf16 decode kernels over contiguous and over paged caches share: tile sizes, the ranges of a
// split launch dealt by length, rotation of operands, and the combine of a split launch.
#pragma once

#include <algorithm>

#include "odd_values.h"
#include "pic_bounds.h"
#include "pic_internal.h"

namespace pic {
namespace {

constexpr int kWaves = 4;
constexpr int kTile = 32;                          // keys per wave tile
constexpr int kMinWaveKeys = 64;
// Sizes that follow the head dim HD (128 or 64): a row is HD/8 16-byte chunks; a lane's
// operands hold HD/32 steps of 32 head dims; the output is HD/16 blocks of 16 head dims.
template <int HD>
struct Dims {
  static_assert(HD == 128 || HD == 64, "head_dim 128 or 64");
  static constexpr int kRowBytes = HD * 2;                  // 256 or 128
  static constexpr int kVTileBytes = kTile * kRowBytes;     // per wave per buffer
  static constexpr int kChunks = HD / 8;                    // 16-byte chunks per row
  static constexpr int kSteps = HD / 32;                    // k steps of Q^T / K operands
  static constexpr int kBlocks = HD / 16;                   // 16-dim output blocks
  static constexpr int kRowsPerMove = 64 / kChunks;         // rows one 1 KB V move fills
};
static_assert(kDecodeUnit == kWaves * kTile, "a unit is one tile per wave");
static_assert(kWaves == kDecodeWaves && kMinWaveKeys == kDecodeMinWaveKeys, "host split planner tiling");
constexpr int kNonTemporal = 2;                    // cache-policy bits of a streaming load
// Decode over pages: the reference maximum of a row before its first key.  Finite, so that a row without keys, or
// whose scores are all -inf, has probabilities, and in a merge a weight, of 0 times 0, and one whose scores
// are NaN (which a maximum passes over) brings its NaN sums into the merge.
constexpr float kNoMax = -3.402823466e38f;

#define LDS_AS __attribute__((address_space(3)))
#define GLOBAL_AS __attribute__((address_space(1)))

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));
typedef short i16x4 __attribute__((ext_vector_type(4)));
__device__ __forceinline__ bf16x8_t as_bf16x8(u32x4 v) { return __builtin_bit_cast(bf16x8_t, v); }

// 16-byte chunk c of V row `key` sits at slot c ^ v_swz(key) of its row in LDS (256-byte rows:
// 16 slots; 128-byte rows: 8 slots, so the XOR keeps to the low three bits).
template <int HD>
__device__ __forceinline__ int v_swz(int key) {
  if constexpr (HD == 128) return ((key & 3) << 1) | (((key >> 2) & 1) << 3);
  else return (key & 3) << 1;
}

// The dealt ranges of a batch whose contexts all have the greatest length the call allows.
struct EqualDeal {
  int32_t units, n, chunk;   // units of every context, its ranges, keys per range
};

// How the key ranges of a split launch are dealt to the requests (pic_bounds.h): worked out by
// every wave from the context lengths, request b in lane b.  Request b's partials are slots
// [Hq first, Hq (first + n)), query head by query head.  Contexts of one length take a short way to
// the same ranges (the long one costs about 0.5 us, paid in the kernel and its combine), and where that
// is the greatest length the host has worked them out (EqualDeal): the place follows, and the combine
// loads its partials, while the lengths are on their way.
struct SplitDeal {
  int32_t chunk;   // keys per range, a multiple of 128
  int32_t n;       // ranges of every request; -1: lane b holds those of request b in mine
  int32_t mine;
};
struct SplitLens {
  int32_t u, base;   // lane b: request b's units and context length
};
struct SplitPlace {
  int32_t n, first;   // ranges of the request; those of the requests before it
};
// kPages: a negative length is padding of the batch and gets no range
template <bool kPages>
__device__ __forceinline__ SplitLens split_lens(const int32_t* base_len, int32_t batch, int32_t max_base, int32_t step,
                                                int32_t cache_cap) {
  const int lane = threadIdx.x & 63;
  SplitLens x = {0, 0};
  if (lane < batch) {
    const int32_t len = base_len[lane];
    x.base = clamp_len(len, max_base);
    if (!kPages || len >= 0) x.u = decode_units(min(x.base + step + 1, cache_cap));
  }
  return x;
}
__device__ __forceinline__ bool all_of(const SplitLens& x, int32_t units, int32_t batch) {
  return __ballot((int)(threadIdx.x & 63) < batch && x.u != units) == 0;
}
template <bool kPages>
__device__ __forceinline__ SplitDeal deal_splits(const SplitLens& x, int32_t batch, int32_t n_splits) {
  const int lane = threadIdx.x & 63;
  const int32_t u = x.u, u0 = __builtin_amdgcn_readfirstlane(u);
  if (all_of(x, u0, batch)) {
    if (kPages && u0 == 0) return {kDecodeUnit, 0, 0};   // nothing but padding
    const int32_t s = min(n_splits, u0), cu = __builtin_amdgcn_readfirstlane(ceil_div24(u0, s, __builtin_amdgcn_rcpf((float)s)));
    return {cu * kDecodeUnit, __builtin_amdgcn_readfirstlane(ceil_div24(u0, cu, __builtin_amdgcn_rcpf((float)cu))), 0};
  }
  int32_t total = 0, longest = 0;
  for (int b = 0; b < batch; ++b) {
    const int32_t ub = __builtin_amdgcn_readlane(u, b);
    total += ub;
    longest = max(longest, ub);
  }
  const RangeCandidates rc = decode_range_candidates(total, longest, n_splits, batch);
  const int32_t c = rc.at(lane);   // lane i weighs candidate i
  const float inv = __builtin_amdgcn_rcpf((float)c);
  int32_t sum = 0;
  for (int b = 0; b < batch; ++b) sum += ceil_div24(__builtin_amdgcn_readlane(u, b), c, inv);
  const uint64_t fits = __ballot(sum <= n_splits * batch);   // (lane 63: always)
  const int32_t cu = __builtin_amdgcn_readlane(c, __ffsll((unsigned long long)fits) - 1);
  return {cu * kDecodeUnit, -1, ceil_div24(u, cu, __builtin_amdgcn_rcpf((float)cu))};
}
__device__ __forceinline__ SplitPlace place_of(const SplitDeal& d, int b) {   // b uniform
  if (d.n >= 0) return {d.n, b * d.n};
  SplitPlace p = {__builtin_amdgcn_readlane(d.mine, b), 0};
  for (int i = 0; i < b; ++i) p.first += __builtin_amdgcn_readlane(d.mine, i);
  return p;
}

// (x, y) turned by (c, s) in the float32 form of the re-rotation kernel.
__device__ __forceinline__ void rot_pair(float& x, float& y, float c, float s) {
  const float u = x, v = y;
  x = fmaf(u, c, -(v * s));
  y = fmaf(u, s, v * c);
}
__device__ __forceinline__ void unpack8(u32x4 w, float (&x)[8]) {
#pragma unroll
  for (int e = 0; e < 4; ++e) {
    x[2 * e] = __uint_as_float(w[e] << 16);
    x[2 * e + 1] = __uint_as_float(w[e] & 0xFFFF0000u);
  }
}
__device__ __forceinline__ u32x4 pack8(const float (&x)[8]) {
  return u32x4{pack_bf16x2(x[0], x[1]), pack_bf16x2(x[2], x[3]), pack_bf16x2(x[4], x[5]),
               pack_bf16x2(x[6], x[7])};
}
// x in two bfloat16 terms
__device__ __forceinline__ void pack8_terms(const float (&x)[8], u32x4& hi, u32x4& lo) {
  float h[8], r[8];
  hi = pack8(x);
  unpack8(hi, h);
#pragma unroll
  for (int e = 0; e < 8; ++e) r[e] = x[e] - h[e];
  lo = pack8(r);
}
// The head dims 32 ks + 8 g4 .. + 8 (ks < HD/32) a lane holds of one row (the A / B operand
// layout below), turned by row `trow` of the table: rotate-half pairs are chunks ks and
// ks + HD/64 (frequencies 32 ks + 8 g4 + j), interleaved pairs sit inside a chunk (16 ks + 4 g4 + m).
// With `lo`, what the rounding to bfloat16 leaves.
template <int HD, bool kInterleaved>
__device__ __forceinline__ void rot_operand(u32x4 (&c)[Dims<HD>::kSteps], const float2* trow, int g4,
                                            u32x4 (*lo)[Dims<HD>::kSteps] = nullptr) {
  constexpr int KS = Dims<HD>::kSteps;
  auto put = [&](int ks, const float (&x)[8]) {
    if (lo) pack8_terms(x, c[ks], (*lo)[ks]);
    else c[ks] = pack8(x);
  };
  if constexpr (!kInterleaved) {
#pragma unroll
    for (int ks = 0; ks < KS / 2; ++ks) {
      float x[8], y[8];
      unpack8(c[ks], x);
      unpack8(c[ks + KS / 2], y);
#pragma unroll
      for (int j = 0; j < 8; ++j) {
        const float2 cs = trow[32 * ks + 8 * g4 + j];
        rot_pair(x[j], y[j], cs.x, cs.y);
      }
      put(ks, x);
      put(ks + KS / 2, y);
    }
  } else {
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) {
      float x[8];
      unpack8(c[ks], x);
#pragma unroll
      for (int m = 0; m < 4; ++m) {
        const float2 cs = trow[16 * ks + 4 * g4 + m];
        rot_pair(x[2 * m], x[2 * m + 1], cs.x, cs.y);
      }
      put(ks, x);
    }
  }
}

// grid (rows, L), 256 threads, rows [row0, row0 + grid) of the B * Hq: merge the ranges of one query
// head by log-sum-exp.  HD / 4 lanes
// hold 4 head dims each of one range, 1024 / HD ranges side by side, and every range's loads are
// issued before any is used; the range groups then merge in LDS.  (One wave walking the ranges
// took 4.9 us for 8 or 32 of them: a memory round trip per 8, once for the maxima and once for
// the sums.)  A range that saw no key (maximum -inf; over pages kNoMax and sums of 0) adds nothing.
// (pages, heads > 0: `heads` query rows for each of n_new tokens per request, n_q_heads counting them all)
struct FewTokens {
  const int32_t* n_valid = nullptr;
  int32_t n_new = 1, heads = 0;
};
template <int HD, bool kDealt, bool kPages>
__global__ void __launch_bounds__(256) decode_combine_kernel(const float* __restrict__ ws_o,
                                                             const float* __restrict__ ws_ml,
                                                             const int32_t* __restrict__ base_len, int32_t batch,
                                                             int32_t n_q_heads, int32_t max_base, int32_t step,
                                                             int32_t cache_cap, int32_t n_splits, EqualDeal eq,
                                                             int32_t row0, bf16_t* __restrict__ out, FewTokens few) {
  constexpr int kLanes = HD / 4, kGroups = 256 / kLanes, kBatch = 4;
  __shared__ float m_s[kGroups], l_s[kGroups];
  __shared__ __attribute__((aligned(16))) float o_s[kGroups * HD];
  const int bh = row0 + blockIdx.x, b = bh / n_q_heads, h = bh - b * n_q_heads, l = blockIdx.y;
  const int grp = threadIdx.x / kLanes, d = 4 * (threadIdx.x % kLanes);
  const int64_t layer0 = (int64_t)l * batch * n_splits * n_q_heads;   // (slots)
  const int32_t n0 = kDealt ? eq.n : n_splits;
  SplitPlace place = {n0, b * n0};
  float2 ml[kBatch];
  f32x4_t x[kBatch];
  auto load = [&](int s0) {
    const int64_t slot0 = layer0 + (int64_t)place.first * n_q_heads + (int64_t)h * place.n;
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      const int s = s0 + u * kGroups;
      ml[u] = s < place.n ? *reinterpret_cast<const float2*>(ws_ml + 2 * (slot0 + s)) : make_float2(-INFINITY, 0.f);
      x[u] = s < place.n ? *reinterpret_cast<const f32x4_t*>(ws_o + (slot0 + s) * HD + d) : f32x4_t{};
    }
  };
  if constexpr (kDealt) {
    const SplitLens lens = split_lens<kPages>(base_len, batch, max_base, step, cache_cap);
    load(grp);   // (equal ranges fit the array whatever the lengths are)
    if (!all_of(lens, eq.units, batch)) {
      place = place_of(deal_splits<kPages>(lens, batch, n_splits), b);
      load(grp);
    }
    // (uniform) a whole request: its output is stored; padding: there is none
    if (kPages ? place.n <= 1 : place.n == 1) return;
  } else {
    load(grp);
    // (uniform) padding of the batch, or of the request's tokens
    if (kPages && (few.heads > 0 ? h / few.heads >= page_new_tokens(base_len, few.n_valid, b, few.n_new) : base_len[b] < 0))
      return;
  }
  float M = -INFINITY, den = 0.f;
  f32x4_t o = {};
  for (int s0 = grp; s0 < place.n; s0 += kBatch * kGroups) {
    if (s0 != grp) load(s0);
#pragma unroll
    for (int u = 0; u < kBatch; ++u) {
      if (ml[u].x == -INFINITY) continue;
      const float m_new = fmaxf(M, ml[u].x);
      const float keep = __builtin_amdgcn_exp2f(M - m_new), w = __builtin_amdgcn_exp2f(ml[u].x - m_new);
      M = m_new;
      den = den * keep + w * ml[u].y;
      o = o * keep + w * x[u];
    }
  }
  if constexpr (kPages) {
    const int64_t slot0 = layer0 + (int64_t)place.first * n_q_heads + (int64_t)h * place.n;
    float y[4] = {o[0], o[1], o[2], o[3]};
    odd_partials(y, (place.n - grp + kGroups - 1) / kGroups, [&](int i, int e) { return ws_o[(slot0 + grp + i * kGroups) * HD + d + e]; });
    o = f32x4_t{y[0], y[1], y[2], y[3]};
  }
  *reinterpret_cast<f32x4_t*>(o_s + grp * HD + d) = o;
  if (d == 0) {
    m_s[grp] = M;
    l_s[grp] = den;
  }
  __syncthreads();
  if (threadIdx.x >= HD / 2) return;
  float m_all = -INFINITY;
#pragma unroll
  for (int g = 0; g < kGroups; ++g) m_all = fmaxf(m_all, m_s[g]);
  float l_all = 0.f, y[2] = {0.f, 0.f};
#pragma unroll
  for (int g = 0; g < kGroups; ++g) {
    if (m_s[g] == -INFINITY) continue;
    const float w = __builtin_amdgcn_exp2f(m_s[g] - m_all);
    l_all += w * l_s[g];
    y[0] += w * o_s[g * HD + 2 * threadIdx.x];
    y[1] += w * o_s[g * HD + 2 * threadIdx.x + 1];
  }
  if constexpr (kPages) odd_partials(y, kGroups, [&](int g, int e) { return o_s[g * HD + 2 * threadIdx.x + e]; });
  const float inv = 1.f / l_all;
  const int64_t row = ((int64_t)l * batch + b) * n_q_heads + h;
  reinterpret_cast<uint32_t*>(out + row * HD)[threadIdx.x] = pack_bf16x2(y[0] * inv, y[1] * inv);
}


// One combine launch for every query row of a split launch.
template <int HD, bool kDealt, bool kPages>
hipError_t launch_decode_combine(const float* ws_o, const float* ws_ml, const int32_t* base_len, const AttnShape& s,
                                 int32_t max_base, int32_t step, int32_t cache_cap, int32_t n_splits, const EqualDeal& eq,
                                 bf16_t* out, hipStream_t stream, const FewTokens& few = FewTokens()) {
  // (a grid holds fewer than 2^32 threads per dimension)
  hipError_t e = hipSuccess;
  const int64_t rows = (int64_t)s.batch * s.n_q_heads, kPart = int64_t(1) << 23;
  for (int64_t row0 = 0; row0 < rows && e == hipSuccess; row0 += kPart) {
    hipLaunchKernelGGL((decode_combine_kernel<HD, kDealt, kPages>), dim3((unsigned)std::min(rows - row0, kPart), s.n_layers),
                       dim3(256), 0, stream, ws_o, ws_ml, base_len, s.batch, s.n_q_heads, max_base, step, cache_cap, n_splits,
                       eq, (int32_t)row0, out, few);
    e = hipGetLastError();
  }
  return e;
}

}  // namespace
}  // namespace pic
