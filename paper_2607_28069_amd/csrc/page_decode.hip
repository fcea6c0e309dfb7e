// Single-token decode attention over a cache handed out in pages, bf16 storage.
//
// As over a contiguous cache (decode_bf16.hip), a step reads every cached row once and is bound by HBM
// bandwidth: a workgroup of 4 waves covers one key range of one (layer, request, kv head), S^T = K Q^T
// and O^T = V^T P^T run on v_mfma_f32_16x16x32_bf16 with up to 16 query heads along N, K goes from memory
// straight into the A-operand layout, V through LDS with transposing reads, and a context split over
// workgroups leaves float32 partials for a combine.  What is different here:
//  * Pages hold 1 << shift >= 16 tokens, so a tile's two blocks of 16 keys lie in one page each and a
//    wave needs two page numbers per tile.  It holds 64 entries of the page table in a register (lane
//    j: entry win + j) and takes them out with readlane, the 64 after those on their way: no tile's
//    loads wait for the table.
//  * Equal ranges are those of the request's own keys, and a wave takes a quarter of its workgroup's, so
//    that short contexts use every workgroup and wave that the longest one has (37 requests of 70 to 701 keys
//    in a padded batch of 48, head_dim 64, two layers: 22.3 -> 19.6 us; one request of 10K keys where the
//    call allows 33K 24.1 -> 15.4, 16 of 5K where it allows 20K 81.9 -> 59.3; 16 of 8K to 16K 140 -> 146).
//  * Probabilities enter the product with V as two bfloat16 terms, the rounded value and what the
//    rounding left (2^-17 relative to the value then).  The matrix cores have the time: 0.5 to 2 %, and
//    the output's error against 64 bits falls from 0.0023 to that of its own rounding, 0.0017.  The rope
//    variant keeps two terms of its turned queries as well (0.3 to 1.5 %, 0.0024 -> 0.0017).
//  * A value that is not finite reaches the outputs in its head dim, whatever its probability (odd_values); the
//    merge sees it by 8 additions a thread, which do not show in any time.
//  * The new token is stored after the key loop, with a table entry that nothing waited for; the
//    queries are turned (rope variant) with the first tile's rows on their way.
//  * Requests with a negative length are padding of the batch: their workgroups leave at once, and
//    where ranges are dealt by length they get none.
#include <type_traits>

#include "decode_common.h"

namespace pic {
namespace {

struct PageDecodeArgs {
  const bf16_t* q;        // [L][B][Hq][D]
  const bf16_t* k_new;    // [L][B][Hkv][D]
  const bf16_t* v_new;
  bf16_t* pages_k;        // [L][Hkv][stream_rows][D]
  bf16_t* pages_v;
  PageMap map;
  const int32_t* base_len;
  bf16_t* out;            // [L][B][Hq][D]
  float* ws_o;            // [L][slots][D]   (n_splits > 1; slots = B Hq n_splits, see SplitDeal)
  float* ws_ml;           // [L][slots][2]
  int32_t batch, slot_cap, stream_rows, n_q_heads, n_kv_heads, max_base, step, n_splits;
  int32_t head_groups;    // groups of up to 16 query heads per kv head (ceil(n_rep / 16))
  EqualDeal eq;
  float scale_log2;
  const float2* table;    // rope variant: [L or 1][max_abs_delta + 1][D/2] cos/sin rows
  int64_t table_stride;
  int32_t max_abs_delta;
};

// grid (S * B * Hkv * head_groups, L), 256 threads.  kDealt: ranges dealt by length (decode_dealt), else
// n_splits equal ones.  The next tile of a wave is on its way while one is used, and no more: with two, or
// with the next one asked for before this one had arrived, launches were slower (one request of 10K keys
// 14.7 us -> 16.0 and 15.3, 16 of 10K 113 -> 117 and 114, 8 of up to 33K 84 -> 94 and 87).
template <int HD, bool kRope, bool kInterleaved, bool kDealt>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2)))
page_decode_kernel(PageDecodeArgs a) {
  constexpr int kRowBytes = Dims<HD>::kRowBytes, kVTileBytes = Dims<HD>::kVTileBytes;
  constexpr int KC = Dims<HD>::kChunks, KS = Dims<HD>::kSteps, DB = Dims<HD>::kBlocks;
  constexpr int RPM = Dims<HD>::kRowsPerMove;
  // (buffers of their own, so that the compiler sees that moves into one do not alias reads of another)
  __shared__ __attribute__((aligned(16))) uint8_t v_lds0[kWaves * kVTileBytes];
  __shared__ __attribute__((aligned(16))) uint8_t v_lds1[kWaves * kVTileBytes];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int hgrp = blockIdx.x % a.head_groups;           // query heads 16 hgrp .. of kv head g
  const int at = blockIdx.x / a.head_groups;             // [request][kv head][range]
  int b, g, split, chunk = 0;
  int32_t base;
  SplitPlace place;
  if constexpr (!kDealt) {
    split = at % a.n_splits;
    const int bg = at / a.n_splits;
    b = bg / a.n_kv_heads;
    g = bg % a.n_kv_heads;
    place = {a.n_splits, b * a.n_splits};
    base = a.base_len[b];
    if (base < 0) return;   // (uniform) padding of the batch
    base = min(base, a.max_base);
    chunk = decode_units(ceil_div(base + a.step + 1, a.n_splits)) * kDecodeUnit;   // (of this request's keys)
  } else {
    const SplitLens lens = split_lens<true>(a.base_len, a.batch, a.max_base, a.step, a.slot_cap);
    const int bg = at / a.eq.n;
    split = at % a.eq.n;
    b = bg / a.n_kv_heads;
    g = bg % a.n_kv_heads;
    place = {a.eq.n, b * a.eq.n};
    chunk = a.eq.chunk;
    if (!all_of(lens, a.eq.units, a.batch)) {
      const SplitDeal deal = deal_splits<true>(lens, a.batch, a.n_splits);
      if (deal.n == 0) return;   // (uniform) a batch of padding
      chunk = deal.chunk;
      if (deal.n > 0) {
        b = at / (deal.n * a.n_kv_heads);
        place = place_of(deal, b);
      } else {
        place = {0, 0};
        for (b = 0; b < a.batch; ++b) {
          place.n = __builtin_amdgcn_readlane(deal.mine, b);
          if (at < (place.first + place.n) * a.n_kv_heads) break;
          place.first += place.n;
        }
      }
      const int in_b = at - place.first * a.n_kv_heads;
      g = in_b / place.n;
      split = in_b - g * place.n;
    }
    if (b >= a.batch) return;   // (uniform) more workgroups than ranges
    base = __builtin_amdgcn_readlane(lens.base, b);
  }
  const int l = blockIdx.y;
  const int n_rep = a.n_q_heads / a.n_kv_heads;
  const int rep0 = 16 * hgrp;                             // first query head of this group
  const int n_here = min(16, n_rep - rep0);               // query heads of this group

  const int p = base + a.step;                       // the new token's slot (below slot_cap)
  const int n_vis = p + 1;
  const int wc0 = (int)min((int64_t)split * chunk, (int64_t)n_vis);
  const int wc1 = (int)min((int64_t)wc0 + chunk, (int64_t)n_vis);
  // a wave's keys: a quarter of those there are, in whole tiles
  const int sub = (wc1 - wc0 + kWaves * kTile - 1) / (kWaves * kTile) * kTile;
  const int c0 = min(wc0 + wave * sub, wc1);
  const int c1 = min(c0 + sub, wc1);

  // entries [win, win + 64) of the request's page table and the 64 after them; the entry of the new token
  const int32_t* ptab = a.map.table + (int64_t)b * a.map.cap;
  auto entry = [&](int32_t i) { return ptab[clamp_entry(i, a.map)]; };
  PageWindow win = {c0 >> a.map.shift};
  int32_t w_cur = entry(win.at + lane), w_next = entry(win.at + 64 + lane);
  const int32_t store_page = entry(p >> a.map.shift);
  // the row that slot k0 lies in: k0 uniform, a multiple of 16, never less than the one asked for before
  auto row_at = [&](int k0) -> int32_t {
    const int32_t i = k0 >> a.map.shift;
    if (win.moves(i, 64)) {
      w_cur = w_next;
      w_next = entry(win.at + 64 + lane);
    }
    const int32_t page = clamp_page(__builtin_amdgcn_readlane(w_cur, win.lane(i)), a.map);
    return (page << a.map.shift) + (k0 & ((1 << a.map.shift) - 1));
  };

  const int64_t new_row = ((int64_t)l * a.batch + b) * a.n_kv_heads + g;
  const int64_t row0 = ((int64_t)l * a.n_kv_heads + g) * a.stream_rows;
  const bf16_t* Kg = a.pages_k + row0 * HD;
  const bf16_t* Vg = a.pages_v + row0 * HD;
  const bf16_t* Kn = a.k_new + new_row * HD;
  const bf16_t* Vn = a.v_new + new_row * HD;
  const float2* trow = kRope ? a.table + (int64_t)l * a.table_stride + (int64_t)min(p, a.max_abs_delta) * (HD / 2)
                             : nullptr;   // rope variant: cos/sin of position p

  // Q^T operand: lane (n, g4) holds q[head g*n_rep + n][32 ks + 8 g4 .. +8)
  const int n = lane & 15, g4 = lane >> 4;
  bf16x8_t qop[KS];
  u32x4 qv[KS];
  {
    const bool ok = n < n_here;
    const int64_t qrow = ((int64_t)l * a.batch + b) * a.n_q_heads + g * n_rep + rep0 + (ok ? n : 0);
    const u32x4* qp = reinterpret_cast<const u32x4*>(a.q + qrow * HD);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qv[ks] = ok ? qp[4 * ks + g4] : u32x4{0, 0, 0, 0};
  }
  u32x4 q_lo[KS];   // rope variant: what rounding the turned query to bfloat16 left
  auto take_q = [&]() {
    if constexpr (kRope) rot_operand<HD, kInterleaved>(qv, trow, g4, &q_lo);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qop[ks] = as_bf16x8(qv[ks]);
  };

  // One tile's rows: K straight into the A-operand layout, [mb][ks] = key 16 mb + n, head dims
  // 32 ks + 8 g4 .. +8; V into this wave's part of an LDS buffer, instruction i filling rows RPM i .. RPM i +
  // RPM - 1 (RPM = 64 / KC rows of KC chunks), lane -> row RPM i + lane / KC, chunk slot lane % KC (holding
  // chunk slot ^ v_swz(row)).  Keys past the range are its last block's again (their scores are masked);
  // the new token's row comes from k_new / v_new.  K stays cached (a row in four 64-byte pieces), V (whole
  // rows per instruction) is non-temporal.
  const int ld_r = lane / KC, ld_slot = lane & (KC - 1);
  auto load = [&](int k0, u32x4 (&kr)[2][KS], uint8_t* buf) {
    int slot16[2];
    int64_t row16[2];
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
      slot16[mb] = min(k0 + 16 * mb, (c1 - 1) & ~15);
      row16[mb] = row_at(slot16[mb]);
    }
#pragma unroll
    for (int mb = 0; mb < 2; ++mb) {
      const int key = min(slot16[mb] + n, c1 - 1);
      const bf16_t* src = key == p ? Kn : Kg + (row16[mb] + (key - slot16[mb])) * HD;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kr[mb][ks] = *reinterpret_cast<const u32x4*>(src + 32 * ks + 8 * g4);
    }
#pragma unroll
    for (int i = 0; i < kTile / RPM; ++i) {
      const int rl = RPM * i + ld_r, mb = RPM * i / 16;
      const int key = min(slot16[mb] + (RPM * i & 15) + ld_r, c1 - 1);
      const bf16_t* src = (key == p ? Vn : Vg + (row16[mb] + (key - slot16[mb])) * HD) + 8 * (ld_slot ^ v_swz<HD>(rl));
      __builtin_amdgcn_global_load_lds((const GLOBAL_AS void*)src,
                                       (LDS_AS void*)(buf + wave * kVTileBytes + RPM * i * kRowBytes), 16, 0,
                                       kNonTemporal);
    }
  };

  // Transposing-read offsets: 16-lane group G = g4, lane j = 4 rr + qq points at row
  // 16 half + 4 G + rr, head dims 16 db + 4 qq .. +3; lane i then receives head dim 16 db + i.
  // Kept in registers: computed inline, the compiler makes these reads wait for the V loads in
  // flight into the other buffer.
  const int rr = (lane & 15) >> 2, qq = lane & 3;
  int v_rd[DB][2];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int row = 16 * half + 4 * g4 + rr;
      v_rd[db][half] = row * kRowBytes + (((2 * db + (qq >> 1)) ^ v_swz<HD>(row)) << 4) + 8 * (qq & 1);
    }

  f32x4_t oacc[DB];
#pragma unroll
  for (int i = 0; i < DB; ++i) oacc[i] = f32x4_t{};
  float m_run = kNoMax, l_part = 0.f;
  const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3F803F80u);

  // One tile at k0, resident in kcur and buffer P; the next one's loads are issued first, and have
  // arrived when it ends.
  auto tile = [&](int k0, auto parity, u32x4 (&kcur)[2][KS], u32x4 (&knext)[2][KS]) {
    constexpr int P = decltype(parity)::value;
    const uint8_t* vcur = P ? v_lds1 : v_lds0;
    if (k0 + kTile < c1) load(k0 + kTile, knext, P ? v_lds0 : v_lds1);
    if constexpr (kRope) {   // the new token's key, read unrotated from k_new, turned to p
      if (p >= k0 && p < k0 + kTile) {
#pragma unroll
        for (int mb = 0; mb < 2; ++mb)
          if (min(min(k0 + 16 * mb, (c1 - 1) & ~15) + n, c1 - 1) == p) rot_operand<HD, kInterleaved>(kcur[mb], trow, g4);
      }
    }
    f32x4_t sacc[2] = {f32x4_t{}, f32x4_t{}};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int mb = 0; mb < 2; ++mb) {
        sacc[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kcur[mb][ks]), qop[ks], sacc[mb], 0, 0, 0);
        if constexpr (kRope)
          sacc[mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kcur[mb][ks]), as_bf16x8(q_lo[ks]), sacc[mb], 0, 0, 0);
      }
    float mx = -INFINITY;
#pragma unroll
    for (int mb = 0; mb < 2; ++mb)
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        if (k0 + 16 * mb + 4 * g4 + e >= c1) sacc[mb][e] = -INFINITY;
        mx = fmaxf(mx, sacc[mb][e]);
      }
    mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
    mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
    const float m_tile = mx * a.scale_log2;
    if (__any(m_tile > m_run + 8.f)) {   // lazy reference max: p <= 2^8 (so values up to 2^120 over the number of keys)
      const float m_new = fmaxf(m_run, m_tile);
      const float alpha = __builtin_amdgcn_exp2f(m_run - m_new);
      m_run = m_new;
      l_part *= alpha;
#pragma unroll
      for (int db = 0; db < DB; ++db) oacc[db] *= alpha;
    }
    // probabilities in bfloat16, and what that rounding left
    uint32_t ph[4], pl[4];
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      const float p0 = __builtin_amdgcn_exp2f(fmaf(sacc[j >> 1][2 * (j & 1)], a.scale_log2, -m_run));
      const float p1 = __builtin_amdgcn_exp2f(fmaf(sacc[j >> 1][2 * (j & 1) + 1], a.scale_log2, -m_run));
      ph[j] = pack_bf16x2(p0, p1);
      pl[j] = pack_bf16x2(p0 - __uint_as_float(ph[j] << 16), p1 - __uint_as_float(ph[j] & 0xFFFF0000u));
    }
#pragma unroll
    for (int j = 0; j < 4; ++j) {
      l_part = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, ph[j]), ones, l_part, false);
      l_part = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pl[j]), ones, l_part, false);
    }
    // P^T operands: k index 8 g4 + j <-> key 16 (j / 4) + 4 g4 + j % 4 (accumulator order)
    const bf16x8_t pop_h = as_bf16x8(u32x4{ph[0], ph[1], ph[2], ph[3]});
    const bf16x8_t pop_l = as_bf16x8(u32x4{pl[0], pl[1], pl[2], pl[3]});
    const uint8_t* vw = vcur + wave * kVTileBytes;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS i16x4*)(vw + v_rd[db][0]));
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS i16x4*)(vw + v_rd[db][1]));
      const bf16x8_t vv = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      oacc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pop_h, oacc[db], 0, 0, 0);
      oacc[db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pop_l, oacc[db], 0, 0, 0);
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0)
  };

  u32x4 k_a[2][KS], k_b[2][KS];
  if (c0 < c1) {
    load(c0, k_a, v_lds0);
    take_q();
    __builtin_amdgcn_s_waitcnt(0x0F70);
    for (int k0 = c0; k0 < c1; k0 += 2 * kTile) {
      tile(k0, std::integral_constant<int, 0>{}, k_a, k_b);
      if (k0 + kTile < c1) tile(k0 + kTile, std::integral_constant<int, 1>{}, k_b, k_a);
    }
  }

  // The workgroup holding slot p stores the new token.  Nobody reads that row from the pages during
  // this launch: the wave whose range holds it reads k_new / v_new.
  if (hgrp == 0 && p >= wc0 && p < wc1 && wave == 0 && lane < 2 * KC && store_page >= 0 && store_page < a.map.n_pages) {
    const int c = lane & (KC - 1);   // lanes [0, KC): K chunks, [KC, 2 KC): V chunks
    const int64_t row = row0 + ((int64_t)store_page << a.map.shift) + (p & ((1 << a.map.shift) - 1));
    u32x4* dst = reinterpret_cast<u32x4*>((lane < KC ? a.pages_k : a.pages_v) + row * HD);
    if (kRope && lane < KC) {   // the new key turned to p: lane c < KC/2 takes a chunk pair
      if (c < KC / 2) {
        // rotate-half: chunks c, c + KC/2 (frequencies 8 c ..); interleaved: 2 c, 2 c + 1 (8 c ..)
        const int ca = kInterleaved ? 2 * c : c, cb = kInterleaved ? 2 * c + 1 : c + KC / 2;
        float x[8], y[8];
        unpack8(reinterpret_cast<const u32x4*>(Kn)[ca], x);
        unpack8(reinterpret_cast<const u32x4*>(Kn)[cb], y);
#pragma unroll
        for (int i = 0; i < 8; ++i) {
          const float2 cs = trow[8 * c + i];
          if constexpr (kInterleaved) {
            float* z = i < 4 ? x : y;
            rot_pair(z[2 * (i & 3)], z[2 * (i & 3) + 1], cs.x, cs.y);
          } else {
            rot_pair(x[i], y[i], cs.x, cs.y);
          }
        }
        dst[ca] = pack8(x);
        dst[cb] = pack8(y);
      }
    } else {
      dst[c] = reinterpret_cast<const u32x4*>(lane < KC ? Kn : Vn)[c];
    }
  }

  // ---- merge the 4 waves (log-sum-exp) through LDS, reusing the V buffers
  float l_tot = l_part + __shfl_xor(l_part, 16, 64);
  l_tot += __shfl_xor(l_tot, 32, 64);
  __syncthreads();
  // [4][16][HD] fp32, all of v_lds0; 16-byte chunk c of row r at c ^ r: a store's rows would meet in one
  // bank otherwise
  auto o_lds = [&](int w, int r, int c) { return reinterpret_cast<f32x4_t*>(v_lds0) + (w * 16 + r) * (HD / 4) + (c ^ r); };
  float* ml_lds = reinterpret_cast<float*>(v_lds1);   // [4][16][2]
  if (n < n_here) {
#pragma unroll
    for (int db = 0; db < DB; ++db)
      *o_lds(wave, n, 4 * db + g4) = oacc[db];
    if (g4 == 0) {
      ml_lds[(wave * 16 + n) * 2] = m_run;
      ml_lds[(wave * 16 + n) * 2 + 1] = l_tot;
    }
  }
  __syncthreads();
  // thread -> (query n = tid / KC, head dims 8 (tid % KC) .. +8)
  const int mn = tid / KC, md = 8 * (tid & (KC - 1));
  float M = kNoMax, den = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  if (mn < n_here) {
#pragma unroll
    for (int w = 0; w < kWaves; ++w) M = fmaxf(M, ml_lds[(w * 16 + mn) * 2]);
#pragma unroll
    for (int w = 0; w < kWaves; ++w) {
      const float wt = __builtin_amdgcn_exp2f(ml_lds[(w * 16 + mn) * 2] - M);
      den += wt * ml_lds[(w * 16 + mn) * 2 + 1];
      const f32x4_t x0 = *o_lds(w, mn, md / 4), x1 = *o_lds(w, mn, md / 4 + 1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[e] += wt * x0[e];
        o[4 + e] += wt * x1[e];
      }
    }
  }
  // values that are not finite (where the scores are: else the outputs are NaN anyway)
  if (__any(any_odd(o) && fabsf(den) < INFINITY)) {
    float v[8] = {};
    odd_values<KC>([&](int key) { return key == p ? Vn : Vg + page_row(a.map, b, key) * HD; }, wc0, wc1, v);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!(fabsf(v[e]) < INFINITY)) o[e] = v[e];
  }
  if (mn < n_here) {
    const int64_t row = ((int64_t)l * a.batch + b) * a.n_q_heads + g * n_rep + rep0 + mn;
    if (place.n == 1) {
      const float inv = 1.f / den;
      *reinterpret_cast<u32x4*>(a.out + row * HD + md) =
          u32x4{pack_bf16x2(o[0] * inv, o[1] * inv), pack_bf16x2(o[2] * inv, o[3] * inv),
                pack_bf16x2(o[4] * inv, o[5] * inv), pack_bf16x2(o[6] * inv, o[7] * inv)};
    } else {
      const int64_t slot = ((int64_t)l * a.batch * a.n_splits + place.first) * a.n_q_heads +
                           (int64_t)(g * n_rep + rep0 + mn) * place.n + split;
      float* wo = a.ws_o + slot * HD + md;
      *reinterpret_cast<float4*>(wo) = make_float4(o[0], o[1], o[2], o[3]);
      *reinterpret_cast<float4*>(wo + 4) = make_float4(o[4], o[5], o[6], o[7]);
      if (md == 0) *reinterpret_cast<float2*>(a.ws_ml + 2 * slot) = make_float2(M, den);
    }
  }
}

template <int HD, bool kDealt>
hipError_t launch_as(const PageDecodeArgs& a, dim3 grid, bool interleaved, const AttnShape& s, hipStream_t stream) {
  if (!a.table)
    hipLaunchKernelGGL((page_decode_kernel<HD, false, false, kDealt>), grid, dim3(256), 0, stream, a);
  else if (interleaved)
    hipLaunchKernelGGL((page_decode_kernel<HD, true, true, kDealt>), grid, dim3(256), 0, stream, a);
  else
    hipLaunchKernelGGL((page_decode_kernel<HD, true, false, kDealt>), grid, dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_splits == 1) return e;
  return launch_decode_combine<HD, kDealt, true>(a.ws_o, a.ws_ml, a.base_len, s, a.max_base, a.step, a.slot_cap, a.n_splits,
                                                 a.eq, a.out, stream);
}

template <int HD>
hipError_t launch_hd(const PageDecodeArgs& a, dim3 grid, bool interleaved, const AttnShape& s, hipStream_t stream) {
  const bool dealt = decode_dealt(a.n_splits, a.batch, a.max_base + a.step + 1);
  return dealt ? launch_as<HD, true>(a, grid, interleaved, s, stream) : launch_as<HD, false>(a, grid, interleaved, s, stream);
}

}  // namespace

hipError_t launch_decode_bf16_pages(const PageAttnArgs& p) {
  const AttnShape& s = p.s;
  const int32_t max_len = p.max_base + p.offset + 1;
  PageDecodeArgs a = {};
  a.q = static_cast<const bf16_t*>(p.q);
  a.k_new = static_cast<const bf16_t*>(p.k_new);
  a.v_new = static_cast<const bf16_t*>(p.v_new);
  a.pages_k = static_cast<bf16_t*>(p.pages_k);
  a.pages_v = static_cast<bf16_t*>(p.pages_v);
  a.map = p.map;
  a.base_len = p.base_len;
  a.out = static_cast<bf16_t*>(p.out);
  const size_t rows = (size_t)s.n_layers * s.batch * s.n_q_heads * p.n_splits;
  a.ws_o = static_cast<float*>(p.workspace);
  a.ws_ml = a.ws_o ? a.ws_o + rows * s.head_dim : nullptr;
  a.batch = s.batch;
  a.slot_cap = (int32_t)std::min((int64_t)p.map.cap << p.map.shift, (int64_t)INT32_MAX);
  a.stream_rows = s.cache_cap;
  a.n_q_heads = s.n_q_heads;
  a.n_kv_heads = s.n_kv_heads;
  a.max_base = p.max_base;
  a.step = p.offset;
  a.n_splits = p.n_splits;
  if (decode_dealt(p.n_splits, s.batch, max_len)) {
    a.eq.units = decode_units(std::min(max_len, a.slot_cap));
    const int32_t per = ceil_div(a.eq.units, std::min(p.n_splits, a.eq.units));   // units per range
    a.eq.n = ceil_div(a.eq.units, per);
    a.eq.chunk = per * kDecodeUnit;
  }
  a.scale_log2 = s.scale_log2;
  a.head_groups = decode_head_groups(s);
  a.table = p.table;
  a.table_stride = p.table_stride;
  a.max_abs_delta = p.max_abs_delta;
  const dim3 grid(a.head_groups * p.n_splits * s.batch * s.n_kv_heads, s.n_layers);
  return s.head_dim == 64 ? launch_hd<64>(a, grid, p.interleaved, s, p.stream) : launch_hd<128>(a, grid, p.interleaved, s, p.stream);
}

}  // namespace pic
