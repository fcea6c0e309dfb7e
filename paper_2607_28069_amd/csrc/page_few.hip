// Attention of a few new tokens per request over a cache handed out in pages, bf16 storage: at most 32
// query rows per kv head (drafted tokens to be checked, the last piece of a prompt, one token of a model
// with many query heads per kv head).
//
// The prefill kernel gives each of its 8 waves 32 query rows and shares every key tile among them; of so few
// rows it would feed one wave, which needs about 1 us for a tile's products and exponentials
// whatever the loads do.  Here, as in decode, every wave takes all the rows and an eighth of the workgroup's keys,
// and the waves' results merge by log-sum-exp: the launch is bound by the bytes of K and V again.
//  * Row r = token r / n_rep, head r % n_rep, along N of v_mfma_f32_16x16x32_bf16 in one or two blocks of
//    16; tiles, page numbers, K and V moves, and probabilities and turned queries in two terms as in
//    page_decode.hip.
//  * A row sees the keys up to its own token: the last tiles are masked per row, and a row that a wave's
//    keys all lie past keeps its first reference maximum there and adds nothing.
//  * A probability of 0 times a value that is not finite is no 0: new tokens' values that are not finite
//    are cleared in LDS, so that rows that do not see them stay as they are.  Those, and cached ones, reach the rows
//    that see them when the waves merge (odd_values).
//  * The new tokens' rows come from k_new / v_new (keys turned on load in the rope variant) and are stored
//    into their pages by the workgroup whose range holds them.
#include <type_traits>

#include "decode_common.h"

namespace pic {
namespace {

constexpr int kFewWaves = 8, kFewThreads = 64 * kFewWaves;

struct PageFewArgs {
  const bf16_t* q;        // [L][B][n_new][Hq][D]
  const bf16_t* k_new;    // [L][B][n_new][Hkv][D]
  const bf16_t* v_new;
  bf16_t* pages_k;        // [L][Hkv][stream_rows][D]
  bf16_t* pages_v;
  PageMap map;
  const int32_t* ctx_len;
  const int32_t* n_valid;
  bf16_t* out;            // [L][B][n_new][Hq][D]
  float* ws_o;            // [L][B][n_new][Hq][n_splits][D]   (n_splits > 1)
  float* ws_ml;           // [L][B][n_new][Hq][n_splits][2]
  int32_t batch, stream_rows, n_q_heads, n_kv_heads, n_new, max_ctx, n_splits;
  float scale_log2;
  const float2* table;    // rope variant: [L or 1][max_abs_delta + 1][D/2] cos/sin rows
  int64_t table_stride;
  int32_t max_abs_delta;
};

// grid (n_splits * B * Hkv, L), 512 threads; NB blocks of 16 query rows
template <int HD, int NB, bool kRope, bool kInterleaved>
__global__ void __launch_bounds__(kFewThreads) __attribute__((amdgpu_waves_per_eu(2, 2)))
page_few_kernel(PageFewArgs a) {
  constexpr int kRowBytes = Dims<HD>::kRowBytes, kVTileBytes = Dims<HD>::kVTileBytes;
  constexpr int KC = Dims<HD>::kChunks, KS = Dims<HD>::kSteps, DB = Dims<HD>::kBlocks;
  constexpr int RPM = Dims<HD>::kRowsPerMove, ROWS = 16 * NB;
  __shared__ __attribute__((aligned(16))) uint8_t v_lds0[kFewWaves * kVTileBytes];
  __shared__ __attribute__((aligned(16))) uint8_t v_lds1[kFewWaves * kVTileBytes];
  __shared__ float ml_lds[kFewWaves * ROWS * 2];
  __shared__ bool odd_lds[kFewWaves];   // a value of the new tokens in a wave's keys was not finite
  // rope variant: the turned queries in two bfloat16 terms, the same in every wave; at head_dim 128 those of two
  // blocks of rows have no room in registers (16 requests of 10K x 8 tokens 165 us; the second terms in LDS 132,
  // both 126)
  constexpr bool kQueryLds = kRope && HD == 128 && NB == 2;
  __shared__ __attribute__((aligned(16))) u32x4 q_lds[kQueryLds ? 2 * NB * KS * 64 : 1];

  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int split = blockIdx.x % a.n_splits, bg = blockIdx.x / a.n_splits;
  const int b = bg / a.n_kv_heads, g = bg % a.n_kv_heads, l = blockIdx.y;
  const int n_tok = page_new_tokens(a.ctx_len, a.n_valid, b, a.n_new);
  if (n_tok == 0) return;   // (uniform) padding of the batch
  const int ctx = clamp_len(a.ctx_len[b], a.max_ctx);
  const int n_rep = a.n_q_heads / a.n_kv_heads, M = n_tok * n_rep;   // M <= ROWS
  const int n_vis = ctx + n_tok;
  const int chunk = decode_units(ceil_div(n_vis, a.n_splits)) * kDecodeUnit;   // (equal ranges of this request's keys)
  const int wc0 = (int)min((int64_t)split * chunk, (int64_t)n_vis);
  const int wc1 = (int)min((int64_t)wc0 + chunk, (int64_t)n_vis);
  // a wave's keys: an eighth of those there are, in whole tiles
  const int sub = (wc1 - wc0 + kFewWaves * kTile - 1) / (kFewWaves * kTile) * kTile;
  const int c0 = min(wc0 + wave * sub, wc1);
  const int c1 = min(c0 + sub, wc1);

  // entries [win, win + 64) of the request's page table and the 64 after them
  const int32_t* ptab = a.map.table + (int64_t)b * a.map.cap;
  auto entry = [&](int32_t i) { return ptab[clamp_entry(i, a.map)]; };
  PageWindow win = {c0 >> a.map.shift};
  int32_t w_cur = entry(win.at + lane), w_next = entry(win.at + 64 + lane);
  // the new tokens this workgroup stores, [st0, st1), 2 KC threads each, and the page of this thread's first
  const int st0 = min(max(wc0 - ctx, 0), n_tok), st1 = min(max(wc1 - ctx, 0), n_tok);
  const int st_i = st0 + tid / (2 * KC);
  const int32_t st_page = entry((ctx + st_i) >> a.map.shift);
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

  const int64_t row0 = ((int64_t)l * a.n_kv_heads + g) * a.stream_rows;
  const bf16_t* Kg = a.pages_k + row0 * HD;
  const bf16_t* Vg = a.pages_v + row0 * HD;
  const int64_t new0 = (((int64_t)l * a.batch + b) * a.n_new * a.n_kv_heads + g) * HD, new_stride = (int64_t)a.n_kv_heads * HD;
  const bf16_t* Kn = a.k_new + new0;
  const bf16_t* Vn = a.v_new + new0;
  const float2* tab = kRope ? a.table + (int64_t)l * a.table_stride : nullptr;
  auto trow = [&](int pos) { return tab + (int64_t)min(pos, a.max_abs_delta) * (HD / 2); };   // cos/sin of a position

  // Q^T operands: lane (n, g4) of block nb holds row 16 nb + n, head dims 32 ks + 8 g4 .. +8
  const int n = lane & 15, g4 = lane >> 4;
  bf16x8_t qop[NB][KS];
  u32x4 qv[NB][KS];
  int qpos[NB];
  // row of q / out of packed row r (token r / n_rep, head g n_rep + r % n_rep)
  auto row_of = [&](int r) {
    const int tok = r / n_rep;
    return (((int64_t)l * a.batch + b) * a.n_new + tok) * a.n_q_heads + g * n_rep + (r - tok * n_rep);
  };
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = 16 * nb + n;
    const bool ok = r < M;
    qpos[nb] = ctx + (ok ? r / n_rep : n_tok - 1);
    const u32x4* qp = reinterpret_cast<const u32x4*>(a.q + row_of(ok ? r : 0) * HD);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qv[nb][ks] = ok ? qp[4 * ks + g4] : u32x4{0, 0, 0, 0};
  }
  u32x4 q_lo[NB][KS];
  auto take_q = [&]() {
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      if constexpr (kRope) rot_operand<HD, kInterleaved>(qv[nb], trow(qpos[nb]), g4, &q_lo[nb]);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) {
        qop[nb][ks] = as_bf16x8(qv[nb][ks]);
        if constexpr (kQueryLds) {   // (all waves write the same)
          q_lds[(nb * KS + ks) * 64 + lane] = qv[nb][ks];
          q_lds[((NB + nb) * KS + ks) * 64 + lane] = q_lo[nb][ks];
        }
      }
    }
  };

  // One tile's rows, as in page_decode.hip
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
      const bf16_t* src = key >= ctx ? Kn + (key - ctx) * new_stride : Kg + (row16[mb] + (key - slot16[mb])) * HD;
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kr[mb][ks] = *reinterpret_cast<const u32x4*>(src + 32 * ks + 8 * g4);
    }
#pragma unroll
    for (int i = 0; i < kTile / RPM; ++i) {
      const int rl = RPM * i + ld_r, mb = RPM * i / 16;
      const int key = min(slot16[mb] + (RPM * i & 15) + ld_r, c1 - 1);
      const bf16_t* src = (key >= ctx ? Vn + (key - ctx) * new_stride : Vg + (row16[mb] + (key - slot16[mb])) * HD) +
                          8 * (ld_slot ^ v_swz<HD>(rl));
      __builtin_amdgcn_global_load_lds((const GLOBAL_AS void*)src,
                                       (LDS_AS void*)(buf + wave * kVTileBytes + RPM * i * kRowBytes), 16, 0,
                                       kNonTemporal);
    }
  };

  // transposing-read offsets (kept in registers, see page_decode.hip)
  const int rr = (lane & 15) >> 2, qq = lane & 3;
  int v_rd[DB][2];
#pragma unroll
  for (int db = 0; db < DB; ++db)
#pragma unroll
    for (int half = 0; half < 2; ++half) {
      const int row = 16 * half + 4 * g4 + rr;
      v_rd[db][half] = row * kRowBytes + (((2 * db + (qq >> 1)) ^ v_swz<HD>(row)) << 4) + 8 * (qq & 1);
    }

  f32x4_t oacc[NB][DB];
  float m_run[NB], l_part[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m_run[nb] = kNoMax;
    l_part[nb] = 0.f;
#pragma unroll
    for (int i = 0; i < DB; ++i) oacc[nb][i] = f32x4_t{};
  }
  const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3F803F80u);

  bool odd = false;   // a value of the new tokens in this lane's pieces was not finite
  auto tile = [&](int k0, auto parity, u32x4 (&kcur)[2][KS], u32x4 (&knext)[2][KS]) {
    constexpr int P = decltype(parity)::value;
    const uint8_t* vcur = P ? v_lds1 : v_lds0;
    if (k0 + kTile < c1) load(k0 + kTile, knext, P ? v_lds0 : v_lds1);
    const bool fresh = k0 + kTile > ctx;   // the tile reaches the new tokens
    if (fresh) {
#pragma unroll
      for (int i = 0; i < kTile / RPM; ++i) {   // (the pieces this lane moved)
        const int key = min(min(k0 + (RPM * i & ~15), (c1 - 1) & ~15) + (RPM * i & 15) + ld_r, c1 - 1);
        u32x4* piece = reinterpret_cast<u32x4*>(const_cast<uint8_t*>(vcur) + wave * kVTileBytes + RPM * i * kRowBytes + 16 * lane);
        uint32_t w[4] = {(*piece)[0], (*piece)[1], (*piece)[2], (*piece)[3]};
        if (key >= ctx && clear_odd(w)) {
          *piece = u32x4{w[0], w[1], w[2], w[3]};
          odd = true;
        }
      }
    }
    if constexpr (kRope) {
      if (fresh) {   // their keys, read unrotated, turned to their positions
#pragma unroll
        for (int mb = 0; mb < 2; ++mb) {
          const int key = min(min(k0 + 16 * mb, (c1 - 1) & ~15) + n, c1 - 1);
          if (key >= ctx) rot_operand<HD, kInterleaved>(kcur[mb], trow(key), g4);
        }
      }
    }
    int q_at = lane;
    if constexpr (kQueryLds) asm volatile("" : "+v"(q_at));   // (read for each tile, not kept in registers)
    f32x4_t sacc[NB][2];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) sacc[nb][0] = sacc[nb][1] = f32x4_t{};
#pragma unroll
    for (int ks = 0; ks < KS; ++ks)
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb) {
          const bf16x8_t hi = kQueryLds ? as_bf16x8(q_lds[(nb * KS + ks) * 64 + q_at]) : qop[nb][ks];
          sacc[nb][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kcur[mb][ks]), hi, sacc[nb][mb], 0, 0, 0);
          if constexpr (kRope) {
            const u32x4 lo = kQueryLds ? q_lds[((NB + nb) * KS + ks) * 64 + q_at] : q_lo[nb][ks];
            sacc[nb][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(as_bf16x8(kcur[mb][ks]), as_bf16x8(lo), sacc[nb][mb], 0, 0, 0);
          }
        }
    // probabilities in bfloat16, and what that rounding left
    bf16x8_t pop_h[NB], pop_l[NB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float mx = -INFINITY;
      const int lim = fresh ? min(c1, qpos[nb] + 1) : c1;   // this row's keys end here
#pragma unroll
      for (int mb = 0; mb < 2; ++mb)
#pragma unroll
        for (int e = 0; e < 4; ++e) {
          if (k0 + 16 * mb + 4 * g4 + e >= lim) sacc[nb][mb][e] = -INFINITY;
          mx = fmaxf(mx, sacc[nb][mb][e]);
        }
      mx = fmaxf(mx, __shfl_xor(mx, 16, 64));
      mx = fmaxf(mx, __shfl_xor(mx, 32, 64));
      const float m_tile = mx * a.scale_log2;
      if (__any(m_tile > m_run[nb] + 8.f)) {   // lazy reference max: p <= 2^8 (so values up to 2^120 over the number of keys)
        const float m_new = fmaxf(m_run[nb], m_tile);
        const float alpha = __builtin_amdgcn_exp2f(m_run[nb] - m_new);
        m_run[nb] = m_new;
        l_part[nb] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[nb][db] *= alpha;
      }
      uint32_t ph[4], pl[4];
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const float p0 = __builtin_amdgcn_exp2f(fmaf(sacc[nb][j >> 1][2 * (j & 1)], a.scale_log2, -m_run[nb]));
        const float p1 = __builtin_amdgcn_exp2f(fmaf(sacc[nb][j >> 1][2 * (j & 1) + 1], a.scale_log2, -m_run[nb]));
        ph[j] = pack_bf16x2(p0, p1);
        pl[j] = pack_bf16x2(p0 - __uint_as_float(ph[j] << 16), p1 - __uint_as_float(ph[j] & 0xFFFF0000u));
      }
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        l_part[nb] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, ph[j]), ones, l_part[nb], false);
        l_part[nb] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pl[j]), ones, l_part[nb], false);
      }
      pop_h[nb] = as_bf16x8(u32x4{ph[0], ph[1], ph[2], ph[3]});
      pop_l[nb] = as_bf16x8(u32x4{pl[0], pl[1], pl[2], pl[3]});
    }
    const uint8_t* vw = vcur + wave * kVTileBytes;
#pragma unroll
    for (int db = 0; db < DB; ++db) {
      const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS i16x4*)(vw + v_rd[db][0]));
      const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS i16x4*)(vw + v_rd[db][1]));
      const bf16x8_t vv = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        oacc[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pop_h[nb], oacc[nb][db], 0, 0, 0);
        oacc[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv, pop_l[nb], oacc[nb][db], 0, 0, 0);
      }
    }
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): the next tile is resident
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

  // The new tokens of this range into their pages (nobody reads those rows from the pages in this launch).
  for (int i = st_i; i < st1; i += kFewThreads / (2 * KC)) {
    const int slot = ctx + i;
    const int32_t page = i == st_i ? st_page : entry(slot >> a.map.shift);
    if (page < 0 || page >= a.map.n_pages) continue;
    const int c = tid & (KC - 1);
    const bool is_k = (tid & (2 * KC - 1)) < KC;
    const int64_t row = row0 + ((int64_t)page << a.map.shift) + (slot & ((1 << a.map.shift) - 1));
    u32x4* dst = reinterpret_cast<u32x4*>((is_k ? a.pages_k : a.pages_v) + row * HD);
    const u32x4* src = reinterpret_cast<const u32x4*>((is_k ? Kn : Vn) + i * new_stride);
    if (kRope && is_k) {   // the new key turned to its slot: thread c < KC/2 takes a chunk pair
      if (c < KC / 2) {
        // rotate-half: chunks c, c + KC/2 (frequencies 8 c ..); interleaved: 2 c, 2 c + 1 (8 c ..)
        const int ca = kInterleaved ? 2 * c : c, cb = kInterleaved ? 2 * c + 1 : c + KC / 2;
        const float2* cs_row = trow(slot);
        float x[8], y[8];
        unpack8(src[ca], x);
        unpack8(src[cb], y);
#pragma unroll
        for (int e = 0; e < 8; ++e) {
          const float2 cs = cs_row[8 * c + e];
          if constexpr (kInterleaved) {
            float* z = e < 4 ? x : y;
            rot_pair(z[2 * (e & 3)], z[2 * (e & 3) + 1], cs.x, cs.y);
          } else {
            rot_pair(x[e], y[e], cs.x, cs.y);
          }
        }
        dst[ca] = pack8(x);
        dst[cb] = pack8(y);
      }
    } else {
      dst[c] = src[c];
    }
  }

  // ---- merge the 8 waves (log-sum-exp) through LDS, reusing the V buffers: four waves' rows each
  static_assert(4 * ROWS * HD * 4 <= kFewWaves * kVTileBytes, "merge area");
  float l_tot[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    l_tot[nb] = l_part[nb] + __shfl_xor(l_part[nb], 16, 64);
    l_tot[nb] += __shfl_xor(l_tot[nb], 32, 64);
  }
  const bool odd_wave = __any(odd);
  __syncthreads();
  // (16-byte chunk c of row r at c ^ (r & 15): the 16 rows of a store would meet in one bank otherwise)
  auto o_lds = [&](int w, int r, int c) {
    return reinterpret_cast<f32x4_t*>(w < 4 ? v_lds0 : v_lds1) + ((w & 3) * ROWS + r) * (HD / 4) + (c ^ (r & 15));
  };
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = 16 * nb + n;
    if (r >= M) continue;
#pragma unroll
    for (int db = 0; db < DB; ++db)
      *o_lds(wave, r, 4 * db + g4) = oacc[nb][db];
    if (g4 == 0) {
      ml_lds[(wave * ROWS + r) * 2] = m_run[nb];
      ml_lds[(wave * ROWS + r) * 2 + 1] = l_tot[nb];
    }
  }
  if (lane == 0) odd_lds[wave] = odd_wave;
  __syncthreads();
  // thread -> (row r, head dims md .. + 8)
  static_assert(ROWS * KC <= kFewThreads, "a thread per 8 outputs");
  const int r = tid / KC, md = 8 * (tid & (KC - 1));
  float m_all = kNoMax, den = 0.f, o[8] = {0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f, 0.f};
  bool odd_new = false;
  if (r < M) {
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      m_all = fmaxf(m_all, ml_lds[(w * ROWS + r) * 2]);
      odd_new |= odd_lds[w];
    }
#pragma unroll
    for (int w = 0; w < kFewWaves; ++w) {
      const float wt = __builtin_amdgcn_exp2f(ml_lds[(w * ROWS + r) * 2] - m_all);
      den += wt * ml_lds[(w * ROWS + r) * 2 + 1];
      const f32x4_t x0 = *o_lds(w, r, md / 4), x1 = *o_lds(w, r, md / 4 + 1);
#pragma unroll
      for (int e = 0; e < 4; ++e) {
        o[e] += wt * x0[e];
        o[4 + e] += wt * x1[e];
      }
    }
  }
  // values that are not finite (where the scores are: else the outputs are NaN anyway): cached ones, which every row
  // sees, and the new tokens', up to the row's own
  if (__any((odd_new || any_odd(o)) && fabsf(den) < INFINITY)) {
    float v[8] = {};
    odd_values<KC>([&](int key) { return Vg + page_row(a.map, b, key) * HD; }, wc0, min(wc1, ctx), v);
    for (int key = max(wc0, ctx); key < wc1 && key <= ctx + r / n_rep; ++key)
      add_odd(*reinterpret_cast<const uint4*>(Vn + (key - ctx) * new_stride + md), v);
#pragma unroll
    for (int e = 0; e < 8; ++e)
      if (!(fabsf(v[e]) < INFINITY)) o[e] = v[e];
  }
  if (r < M) {
    const int64_t row = row_of(r);
    if (a.n_splits == 1) {
      const float inv = 1.f / den;
#pragma unroll
      for (int e = 0; e < 8; ++e) o[e] *= inv;
      *reinterpret_cast<u32x4*>(a.out + row * HD + md) = pack8(o);
    } else {
      const int64_t slot = row * a.n_splits + split;
      float* wo = a.ws_o + slot * HD + md;
      *reinterpret_cast<f32x4_t*>(wo) = f32x4_t{o[0], o[1], o[2], o[3]};
      *reinterpret_cast<f32x4_t*>(wo + 4) = f32x4_t{o[4], o[5], o[6], o[7]};
      if (md == 0) *reinterpret_cast<float2*>(a.ws_ml + 2 * slot) = make_float2(m_all, den);
    }
  }
}

template <int HD, int NB>
hipError_t launch_as(const PageFewArgs& a, dim3 grid, bool interleaved, const AttnShape& s, hipStream_t stream) {
  if (!a.table)
    hipLaunchKernelGGL((page_few_kernel<HD, NB, false, false>), grid, dim3(kFewThreads), 0, stream, a);
  else if (interleaved)
    hipLaunchKernelGGL((page_few_kernel<HD, NB, true, true>), grid, dim3(kFewThreads), 0, stream, a);
  else
    hipLaunchKernelGGL((page_few_kernel<HD, NB, true, false>), grid, dim3(kFewThreads), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess || a.n_splits == 1) return e;
  AttnShape rows = s;   // (the combine's rows of a request: every head of every token)
  rows.n_q_heads = a.n_new * s.n_q_heads;
  return launch_decode_combine<HD, false, true>(a.ws_o, a.ws_ml, a.ctx_len, rows, a.max_ctx, 0, 0, a.n_splits, EqualDeal{},
                                                a.out, stream, FewTokens{a.n_valid, a.n_new, s.n_q_heads});
}

}  // namespace

hipError_t launch_few_bf16_pages(const PageAttnArgs& p) {
  const AttnShape& s = p.s;
  PageFewArgs a = {};
  a.q = static_cast<const bf16_t*>(p.q);
  a.k_new = static_cast<const bf16_t*>(p.k_new);
  a.v_new = static_cast<const bf16_t*>(p.v_new);
  a.pages_k = static_cast<bf16_t*>(p.pages_k);
  a.pages_v = static_cast<bf16_t*>(p.pages_v);
  a.map = p.map;
  a.ctx_len = p.base_len;
  a.n_valid = p.n_valid;
  a.out = static_cast<bf16_t*>(p.out);
  a.batch = s.batch;
  a.stream_rows = s.cache_cap;
  a.n_q_heads = s.n_q_heads;
  a.n_kv_heads = s.n_kv_heads;
  a.n_new = p.n_new;
  a.max_ctx = p.max_base;
  a.scale_log2 = s.scale_log2;
  a.table = p.table;
  a.table_stride = p.table_stride;
  a.max_abs_delta = p.max_abs_delta;
  a.n_splits = few_bf16_splits(s, p.n_new, p.max_base, p.workspace ? p.ws_bytes : 0);
  const size_t rows = (size_t)s.n_layers * s.batch * p.n_new * s.n_q_heads;
  a.ws_o = static_cast<float*>(p.workspace);
  a.ws_ml = a.n_splits > 1 ? a.ws_o + rows * a.n_splits * s.head_dim : nullptr;
  const dim3 grid((unsigned)(a.n_splits * s.batch * s.n_kv_heads), s.n_layers);
  const bool two = (int64_t)p.n_new * (s.n_q_heads / s.n_kv_heads) > 16;
  if (s.head_dim == 64)
    return two ? launch_as<64, 2>(a, grid, p.interleaved, s, p.stream) : launch_as<64, 1>(a, grid, p.interleaved, s, p.stream);
  return two ? launch_as<128, 2>(a, grid, p.interleaved, s, p.stream) : launch_as<128, 1>(a, grid, p.interleaved, s, p.stream);
}

}  // namespace pic
