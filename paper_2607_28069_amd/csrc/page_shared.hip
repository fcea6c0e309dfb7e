// Attention of new tokens over a cache handed out in pages, for a batch whose requests share long prefixes: each shared
// prefix is read once for all the requests of its group.  bf16 storage.
//
// With softmax sums split by keys, out = sum_x e^(m_x - m) o_x / sum_x e^(m_x - m) l_x over parts x with maxima m_x,
// sums l_x and weighted values o_x.  The parts of a request are key ranges of its group's prefix, whose workgroups take
// the query rows of all its requests side by side, and key ranges of its own slots; a combine joins them.  The
// prefix then costs its bytes once, and as many products as before.
//
//  * A workgroup of 4 waves has up to 64 NB query rows (16 NB a wave) and one key range of one page table row, in
//    tiles of 64 keys: S^T = K Q^T and O^T = V^T P^T on v_mfma_f32_16x16x32_bf16 as in page_decode.hip, K and V both
//    through LDS, where all four waves read them.  Each wave moves 16 keys of a tile, which lie in one page.
//  * Both parts of a launch run side by side: workgroups [0, prefix_blocks) are the prefixes', the others the requests'.
//  * What is served together ends with a whole tile: a prefix's last keys are read by each request.  A row sees keys up
//    to its limit; tiles that some row of the workgroup sees in part are masked, and values there that are not finite
//    cleared in LDS, so that rows that do not see them stay as they are (the others get them back at the end).
//
// Measured (combine included, 32 + 2 x 8 heads of 128): 2 requests over 2K 11 us, 16 over 10K 19, 64 over 16K 49, about 1.2 us a
// tile of 64 keys that a workgroup of 64 rows has to itself, the first one after 4 to 5 where all start at once; 37 requests in
// 4 groups of up to 32K (28 + 2 x 4 heads) 57 us, 3.9 TB/s in all; 16 x 24 tokens over 10K 80 us, 820 TFLOP/s.
#include <type_traits>

#include "decode_common.h"

namespace pic {
namespace {

constexpr int kRowsPerMfma = 16, kNumXcd = 8;
constexpr int kKeys = kSharedKeys;       // keys per tile
constexpr int kMoved = kKeys / kWaves;   // keys of a tile that a wave moves
static_assert(kMoved == 16, "they lie in one page");

struct PageSharedArgs {
  const bf16_t* q;        // [L][B][n_new][Hq][D]
  const bf16_t* k_new;    // [L][B][n_new][Hkv][D]
  const bf16_t* v_new;
  bf16_t* pages_k;        // [L][Hkv][stream_rows][D]
  bf16_t* pages_v;
  PageMap map;
  SharedMap groups;
  const int32_t* base_len;
  const int32_t* n_valid;
  float* ws_o;            // [L][B][n_new][Hq][parts][D], a row's parts: prefix_splits, then own_splits
  float* ws_ml;           // [L][B][n_new][Hq][parts][2]
  int32_t batch, stream_rows, n_q_heads, n_kv_heads, n_new, max_base, offset;
  int32_t prefix_splits, own_splits, prefix_row_tiles, own_row_tiles, prefix_blocks;
  float scale_log2;
};

typedef __amdgpu_buffer_rsrc_t rsrc_t;
__device__ __forceinline__ rsrc_t make_rsrc(const void* base) {   // (every offset formed is in bounds)
  return __builtin_amdgcn_make_buffer_rsrc(const_cast<void*>(base), 0, -1, 0x00020000);
}
// 16 bytes a lane from base + off into LDS at lds + 16 * lane; the indexed form is for the second of two moves under
// complementary lane masks, so that the compiler does not fold them into one.  (The global-address form would make every
// LDS read wait for all moves on their way.)
template <bool kStream>
__device__ __forceinline__ void move16(rsrc_t r, uint32_t off, void* lds) {
  __builtin_amdgcn_raw_ptr_buffer_load_lds(r, (LDS_AS void*)lds, 16, off, 0, 0, kStream ? kNonTemporal : 0);
}
__device__ __forceinline__ void move16_other(rsrc_t r, uint32_t off, void* lds) {
  __builtin_amdgcn_struct_ptr_buffer_load_lds(r, (LDS_AS void*)lds, 16, 0, off, 0, 0, 0);
}
template <int HD>
__device__ __forceinline__ int k_swz(int row) {   // 16-byte chunk c of K row `row` sits at c ^ k_swz(row)
  if constexpr (HD == 128) return row & 15;
  else return (row >> 1) & 7;
}
// Lanes n, n + 16, n + 32, n + 48 hold the same query column.
__device__ __forceinline__ float column_max(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return fmaxf(__uint_as_float(r[0]), __uint_as_float(r[1]));
}
__device__ __forceinline__ float column_sum(float x) {
  auto r = __builtin_amdgcn_permlane32_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  x = __uint_as_float(r[0]) + __uint_as_float(r[1]);
  r = __builtin_amdgcn_permlane16_swap(__float_as_uint(x), __float_as_uint(x), false, false);
  return __uint_as_float(r[0]) + __uint_as_float(r[1]);
}

// What a workgroup's waves share: two buffers each of a tile's keys and values.
struct Buffers {
  uint8_t *k0, *k1, *v0, *v1;
  int* odd;   // a value that some rows do not see was not finite
};

// One part: rows of a group over a key range of its prefix, or of a request over a key range of its own slots.  NB blocks of
// 16 rows a wave; kTerms: bfloat16 terms of a probability.
template <int HD, int NB, int kTerms, bool kPrefix, bool kStream>
__device__ __forceinline__ void part_of(const PageSharedArgs& a, int block, const Buffers& lds) {
  constexpr int kRowBytes = Dims<HD>::kRowBytes;
  constexpr int KC = Dims<HD>::kChunks, KS = Dims<HD>::kSteps, DB = Dims<HD>::kBlocks;
  constexpr int RPM = Dims<HD>::kRowsPerMove, MOVES = kMoved / RPM, ROWS = kRowsPerMfma * NB * kWaves;
  const int tid = threadIdx.x, lane = tid & 63;
  const int wave = __builtin_amdgcn_readfirstlane(tid >> 6);
  const int l = blockIdx.y, n_rep = a.n_q_heads / a.n_kv_heads, parts = a.prefix_splits + a.own_splits;
  const int row_tiles = kPrefix ? a.prefix_row_tiles : a.own_row_tiles, splits = kPrefix ? a.prefix_splits : a.own_splits;
  // blocks are dealt to the XCDs in turn: the tiles of rows over one key range go to one XCD, whose L2 brings it once
  const int rt = block / kNumXcd % row_tiles, range = block / kNumXcd / row_tiles * kNumXcd + block % kNumXcd;
  const int split = range % splits, g = range / splits % a.n_kv_heads, owner = range / splits / a.n_kv_heads;
  if (owner >= (kPrefix ? a.groups.n_groups : a.batch)) return;
  // (uniform) rows [row0, row0 + n_rows) of the packed ones, first request, key range [k0, k1) of its page table row, the
  // first new token's slot
  const int row0 = rt * ROWS;
  int b0 = owner, n_rows, k0, k1, ctx = INT32_MAX, n_tok = 0;
  bool grouped = true;
  // requests of a group: those side by side that this part's rows are of
  if constexpr (kPrefix) {
    b0 = a.groups.first(owner);
    const int tiles = a.groups.slots(owner) / kSharedKeys, per = ceil_div(tiles, splits);
    n_rows = min(a.groups.requests(owner) * a.n_new * n_rep - row0, ROWS);
    if (n_rows <= 0) return;
    k0 = min(split * per, tiles) * kSharedKeys;
    k1 = min(split * per + per, tiles) * kSharedKeys;
  } else {
    // the request's group, all starts looked at at once
    int gi = -1, slots = 0;
    const int32_t base = a.base_len[b0], valid = a.n_valid ? a.n_valid[b0] : a.n_new;
    if (a.groups.n_groups < 64) {
      const int32_t first = lane <= a.groups.n_groups ? a.groups.first(lane) : INT32_MAX;
      const int32_t len = lane < a.groups.n_groups ? a.groups.slots(lane) : 0;
      gi = __popcll(__ballot(lane < a.groups.n_groups && first <= b0)) - 1;
      const int at = max(gi, 0), from = __builtin_amdgcn_readlane(first, at), to = __builtin_amdgcn_readlane(first, at + 1);
      slots = __builtin_amdgcn_readlane(len, at);
      if (b0 >= to || b0 - from >= a.groups.max_group) gi = -1;
    } else {
      gi = a.groups.group_of(b0);
      slots = gi < 0 ? 0 : a.groups.slots(gi);
    }
    grouped = gi >= 0;
    n_tok = base < 0 ? 0 : clamp_len(valid, a.n_new);
    n_rows = min(n_tok * n_rep - row0, ROWS);
    if (n_rows <= 0) return;   // padding of the batch
    ctx = clamp_len(base, a.max_base) + a.offset;
    const int from = grouped ? shared_part(slots, ctx) : 0, end = ctx + n_tok;
    const int tiles = ceil_div(end - from, kSharedKeys), per = ceil_div(tiles, splits);
    k0 = from + min(split * per, tiles) * kSharedKeys;
    k1 = min(from + min(split * per + per, tiles) * kSharedKeys, end);
  }
  // keys past the last row's are nobody's
  const int k_end = kPrefix ? k1 : min(k1, ctx + (row0 + n_rows - 1) / n_rep + 1);

  // page numbers: entries [win, win + 64) of the page table row and the 64 after them
  const int tab = min(b0, a.batch - 1);
  const int32_t* ptab = a.map.table + (int64_t)tab * a.map.cap;
  auto entry = [&](int32_t i) { return ptab[clamp_entry(i, a.map)]; };
  PageWindow win = {min(k0 + kMoved * wave, max(k_end - 1, 0) & ~(kMoved - 1)) >> a.map.shift};
  int32_t w_cur = entry(win.at + lane), w_next = entry(win.at + 64 + lane);
  auto row_at = [&](int s) -> int64_t {   // (s uniform, a multiple of kMoved, never less than the one asked for before)
    const int32_t i = s >> a.map.shift;
    if (win.moves(i, 64)) {
      w_cur = w_next;
      w_next = entry(win.at + 64 + lane);
    }
    const int32_t page = clamp_page(__builtin_amdgcn_readlane(w_cur, win.lane(i)), a.map);
    return ((int64_t)page << a.map.shift) + (s & ((1 << a.map.shift) - 1));
  };
  const int64_t stream0 = ((int64_t)l * a.n_kv_heads + g) * a.stream_rows;
  const bf16_t* Kg = a.pages_k + stream0 * HD;
  const bf16_t* Vg = a.pages_v + stream0 * HD;
  const int64_t new0 = (((int64_t)l * a.batch + tab) * a.n_new * a.n_kv_heads + g) * HD;
  const uint32_t new_stride = (uint32_t)a.n_kv_heads * kRowBytes;   // bytes
  const bf16_t* Kn = a.k_new + new0;
  const bf16_t* Vn = a.v_new + new0;

  // This wave's keys of the tile at s0 into LDS rows kMoved wave ..: instruction i fills rows RPM i + lane / KC, chunk
  // place lane % KC.  Keys past the range are its last one again (their scores are masked).
  const int ld_r = lane / KC, ld_c = lane & (KC - 1);
  auto load = [&](int s0, uint8_t* kb, uint8_t* vb) {
    const int s = min(s0 + kMoved * wave, (k_end - 1) & ~(kMoved - 1));
    const int64_t row = kPrefix || s < ctx ? row_at(s) : 0;
    const rsrc_t rk = make_rsrc(Kg + row * HD), rv = make_rsrc(Vg + row * HD);
    kb += kMoved * wave * kRowBytes;
    vb += kMoved * wave * kRowBytes;
    if (kPrefix || s + kMoved <= ctx) {
#pragma unroll
      for (int i = 0; i < MOVES; ++i) {
        const int r = RPM * i + ld_r, from = kPrefix ? r : min(s + r, k_end - 1) - s;
        move16<kStream>(rk, from * kRowBytes + 16 * (ld_c ^ k_swz<HD>(kMoved * wave + r)), kb + RPM * i * kRowBytes);
        move16<kStream>(rv, from * kRowBytes + 16 * (ld_c ^ v_swz<HD>(kMoved * wave + r)), vb + RPM * i * kRowBytes);
      }
    } else {   // some of them are new tokens
      const rsrc_t nk = make_rsrc(Kn), nv = make_rsrc(Vn);
#pragma unroll
      for (int i = 0; i < MOVES; ++i) {
        const int r = RPM * i + ld_r, key = min(s + r, k_end - 1);
        const uint32_t ck = 16 * (ld_c ^ k_swz<HD>(kMoved * wave + r)), cv = 16 * (ld_c ^ v_swz<HD>(kMoved * wave + r));
        if (key < ctx) {
          move16<kStream>(rk, (key - s) * kRowBytes + ck, kb + RPM * i * kRowBytes);
          move16<kStream>(rv, (key - s) * kRowBytes + cv, vb + RPM * i * kRowBytes);
        } else {
          move16_other(nk, (key - ctx) * new_stride + ck, kb + RPM * i * kRowBytes);
          move16_other(nv, (key - ctx) * new_stride + cv, vb + RPM * i * kRowBytes);
        }
      }
    }
  };
  if (k0 < k_end) load(k0, lds.k0, lds.v0);
  if (tid == 0) *lds.odd = 0;

  // A packed row: its place among the rows of q / out, and where its keys end here (-1: padding).
  auto row_of = [&](int r, int64_t& at) -> int {
    if constexpr (!kPrefix) {
      const int tok = r / n_rep;
      at = (((int64_t)l * a.batch + b0) * a.n_new + tok) * a.n_q_heads + g * n_rep + (r - tok * n_rep);
      return min(k1, ctx + tok + 1);
    } else {
      const int t = r / n_rep, b = b0 + t / a.n_new, tok = t - (b - b0) * a.n_new;   // (t: of the group's tokens)
      at = (((int64_t)l * a.batch + b) * a.n_new + tok) * a.n_q_heads + g * n_rep + (r - t * n_rep);
      const int32_t base = a.base_len[b], valid = a.n_valid ? a.n_valid[b] : a.n_new;
      if (base < 0 || tok >= valid) return -1;
      return min(k1, shared_part(k1, clamp_len(base, a.max_base) + a.offset));
    }
  };
  const int n = lane & 15, g4 = lane >> 4;
  // this lane's query columns, rows 16 (NB wave + nb) + n: Q^T operands, head dims 32 ks + 8 g4 .. + 8
  bool row_ok[NB];
  int lim[NB];
  int64_t qrow[NB];
  u32x4 qv[NB][KS];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const int r = 16 * (NB * wave + nb) + n;
    lim[nb] = row_of(row0 + (r < n_rows ? r : 0), qrow[nb]);
    const u32x4* qp = reinterpret_cast<const u32x4*>(a.q + qrow[nb] * HD);
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qv[nb][ks] = r < n_rows ? qp[4 * ks + g4] : u32x4{0, 0, 0, 0};
    row_ok[nb] = r < n_rows && lim[nb] >= 0;
    // (rows of padding hold anything: they are asked for with the others, and are no queries)
#pragma unroll
    for (int ks = 0; ks < KS; ++ks) qv[nb][ks] = row_ok[nb] ? qv[nb][ks] : u32x4{0, 0, 0, 0};
  }
  // (uniform) keys before `clear` are seen by every row of the workgroup
  int clear = INT32_MAX;
  if constexpr (kPrefix) {
#pragma unroll
    for (int i = 0; i < ROWS / 64; ++i) {
      int64_t at;
      const int x = 64 * i + lane < n_rows ? row_of(row0 + 64 * i + lane, at) : -1;
      if (x >= 0) clear = min(clear, x);
    }
#pragma unroll
    for (int off = 1; off < 64; off <<= 1) clear = min(clear, __shfl_xor(clear, off, 64));
    clear = __builtin_amdgcn_readfirstlane(clear);
  } else {
    clear = min(k1, ctx + row0 / n_rep + 1);
  }

  // operand reads: K row 16 mb + n, chunk 4 ks + g4; V transposed, see page_decode.hip
  int k_rd[KS], v_rd[DB];
#pragma unroll
  for (int ks = 0; ks < KS; ++ks) k_rd[ks] = n * kRowBytes + (((4 * ks + g4) ^ k_swz<HD>(n)) << 4);
  const int rr = (lane & 15) >> 2, qq = lane & 3;
#pragma unroll
  for (int db = 0; db < DB; ++db) {
    const int row = 4 * g4 + rr;   // (16 rows further on the swizzle is the same)
    v_rd[db] = row * kRowBytes + (((2 * db + (qq >> 1)) ^ v_swz<HD>(row)) << 4) + 8 * (qq & 1);
  }

  f32x4_t oacc[NB][DB];
  float m_run[NB], l_part[NB];
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    m_run[nb] = kNoMax;
    l_part[nb] = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db) oacc[nb][db] = f32x4_t{};
  }
  bool odd = false;
  const bf16x2_t ones = __builtin_bit_cast(bf16x2_t, 0x3F803F80u);
  const bool busy = 16 * NB * wave < n_rows;   // (uniform) a wave of no rows moves its share of the keys only

  auto use = [&](int s0, bool masked, const uint8_t* kb, const uint8_t* vb) {
    constexpr int MB = kKeys / 16, H = kKeys / 32;
    f32x4_t sacc[NB][MB];
#pragma unroll
    for (int nb = 0; nb < NB; ++nb)
#pragma unroll
      for (int mb = 0; mb < MB; ++mb) sacc[nb][mb] = f32x4_t{};
    // 16 keys' operands two blocks ahead of their products, in this order: left to itself the compiler asks for most of them
    // when they are due (16 over 10K 20.0 -> 19.6 us, 16 x 24 tokens over 10K 81 -> 79; three ahead is no better)
    bf16x8_t kk[2][KS];
    auto read_k = [&](int mb) {
#pragma unroll
      for (int ks = 0; ks < KS; ++ks) kk[mb & 1][ks] = as_bf16x8(*reinterpret_cast<const u32x4*>(kb + 16 * mb * kRowBytes + k_rd[ks]));
    };
    read_k(0);
    read_k(1);
#pragma unroll
    for (int mb = 0; mb < MB; ++mb) {
      __builtin_amdgcn_sched_barrier(0);
#pragma unroll
      for (int ks = 0; ks < KS; ++ks)
#pragma unroll
        for (int nb = 0; nb < NB; ++nb)
          sacc[nb][mb] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(kk[mb & 1][ks], as_bf16x8(qv[nb][ks]), sacc[nb][mb], 0, 0, 0);
      __builtin_amdgcn_sched_barrier(0);
      if (mb + 2 < MB) read_k(mb + 2);
    }
    __builtin_amdgcn_sched_barrier(0);
    // values of 32 keys, read while the probabilities before them are made
    bf16x8_t vv[DB];
    auto read_v = [&](int h) {
#pragma unroll
      for (int db = 0; db < DB; ++db) {
        const i16x4 lo = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS i16x4*)(vb + 32 * h * kRowBytes + v_rd[db]));
        const i16x4 hi = __builtin_amdgcn_ds_read_tr16_b64_v4i16((LDS_AS i16x4*)(vb + (32 * h + 16) * kRowBytes + v_rd[db]));
        vv[db] = __builtin_bit_cast(bf16x8_t, __builtin_shufflevector(lo, hi, 0, 1, 2, 3, 4, 5, 6, 7));
      }
    };
    read_v(0);
    // (a wave that has its scores goes before one still at its products: the two of a SIMD, from different workgroups, then
    // keep out of step.  16 x 24 tokens over 10K 83.6 -> 80.6 us; waves alone on their SIMD do not notice)
    __builtin_amdgcn_s_setprio(1);
    if (masked) {
      asm volatile("");   // (a branch: as selects the masks would cost every tile)
#pragma unroll
      for (int nb = 0; nb < NB; ++nb)
#pragma unroll
        for (int mb = 0; mb < MB; ++mb)
#pragma unroll
          for (int e = 0; e < 4; ++e)
            if (s0 + 16 * mb + 4 * g4 + e >= lim[nb]) sacc[nb][mb][e] = -INFINITY;
    }
    float m_tile[NB];
    bool rises = false;
#pragma unroll
    for (int nb = 0; nb < NB; ++nb) {
      float mx = -INFINITY;
#pragma unroll
      for (int mb = 0; mb < MB; ++mb)
#pragma unroll
        for (int e = 0; e < 4; ++e) mx = fmaxf(mx, sacc[nb][mb][e]);
      m_tile[nb] = column_max(mx) * a.scale_log2;
      rises |= m_tile[nb] > m_run[nb] + 8.f;
    }
    // lazy reference max: p <= 2^8 (so values up to 2^120 over the number of keys).  Each column's own scores alone raise its
    // maximum: the columns of a wave are different requests', and a row's rounding is not to depend on its neighbours.
    if (__any(rises)) {
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        const float m_new = m_tile[nb] > m_run[nb] + 8.f ? m_tile[nb] : m_run[nb];
        const float alpha = __builtin_amdgcn_exp2f(m_run[nb] - m_new);
        m_run[nb] = m_new;
        l_part[nb] *= alpha;
#pragma unroll
        for (int db = 0; db < DB; ++db) oacc[nb][db] *= alpha;
      }
    }
    // probabilities in bfloat16, and what that rounding left
#pragma unroll
    for (int h = 0; h < H; ++h) {
      bf16x8_t pop[NB][kTerms];
#pragma unroll
      for (int nb = 0; nb < NB; ++nb) {
        uint32_t ph[4], pl[4];
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float p0 = __builtin_amdgcn_exp2f(fmaf(sacc[nb][2 * h + (j >> 1)][2 * (j & 1)], a.scale_log2, -m_run[nb]));
          const float p1 = __builtin_amdgcn_exp2f(fmaf(sacc[nb][2 * h + (j >> 1)][2 * (j & 1) + 1], a.scale_log2, -m_run[nb]));
          ph[j] = pack_bf16x2(p0, p1);
          if constexpr (kTerms == 2) pl[j] = pack_bf16x2(p0 - __uint_as_float(ph[j] << 16), p1 - __uint_as_float(ph[j] & 0xFFFF0000u));
        }
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          l_part[nb] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, ph[j]), ones, l_part[nb], false);
          if constexpr (kTerms == 2)
            l_part[nb] = __builtin_amdgcn_fdot2_f32_bf16(__builtin_bit_cast(bf16x2_t, pl[j]), ones, l_part[nb], false);
        }
        pop[nb][0] = as_bf16x8(u32x4{ph[0], ph[1], ph[2], ph[3]});
        if constexpr (kTerms == 2) pop[nb][1] = as_bf16x8(u32x4{pl[0], pl[1], pl[2], pl[3]});
      }
#pragma unroll
      for (int t = 0; t < kTerms; ++t)
#pragma unroll
        for (int db = 0; db < DB; ++db)
#pragma unroll
          for (int nb = 0; nb < NB; ++nb)
            oacc[nb][db] = __builtin_amdgcn_mfma_f32_16x16x32_bf16(vv[db], pop[nb][t], oacc[nb][db], 0, 0, 0);
      if (h + 1 < H) read_v(h + 1);
    }
    __builtin_amdgcn_s_setprio(0);
  };

  // The tile at s0, on its way into buffers kb / vb; the one after it goes to kn / vn.  (Both at once, or shorter tiles three
  // ahead, were slower.)
  auto tile = [&](int s0, uint8_t* kb, uint8_t* vb, uint8_t* kn, uint8_t* vn) {
    __builtin_amdgcn_s_waitcnt(0x0F70);   // vmcnt(0): this wave's part has arrived
    const bool masked = s0 + kKeys > clear;
    if (masked) {
#pragma unroll
      for (int i = 0; i < MOVES; ++i) {   // (the pieces this lane moved)
        u32x4* piece = reinterpret_cast<u32x4*>(vb + (kMoved * wave + RPM * i) * kRowBytes + 16 * lane);
        uint32_t w[4] = {(*piece)[0], (*piece)[1], (*piece)[2], (*piece)[3]};
        if (clear_odd(w)) {
          *piece = u32x4{w[0], w[1], w[2], w[3]};
          odd = true;
        }
      }
    }
    __syncthreads();   // all parts have, and the buffers of the next one are read
    if (s0 + kKeys < k_end) load(s0 + kKeys, kn, vn);
    if (busy) use(s0, masked, kb, vb);
  };
  for (int s0 = k0; s0 < k_end; s0 += 2 * kKeys) {
    tile(s0, lds.k0, lds.v0, lds.k1, lds.v1);
    if (s0 + kKeys < k_end) tile(s0 + kKeys, lds.k1, lds.v1, lds.k0, lds.v0);
  }

  // The new tokens of this range into their pages (nobody reads those rows from the pages in this launch), 2 KC threads each.
  if (!kPrefix && row0 == 0) {
    const int end = min(k1 - ctx, n_tok);
    for (int i = max(k0 - ctx, 0) + tid / (2 * KC); i < end; i += 256 / (2 * KC)) {
      const int64_t row = page_store_row(a.map, b0, ctx + i);
      if (row < 0) continue;
      const int c = tid & (KC - 1);
      const bool is_k = (tid & (2 * KC - 1)) < KC;
      const u32x4* src = reinterpret_cast<const u32x4*>((is_k ? Kn : Vn) + (int64_t)i * a.n_kv_heads * HD);
      reinterpret_cast<u32x4*>((is_k ? a.pages_k : a.pages_v) + (stream0 + row) * HD)[c] = src[c];
    }
  }

  // this part of every row
  if (__any(odd) && lane == 0) *lds.odd = 1;
  __syncthreads();
  if (!busy) return;
  const bool odd_there = *lds.odd != 0;
#pragma unroll
  for (int nb = 0; nb < NB; ++nb) {
    const float den = column_sum(l_part[nb]);
    // values that are not finite (where the scores are: else the outputs are NaN anyway): those of the keys that the row
    // sees, added up
    float all = 0.f;
#pragma unroll
    for (int db = 0; db < DB; ++db)
#pragma unroll
      for (int e = 0; e < 4; ++e) all += fabsf(oacc[nb][db][e]);
    if (__any((odd_there || !(all < INFINITY)) && fabsf(den) < INFINITY)) {
      f32x4_t sum[DB];
#pragma unroll
      for (int db = 0; db < DB; ++db) sum[db] = f32x4_t{};
      constexpr int kAhead = 8;   // keys' rows on their way at once; past the last one that one again, which changes no sum
      for (int key0 = k0; key0 < lim[nb]; key0 += kAhead) {
        const bf16_t* row[kAhead];
#pragma unroll
        for (int i = 0; i < kAhead; ++i) {
          const int key = min(key0 + i, lim[nb] - 1);
          row[i] = !kPrefix && key >= ctx ? Vn + (int64_t)(key - ctx) * a.n_kv_heads * HD : Vg + page_row(a.map, tab, key) * HD;
        }
#pragma unroll
        for (int db = 0; db < DB; ++db) {
          uint2 w[kAhead];
#pragma unroll
          for (int i = 0; i < kAhead; ++i) w[i] = *reinterpret_cast<const uint2*>(row[i] + 16 * db + 4 * g4);
#pragma unroll
          for (int i = 0; i < kAhead; ++i)
#pragma unroll
            for (int e = 0; e < 4; ++e) {
              const uint32_t x = e < 2 ? w[i].x : w[i].y;
              const float v = __uint_as_float(e & 1 ? x & 0xFFFF0000u : x << 16);
              if (!(fabsf(v) < INFINITY)) sum[db][e] += v;
            }
        }
      }
#pragma unroll
      for (int db = 0; db < DB; ++db)
#pragma unroll
        for (int e = 0; e < 4; ++e)
          if (!(fabsf(sum[db][e]) < INFINITY)) oacc[nb][db][e] = sum[db][e];
    }
    if (!row_ok[nb]) continue;
    const int64_t slot = qrow[nb] * parts + (kPrefix ? split : a.prefix_splits + split);
#pragma unroll
    for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4_t*>(a.ws_o + slot * HD + 16 * db + 4 * g4) = oacc[nb][db];
    if (g4 == 0) *reinterpret_cast<float2*>(a.ws_ml + 2 * slot) = make_float2(m_run[nb], den);
    if (!grouped && split == 0) {   // a request of no group has no parts of a prefix
      for (int i = 0; i < a.prefix_splits; ++i) {
        const int64_t none = qrow[nb] * parts + i;
#pragma unroll
        for (int db = 0; db < DB; ++db) *reinterpret_cast<f32x4_t*>(a.ws_o + none * HD + 16 * db + 4 * g4) = f32x4_t{};
        if (g4 == 0) *reinterpret_cast<float2*>(a.ws_ml + 2 * none) = make_float2(kNoMax, 0.f);
      }
    }
  }
}

// grid (prefix_blocks + own blocks, L), 256 threads; NB blocks of 16 rows a wave over the prefixes, kTerms terms of a
// probability there
template <int HD, int NB, int kTerms, bool kStream>
__global__ void __launch_bounds__(256) __attribute__((amdgpu_waves_per_eu(2, 2))) page_shared_kernel(PageSharedArgs a) {
  constexpr int kTileBytes = kKeys * Dims<HD>::kRowBytes;
  // (arrays of their own, so that the compiler sees that moves into one do not alias reads of another)
  __shared__ __attribute__((aligned(16))) uint8_t k_lds0[kTileBytes], k_lds1[kTileBytes];
  __shared__ __attribute__((aligned(16))) uint8_t v_lds0[kTileBytes], v_lds1[kTileBytes];
  __shared__ int odd;
  const Buffers lds = {k_lds0, k_lds1, v_lds0, v_lds1, &odd};
  if ((int)blockIdx.x < a.prefix_blocks)
    part_of<HD, NB, kTerms, true, kStream>(a, blockIdx.x, lds);
  else
    part_of<HD, 1, 2, false, kStream>(a, blockIdx.x - a.prefix_blocks, lds);
}

// The parts of a query row joined, where they are few: HD / 4 lanes a row, all parts' loads on their way at once.
template <int HD, int kFewParts>
__global__ void __launch_bounds__(256) shared_combine_kernel(PageSharedArgs a, bf16_t* __restrict__ out, int64_t n_rows) {
  constexpr int kLanes = HD / 4;
  const int64_t row = ((int64_t)blockIdx.x * 256 + threadIdx.x) / kLanes;
  const int d = 4 * (threadIdx.x % kLanes), parts = a.prefix_splits + a.own_splits;
  if (row >= n_rows) return;
  const int64_t tok = row / a.n_q_heads, lb = tok / a.n_new;
  const float* po = a.ws_o + row * parts * HD + d;
  const float2* pml = reinterpret_cast<const float2*>(a.ws_ml) + row * parts;
  float2 ml[kFewParts];
  f32x4_t x[kFewParts];
#pragma unroll
  for (int u = 0; u < kFewParts; ++u) {   // (past the last one of up to 8: that one again, with a weight of 0)
    const int s = kFewParts > 8 ? u : min(u, parts - 1);
    if (kFewParts == 8 || s < parts) {
      ml[u] = pml[s];
      x[u] = *reinterpret_cast<const f32x4_t*>(po + (int64_t)s * HD);
    }
  }
  if (tok - lb * a.n_new >= page_new_tokens(a.base_len, a.n_valid, (int)(lb % a.batch), a.n_new)) return;   // padding
  float M = kNoMax, den = 0.f;
#pragma unroll
  for (int u = 0; u < kFewParts; ++u)
    if (u < parts) M = fmaxf(M, ml[u].x);
  f32x4_t o = {};
#pragma unroll
  for (int u = 0; u < kFewParts; ++u)
    if (u < parts) {
      const float w = __builtin_amdgcn_exp2f(ml[u].x - M);
      den += w * ml[u].y;
      o += w * x[u];
    }
  float y[4] = {o[0], o[1], o[2], o[3]};
  odd_partials(y, parts, [&](int i, int e) { return po[(int64_t)i * HD + e]; });
  const float inv = 1.f / den;
  *reinterpret_cast<uint2*>(out + row * HD + d) = make_uint2(pack_bf16x2(y[0] * inv, y[1] * inv), pack_bf16x2(y[2] * inv, y[3] * inv));
}

template <int HD>
hipError_t launch_hd(const PageSharedArgs& a, const SharedPlan& plan, dim3 grid, const AttnShape& s, bf16_t* out, hipStream_t stream) {
  const auto kernel = plan.row_blocks == 1    ? (plan.stream ? page_shared_kernel<HD, 1, 2, true> : page_shared_kernel<HD, 1, 2, false>)
                      : plan.prefix_terms == 2 ? (plan.stream ? page_shared_kernel<HD, 2, 2, true> : page_shared_kernel<HD, 2, 2, false>)
                                               : (plan.stream ? page_shared_kernel<HD, 2, 1, true> : page_shared_kernel<HD, 2, 1, false>);
  hipLaunchKernelGGL(kernel, grid, dim3(256), 0, stream, a);
  const hipError_t e = hipGetLastError();
  if (e != hipSuccess) return e;
  // Few parts, or more rows than workgroups fit the GPU at once (2 layers of 12 x 5 tokens, 32 heads of 64, 9 parts: 27.2 -> 25
  // us for the call, 31.0 -> 29.0 with two terms; 224 rows of 16 parts 8.9 -> 9.3): lanes a row.  Else the combine of page_decode.hip, a workgroup a row
  // (512 rows of 28 parts 19.8 us, 21.0 the other way).
  const int parts = a.prefix_splits + a.own_splits;
  const int64_t row_count = (int64_t)s.n_layers * s.batch * a.n_new * s.n_q_heads;
  if (parts <= 8 || (parts <= 16 && row_count >= 2048)) {
    const auto join = parts <= 8 ? shared_combine_kernel<HD, 8> : shared_combine_kernel<HD, 16>;
    hipLaunchKernelGGL(join, dim3((unsigned)((row_count * (HD / 4) + 255) / 256)), dim3(256), 0, stream, a, out, row_count);
    return hipGetLastError();
  }
  AttnShape rows = s;   // (the combine's rows of a request: every head of every token)
  rows.n_q_heads = a.n_new * s.n_q_heads;
  return launch_decode_combine<HD, false, true>(a.ws_o, a.ws_ml, a.base_len, rows, a.max_base, 0, 0, parts, EqualDeal{}, out, stream,
                                                FewTokens{a.n_valid, a.n_new, s.n_q_heads});
}

}  // namespace

hipError_t launch_shared_bf16_pages(const PageAttnArgs& p, const SharedMap& m, const SharedPlan& plan) {
  const AttnShape& s = p.s;
  PageSharedArgs a = {};
  a.q = static_cast<const bf16_t*>(p.q);
  a.k_new = static_cast<const bf16_t*>(p.k_new);
  a.v_new = static_cast<const bf16_t*>(p.v_new);
  a.pages_k = static_cast<bf16_t*>(p.pages_k);
  a.pages_v = static_cast<bf16_t*>(p.pages_v);
  a.map = p.map;
  a.groups = m;
  a.base_len = p.base_len;
  a.n_valid = p.n_valid;
  a.ws_o = static_cast<float*>(p.workspace);
  a.ws_ml = a.ws_o + (size_t)s.n_layers * s.batch * p.n_new * s.n_q_heads * (plan.prefix_splits + plan.own_splits) * s.head_dim;
  a.batch = s.batch;
  a.stream_rows = s.cache_cap;
  a.n_q_heads = s.n_q_heads;
  a.n_kv_heads = s.n_kv_heads;
  a.n_new = p.n_new;
  a.max_base = p.max_base;
  a.offset = p.offset;
  a.prefix_splits = plan.prefix_splits;
  a.own_splits = plan.own_splits;
  a.prefix_row_tiles = plan.prefix_row_tiles;
  a.own_row_tiles = plan.own_row_tiles;
  a.prefix_blocks = (int32_t)plan.prefix_blocks;
  a.scale_log2 = s.scale_log2;
  const dim3 grid((unsigned)(plan.prefix_blocks + plan.own_blocks), s.n_layers);
  bf16_t* out = static_cast<bf16_t*>(p.out);
  return s.head_dim == 64 ? launch_hd<64>(a, plan, grid, s, out, p.stream) : launch_hd<128>(a, plan, grid, s, out, p.stream);
}

}  // namespace pic
