// Index clamping of libpic's kernels: every index a kernel derives from a device-side table
// (gather blocks, group starts, slot and tile maps, context and base lengths, position shifts)
// goes through one of these checks before it addresses memory, so a wrong table gives wrong
// values, never an access outside the buffers whose sizes the host passed.
//
// The functions are __host__ __device__: the kernels call them, and the CPU emulation of the
// launches that the sanitizer tests build (AddressSanitizer, UndefinedBehaviorSanitizer) calls
// the same code on host buffers of the exact sizes.  (Rows of a paged cache the kernels find through a
// PageWindow, the emulation by page_row; that the two agree is a test of its own.)
#pragma once

#include <stdint.h>

#include "pic.h"

#if defined(__HIPCC__) || defined(__HIP__)
#include <hip/hip_runtime.h>
#define PIC_HD __host__ __device__ __forceinline__
#else
#define PIC_HD inline
#endif

namespace pic {

PIC_HD int32_t clamp_i32(int32_t v, int32_t lo, int32_t hi) { return v < lo ? lo : (v > hi ? hi : v); }

// A position shift, clamped to the table's rows (|delta| <= max_abs_delta).
PIC_HD int32_t clamp_delta(int32_t d, int32_t max_abs_delta) { return clamp_i32(d, -max_abs_delta, max_abs_delta); }

// A per-request length read from the device (context or base length), clamped to [0, max_len].
PIC_HD int32_t clamp_len(int32_t n, int32_t max_len) { return clamp_i32(n, 0, max_len); }

// A pool token read from a slot map, clamped into the pool (pool_tokens >= 1).
PIC_HD int32_t clamp_pool_token(int32_t t, int64_t pool_tokens) {
  return t < 0 ? 0 : (t >= pool_tokens ? (int32_t)(pool_tokens - 1) : t);
}

// The pool run a gather block reads lies inside the pool.
PIC_HD bool block_source_ok(const pic_block& b, int64_t pool_tokens) {
  return b.n_tokens > 0 && b.n_tokens <= PIC_BLOCK_TOKENS && b.src_token >= 0 &&
         (int64_t)b.src_token + b.n_tokens <= pool_tokens;
}

// The cache slots a gather block writes lie inside the caches, and its shift inside the table.
PIC_HD bool block_dest_ok(const pic_block& b, int32_t batch, int32_t cache_cap, int32_t max_abs_delta) {
  return b.request >= 0 && b.request < batch && b.n_tokens > 0 && b.n_tokens <= PIC_BLOCK_TOKENS &&
         b.dst_slot >= 0 && (int64_t)b.dst_slot + b.n_tokens <= cache_cap && b.delta <= max_abs_delta &&
         b.delta >= -max_abs_delta;
}

// A gather block composition may move (compose_kernel).
PIC_HD bool block_ok(const pic_block& b, int32_t batch, int64_t pool_tokens, int32_t cache_cap,
                     int32_t max_abs_delta) {
  return block_source_ok(b, pool_tokens) && block_dest_ok(b, batch, cache_cap, max_abs_delta);
}

// A block of a shared-source group: it must read its group's run (the first block's) and write
// inside the caches.
PIC_HD bool shared_block_ok(const pic_block& b, const pic_block& run, int32_t batch, int32_t cache_cap,
                            int32_t max_abs_delta) {
  return b.src_token == run.src_token && b.n_tokens == run.n_tokens &&
         block_dest_ok(b, batch, cache_cap, max_abs_delta);
}

// Blocks [g0, g1) of a group, from two group starts clamped to [0, n_blocks].
PIC_HD void group_range(int32_t start, int32_t end, int32_t n_blocks, int32_t& g0, int32_t& g1) {
  g0 = start < 0 ? 0 : start;
  g1 = end > n_blocks ? n_blocks : end;
}

// A gather block the slot map may expand: its request and slots inside the map.
PIC_HD bool map_block_ok(const pic_block& b, int32_t batch, int32_t map_cap) {
  return b.request >= 0 && b.request < batch && b.n_tokens > 0 && b.n_tokens <= PIC_BLOCK_TOKENS &&
         b.dst_slot >= 0 && (int64_t)b.dst_slot + b.n_tokens <= map_cap;
}

// A tile-map entry (src, delta) for context tile [s0, s0 + 64) of a request with ctx context
// tokens is read from the pool in one piece only when the whole run lies in the pool, its shift
// in the table, and the tile in the context.
PIC_HD bool tile_run_ok(int32_t src, int32_t delta, int32_t s0, int32_t ctx, int64_t pool_tokens,
                        int32_t max_abs_delta) {
  return src >= 0 && (int64_t)src + PIC_BLOCK_TOKENS <= pool_tokens && delta >= -max_abs_delta &&
         delta <= max_abs_delta && s0 + PIC_BLOCK_TOKENS <= ctx;
}

// ---- Paged caches: slot t of request b lives in row page * P + t % P of its (layer, kv head)
// stream, page = table[b][t / P], P = 1 << shift; a stream holds n_pages * P rows.
struct PageMap {
  const int32_t* table = nullptr;   // [batch][cap]
  int32_t cap = 0, n_pages = 0, shift = 0;
};
// Entry i of a request's page table, as a page to read: clamped into the table and the pages.
PIC_HD int32_t clamp_entry(int32_t i, const PageMap& m) { return clamp_i32(i, 0, m.cap - 1); }
PIC_HD int32_t clamp_page(int32_t page, const PageMap& m) { return clamp_i32(page, 0, m.n_pages - 1); }
// A wave's view of its request's page table as its keys go by: lane j of one register holds entry at + j, of
// another one entry at + step + j, loaded a window ahead.  The kernels walk it with these two and take entry i out of
// lane lane(i).
struct PageWindow {
  int32_t at;
  // Entry i is the next one asked for, no more than `step` past the last one.  True: the window has moved on by step
  // (the second register becomes the first, and is loaded anew).
  PIC_HD bool moves(int32_t i, int32_t step) {
    if (i < at + step) return false;
    at += step;
    return true;
  }
  PIC_HD int32_t lane(int32_t i) const { return i - at; }
};
// The row `slot` of request b is read from (slot >= 0), found without a window.
PIC_HD int64_t page_row(const PageMap& m, int32_t b, int32_t slot) {
  const int32_t page = clamp_page(m.table[(int64_t)b * m.cap + clamp_entry(slot >> m.shift, m)], m);
  return ((int64_t)page << m.shift) + (slot & ((1 << m.shift) - 1));
}
// The row `slot` of request b is stored to, -1 where the table gives it no page.
PIC_HD int64_t page_store_row(const PageMap& m, int32_t b, int32_t slot) {
  const int32_t i = slot >> m.shift;
  if (i < 0 || i >= m.cap) return -1;
  const int32_t page = m.table[(int64_t)b * m.cap + i];
  if (page < 0 || page >= m.n_pages) return -1;
  return ((int64_t)page << m.shift) + (slot & ((1 << m.shift) - 1));
}
// New tokens of request b that a call over pages uses: none where its length is negative (padding
// of the batch), else n_valid[b] of the n_new, or all of them.
PIC_HD int32_t page_new_tokens(const int32_t* base_len, const int32_t* n_valid, int32_t b, int32_t n_new) {
  if (base_len[b] < 0) return 0;
  return n_valid ? clamp_len(n_valid[b], n_new) : n_new;
}

// ---- Requests that share a prefix: group i holds requests [start[i], start[i + 1]) (without starts, group 0 the whole
// batch), the first max_group of them served together over slots [0, shared_len[i]) of its first request's pages.
constexpr int32_t kSharedKeys = 64;   // the part that is served together ends with a whole tile
struct SharedMap {
  const int32_t* start = nullptr;   // [n_groups + 1]
  const int32_t* len = nullptr;     // [n_groups]
  int32_t n_groups = 0, max_group = 0, max_len = 0, batch = 0;

  PIC_HD int32_t first(int32_t i) const { return start ? clamp_i32(start[i], 0, batch) : (i == 0 ? 0 : batch); }
  PIC_HD int32_t requests(int32_t i) const {
    const int32_t n = first(i + 1) - first(i);
    return n < 0 ? 0 : (n < max_group ? n : max_group);
  }
  // Slots of group i that are served together.
  PIC_HD int32_t slots(int32_t i) const { return clamp_len(len[i], max_len) & ~(kSharedKeys - 1); }
  // The group whose prefix request b is served with, -1: none.  (Starts that do not increase: some group, or none.)
  PIC_HD int32_t group_of(int32_t b) const {
    int32_t lo = 0, hi = n_groups;   // first(lo) <= b < first(hi), once it is known that first(0) <= b
    while (hi - lo > 1) {
      const int32_t mid = lo + (hi - lo) / 2;
      if (first(mid) <= b) lo = mid;
      else hi = mid;
    }
    return b >= first(lo) && b - first(lo) < requests(lo) ? lo : -1;
  }
};
// Slots of a request that its group serves, of a group that serves `slots` of them: whole tiles before the first new
// token, at `ctx`.
PIC_HD int32_t shared_part(int32_t slots, int32_t ctx) {
  const int32_t whole = ctx & ~(kSharedKeys - 1);
  return slots < whole ? slots : whole;
}

// ---- Split decode: the key ranges of a batch of uneven contexts ----
// A split launch has n_splits workgroups per (request, kv head).  They are dealt to the requests
// by length: request b of u_b units (kDecodeUnit keys each, the last one partial) gets
// ceil(u_b / c) ranges of c units, c the smallest size for which the batch's ranges fit
// n_splits * batch.  Candidate i of 64 for c, from the mean up to the size at which the longest
// request alone takes n_splits ranges (which always fits):
constexpr int32_t kDecodeUnit = 128;        // keys; every range is a multiple
constexpr int32_t kDecodeDealt = 64;        // most requests whose ranges are dealt by length
// Dealing takes 0.9 us (in the kernel and in its combine) and rounds each request's last range up,
// so it is for launches of many ranges of long contexts.  Equal ranges / dealt: 8 requests of 16K
// to 33K keys in 8 ranges each 81 / 68 us, of 33K each 86.6 / 87.3; 4 of 5K to 10K in 8 29.1 /
// 25.8, 4 of 4K 16.4 / 17.3; 16 of 5K to 10K in 2 87.5 / 91.7.
PIC_HD bool decode_dealt(int32_t n_splits, int32_t batch, int32_t max_len) {
  return n_splits >= 8 && batch >= 2 && batch <= kDecodeDealt && max_len >= 8192;
}
PIC_HD int32_t decode_units(int32_t n_keys) { return (int32_t)(((uint32_t)n_keys + kDecodeUnit - 1) / kDecodeUnit); }
PIC_HD int32_t ceil_div(int32_t n, int32_t d) { return (int32_t)(((uint32_t)n + (uint32_t)d - 1) / (uint32_t)d); }
struct RangeCandidates {
  int32_t lo, step, top;
  PIC_HD int32_t at(int32_t i) const {   // i < 64: the last one is top
    const int32_t c = lo + step * i;
    return c < top ? c : top;
  }
};
// (at most 64 requests of at most 2^24 units: every sum fits 32 bits)
PIC_HD RangeCandidates decode_range_candidates(int32_t units_total, int32_t units_longest, int32_t n_splits,
                                               int32_t batch) {
  const int32_t s = n_splits < units_longest ? n_splits : units_longest;
  RangeCandidates r;
  r.lo = ceil_div(units_total, s * batch);
  r.top = ceil_div(units_longest, s);
  r.step = ceil_div(r.top > r.lo ? r.top - r.lo : 1, kDecodeDealt - 1);
  return r;
}

// ---- Split prefill over pages: the key ranges of uneven requests ----
// A split launch has n_splits workgroups per (request, kv head, tile of query rows).  Request b with u_b key
// tiles, t_b used tokens and m_b tiles of query rows gets ceil(u_b / c) equal ranges, c the smallest size for
// which workgroups (sum of m_b ceil(u_b / c)) and partials (of t_b ceil(u_b / c)) fit in those of n_splits ranges
// of every request.  Candidates as above, from the mean, of 8 tiles at least (the combine reads a row's
// partials one after another), up to what always fits; and where that is not enough shorter than the
// longest request's share, every request gets n_splits ranges.  Equal shares / dealt, us, by c of that
// share's tiles: 5 of 2K to 4K keys x 1 to 67 tokens (head_dim 64) 15 of 23 37.6 / 30.8; 6 of 15K to 33K x 100
// (28 heads over 4) 74 of 103 260 / 207; 8 of 5K to 10K x 64 33 of 41 96 / 92.  Shorter by less than an eighth
// or 4 tiles is not worth the 1.5 us that the combine's longer rows cost (4 of 7K to 10K x 32, 19 of 21, 45.3 /
// 47.2); finding that out costs 1 us where lengths differ, and nothing that shows where they are equal.
PIC_HD bool suffix_dealt(int32_t n_splits, int32_t batch) { return n_splits >= 2 && batch >= 2 && batch <= kDecodeDealt; }
PIC_HD bool suffix_deal_pays(int32_t size, int32_t top) { return size + 4 <= top && size <= top - top / 8; }
// tiles_total: sum of m_b u_b;  groups: batch * (tiles of the longest request's query rows)
PIC_HD RangeCandidates suffix_range_candidates(int64_t tiles_total, int32_t tiles_longest, int32_t n_splits, int32_t groups) {
  RangeCandidates r;
  r.top = ceil_div(tiles_longest, n_splits < tiles_longest ? n_splits : tiles_longest);
  const int64_t wgs = (int64_t)n_splits * groups;
  const int32_t mean = (int32_t)((tiles_total + wgs - 1) / wgs), least = r.top < 8 ? r.top : 8;
  r.lo = mean > least ? mean : least;
  r.step = ceil_div(r.top > r.lo ? r.top - r.lo : 1, kDecodeDealt - 1);
  return r;
}
// Workgroup `block` of a dealt launch, whose `total` workgroups are shared out to the XCDs in neighbours: its request,
// kv head, key range and tile of query rows (the last first), and the partials' tokens of the requests before.
// Request b has wgs(b) = heads * ranges(b) * row_tiles(b) workgroups.  False: none is left for it.
struct DealtBlock {
  int32_t b, g, split, mt, ranges, row_tiles, first;
};
template <typename W, typename R, typename M, typename T>
PIC_HD bool dealt_block(int32_t block, int32_t xcds, int32_t total, W wgs, R ranges, M row_tiles, T tokens, DealtBlock& x) {
  const int32_t per = (total + xcds - 1) / xcds, at = block / xcds;
  int32_t in_b = (block % xcds) * per + at;
  if (at >= per || in_b >= total) return false;
  x.first = 0;
  for (x.b = 0; in_b >= wgs(x.b); ++x.b) {
    in_b -= wgs(x.b);
    x.first += ranges(x.b) * tokens(x.b);
  }
  x.ranges = ranges(x.b);
  x.row_tiles = row_tiles(x.b);
  x.mt = x.row_tiles - 1 - in_b % x.row_tiles;
  x.split = (in_b / x.row_tiles) % x.ranges;
  x.g = in_b / (x.row_tiles * x.ranges);
  return true;
}
// ceil(u / c) for 0 <= u <= 2^24, 1 <= c, inv ~ 1 / c: a float32 quotient, off by one at most, put right
PIC_HD int32_t ceil_div24(int32_t u, int32_t c, float inv) {
  int32_t q = (int32_t)((float)u * inv);
  const int32_t r = u - q * c;
  return q + (r > 0 ? 1 : 0) + (r > c ? 1 : 0) - (r <= -c ? 1 : 0);
}

}  // namespace pic
