// Page tables grown on the device from the requests' lengths, entry for entry what pic_page_grow does on the host, and
// the page copies that it asks for.
//
// Growing is a few integers behind a chain of loads that wait for one another (lengths -> table entries -> reference
// counts -> free pages -> the entries that take them), so one workgroup does it all: that chain bounds it, and a second
// workgroup would add a launch or a wait between the two.  What can be asked for early is (the first pages' counts), and
// what the first pass over a decode step's entries finds stays in registers: 64 requests of 16384 tokens over 20000 pages
// of 64 7.8 us, where a pass that found each place again before every step took 10.6.  The order of the host's
// loop (request by request, entry by entry) comes from prefix sums over the workgroup; where several entries hold the
// same shared page, the k-th of them takes a page of its own if the page has more than k + 1 references, so the last
// ones keep it.  Where not everything fits, nothing is changed (references given back are taken again).
#include "pic_bounds.h"
#include "pic_internal.h"

namespace pic {
namespace {

constexpr int kThreads = 1024, kWaves = kThreads / 64;

// Exclusive prefix sums of x over the workgroup, in thread order, and its total.  `sums` is reused by the next call.
struct Scan {
  int before, total;
};
__device__ __forceinline__ Scan scan(int x, int (&sums)[kWaves]) {
  const int lane = threadIdx.x & 63, wave = threadIdx.x >> 6;
  int in = x;
#pragma unroll
  for (int d = 1; d < 64; d <<= 1) {
    const int y = __shfl_up(in, d, 64);
    if (lane >= d) in += y;
  }
  __syncthreads();   // (the last call's sums are read)
  if (lane == 63) sums[wave] = in;
  __syncthreads();
  int before = 0, total = 0;
#pragma unroll
  for (int w = 0; w < kWaves; ++w) {
    before += w < wave ? sums[w] : 0;
    total += sums[w];
  }
  return {before + in - x, total};
}

// 1 workgroup.  workspace: first[batch + 1] (a request's first entry in the order), then of every entry in the order its
// page where it is shared (shared[]), where in the order that was (at[]) and what becomes of it (take[]), and the free
// pages in order (lowest[]).  The first kThreads entries, which are all of them in a decode step, stay in registers, the
// first kFirst requests' places in LDS, and the first pages' reference counts are on their way from the start.
__global__ void __launch_bounds__(kThreads) page_grow_kernel(PageGrowArgs a, int32_t cap_entries) {
  constexpr int kFirst = 4096, kPer = 16;   // requests in LDS; pages a thread looks at at once
  __shared__ int sums[kWaves];
  __shared__ int32_t first_lds[kFirst + 1], held_lds[kThreads];
  __shared__ int bad_cap, bad_entry;
  const int tid = threadIdx.x;
  int32_t* first = a.batch <= kFirst ? first_lds : a.workspace;
  int32_t* shared = a.workspace + a.batch + 1;
  int32_t* at = shared + cap_entries;
  int32_t* take = at + cap_entries;
  int32_t* lowest = take + cap_entries;
  const int32_t P = 1 << a.shift;
  int4 refs[kPer / 4];
  auto look = [&](int64_t p0) {   // at pages [p0, p0 + kPer) (past the last one: not free)
#pragma unroll
    for (int u = 0; u < kPer / 4; ++u) {
      const int64_t p = p0 + 4 * u;
      if (p + 4 <= a.n_pages) refs[u] = *reinterpret_cast<const int4*>(a.refs + p);
      else refs[u] = make_int4(p < a.n_pages ? a.refs[p] : 1, p + 1 < a.n_pages ? a.refs[p + 1] : 1, p + 2 < a.n_pages ? a.refs[p + 2] : 1, 1);
    }
  };
  look((int64_t)kPer * tid);
  if (tid == 0) bad_cap = bad_entry = 0;
  __syncthreads();
  // 1. the entries each request's new slots, [base + offset, + n), lie in
  int32_t entries = 0;
  for (int b0 = 0; b0 < a.batch; b0 += kThreads) {
    const int b = b0 + tid;
    int n = 0;
    if (b < a.batch) {
      const int64_t from = (int64_t)a.base_len[b] + a.offset, to = from + page_new_tokens(a.base_len, a.n_valid, b, a.n_new);
      const int64_t end = (to + P - 1) >> a.shift;
      if (to > from) {
        if (end > a.table_cap) bad_cap = 1;
        else n = (int)(end - (from >> a.shift));
      }
    }
    const Scan s = scan(n, sums);
    if (b < a.batch) first[b] = entries + s.before;
    entries += s.total;
  }
  if (tid == 0) first[a.batch] = entries;
  __syncthreads();
  bool fits = bad_cap == 0;   // (then at most cap_entries of them)
  // Entry e of the order: where it lies in the table, and whether new slots take only part of it.
  struct Place {
    int32_t* entry;
    bool partly;
  };
  auto locate = [&](int e) -> Place {
    int lo = 0, hi = a.batch;   // first[lo] <= e < first[hi]
    while (hi - lo > 1) {
      const int mid = (lo + hi) >> 1;
      if (first[mid] <= e) lo = mid;
      else hi = mid;
    }
    const int64_t from = (int64_t)a.base_len[lo] + a.offset;
    return {a.page_table + (int64_t)lo * a.table_cap + (from >> a.shift) + (e - first[lo]), e == first[lo] && (from & (P - 1)) != 0};
  };
  // 2. what becomes of each: 0 kept, 1 takes a page, 2 shared (settled below).  In the order, `ranks` entries take a page before
  // this thread's of the first kThreads (where none is shared).
  int32_t n_shared = 0, takes = 0;
  Place place = {nullptr, false};
  int32_t page0 = -1;
  int kind0 = 0, ranks = 0;
  if (fits) {
    for (int e0 = 0; e0 < entries; e0 += kThreads) {
      const int e = e0 + tid;
      int kind = 0;
      int32_t page = -1;
      if (e < entries) {
        const Place x = locate(e);
        page = *x.entry;
        if (page == -1 && !x.partly) {
          kind = 1;
        } else if (page < 0 || page >= a.n_pages) {
          bad_entry = 1;
        } else {
          const int32_t held = a.refs[page];
          if (held < 1) bad_entry = 1;
          kind = held > 1 ? 2 : 0;
        }
        if (e0 == 0) place = x, page0 = page, kind0 = kind;
        else take[e] = kind;
      }
      const Scan s = scan((kind == 2) << 16 | (kind == 1), sums);   // (each at most kThreads)
      if (kind == 2) {
        shared[n_shared + (s.before >> 16)] = page;
        at[n_shared + (s.before >> 16)] = e;
      }
      if (e0 == 0) ranks = s.before & 0xFFFF;
      n_shared += s.total >> 16;
      takes += s.total & 0xFFFF;
    }
    __syncthreads();
    fits = bad_entry == 0;
  }
  const bool known = fits;   // (bad tables: nothing is counted)
  int32_t copies = 0, found = 0;
  if (fits) {
    if (n_shared > 0) {
      // (of the first kThreads too, through take[])
      if (tid < entries) take[tid] = kind0;
      // kThreads of them at a time: those before them have given their references back (which the next ones see, past the
      // first-level cache), and the places among the same page's come from LDS
      for (int s0 = 0; s0 < n_shared; s0 += kThreads) {
        const int s = s0 + tid;
        const int32_t page = s < n_shared ? shared[s] : -1;
        held_lds[tid] = page;
        __syncthreads();
        int kind = 0;
        if (s < n_shared) {
          int rank = 0;
          for (int k = 0; k < tid; ++k) rank += held_lds[k] == page;
          if (__hip_atomic_load(a.refs + page, __ATOMIC_RELAXED, __HIP_MEMORY_SCOPE_AGENT) - rank > 1)
            kind = locate(at[s]).partly ? 3 : 1;   // 3: and is copied
          take[at[s]] = kind;
        }
        takes += scan(kind != 0, sums).total;   // (every count is read)
        if (kind != 0) atomicSub(a.refs + page, 1);
        if (s0 + kThreads < n_shared) __threadfence();
        __syncthreads();
      }
      __syncthreads();
      if (tid < entries) kind0 = take[tid];
    }
    // 3. as many free pages, lowest first
    for (int64_t p0 = 0; p0 < a.n_pages && found < takes; p0 += kPer * kThreads) {
      const int64_t p = p0 + (int64_t)kPer * tid;
      if (p0 > 0) look(p);
      int n = 0;
#pragma unroll
      for (int u = 0; u < kPer / 4; ++u) n += (refs[u].x == 0) + (refs[u].y == 0) + (refs[u].z == 0) + (refs[u].w == 0);
      const Scan s = scan(n, sums);
      int k = found + s.before;
      if (n > 0 && k < takes) {
#pragma unroll
        for (int u = 0; u < kPer; ++u) {
          const int32_t held = u % 4 == 0 ? refs[u / 4].x : u % 4 == 1 ? refs[u / 4].y : u % 4 == 2 ? refs[u / 4].z : refs[u / 4].w;
          if (held == 0) {
            if (k < takes) lowest[k] = (int32_t)(p + u);
            ++k;
          }
        }
      }
      found += s.total;
    }
    __syncthreads();
    fits = found >= takes;
    if (!fits) {   // shared pages get their references back
      for (int s = tid; s < n_shared; s += kThreads)
        if (take[at[s]] != 0) atomicAdd(a.refs + shared[s], 1);
    }
  }
  // 4. the tables changed
  if (fits && takes > 0) {
    int32_t taken = 0;
    for (int e0 = 0; e0 < entries; e0 += kThreads) {
      const int e = e0 + tid;
      const int kind = e0 == 0 ? kind0 : e < entries ? take[e] : 0;
      Scan s = {ranks, 0}, c = {0, 0};
      if (n_shared > 0 || entries > kThreads) {
        s = scan((kind == 3) << 16 | (kind != 0), sums);
        c = {s.before >> 16, s.total >> 16};
        s = {s.before & 0xFFFF, s.total & 0xFFFF};
      }
      if (kind != 0) {
        if (e0 > 0) {
          place = locate(e);
          page0 = *place.entry;
        }
        const int32_t page = lowest[taken + s.before];
        a.refs[page] = 1;
        *place.entry = page;
        if (kind == 3) {
          a.pairs[2 * (copies + c.before)] = page0;
          a.pairs[2 * (copies + c.before) + 1] = page;
        }
      }
      taken += s.total;
      copies += c.total;
    }
  }
  for (int64_t i = 2 * (int64_t)copies + tid; i < 2 * (int64_t)a.batch; i += kThreads) a.pairs[i] = -1;
  for (int b = tid; b < a.batch; b += kThreads) {
    const int32_t base = a.base_len[b];
    a.ready[b] = fits && base >= 0 ? base : -1;
  }
  if (tid == 0) {
    a.result[0] = fits ? PIC_OK : bad_cap || known ? PIC_ERR_CAPACITY : PIC_ERR_RANGE;
    a.result[1] = copies;
    a.result[2] = known ? takes : 0;
  }
}

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// Any grid, 256 threads.  Pairs come 64 at a time; a workgroup takes every gridDim.x-th piece (a pair in one stream) of
// those that are pairs, so that a list without any costs one load.
__global__ void __launch_bounds__(256) page_copy_listed_kernel(u32x4* k, u32x4* v, int64_t n_streams, int64_t stream16,
                                                               int32_t page16, const int2* pairs, int32_t cap, int32_t n_pages) {
  constexpr int kAhead = 4;
  __shared__ int2 found[64];
  const int lane = threadIdx.x & 63;
  for (int64_t i0 = 0; i0 < cap; i0 += 64) {
    const int2 mine = i0 + lane < cap ? pairs[i0 + lane] : make_int2(-1, -1);
    const bool ok = mine.x >= 0 && mine.x < n_pages && mine.y >= 0 && mine.y < n_pages;
    const uint64_t mask = __ballot(ok);
    const int n = __popcll(mask);
    if (n == 0) continue;   // (uniform: every wave holds the same 64)
    __syncthreads();
    if (ok && threadIdx.x < 64) found[__popcll(mask & ((uint64_t(1) << lane) - 1))] = mine;
    __syncthreads();
    for (int64_t at = blockIdx.x; at < n * 2 * n_streams; at += gridDim.x) {
      const int32_t pair = (int32_t)(at / (2 * n_streams));
      const int64_t st = at - pair * 2 * n_streams;
      const int2 p = found[pair];
      u32x4* base = st < n_streams ? k + st * stream16 : v + (st - n_streams) * stream16;
      const u32x4* src = base + (int64_t)p.x * page16;
      u32x4* dst = base + (int64_t)p.y * page16;
      for (int i = threadIdx.x; i < page16; i += 256 * kAhead) {
        u32x4 x[kAhead];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (i + 256 * u < page16) x[u] = src[i + 256 * u];
#pragma unroll
        for (int u = 0; u < kAhead; ++u)
          if (i + 256 * u < page16) __builtin_nontemporal_store(x[u], dst + i + 256 * u);
      }
    }
  }
}

}  // namespace

hipError_t launch_page_grow(const PageGrowArgs& a, hipStream_t stream) {
  const int64_t entries = page_grow_entries(1 << a.shift, a.table_cap, a.batch, a.n_new);
  hipLaunchKernelGGL(page_grow_kernel, dim3(1), dim3(kThreads), 0, stream, a, (int32_t)entries);
  return hipGetLastError();
}

hipError_t launch_page_copy_listed(void* pages_k, void* pages_v, int64_t n_streams, int64_t n_pages, int64_t page_bytes,
                                   const int32_t* pairs, int32_t cap, hipStream_t stream) {
  const int64_t page16 = page_bytes / 16;
  const unsigned grid = (unsigned)std::min<int64_t>((int64_t)cap * 2 * std::min<int64_t>(n_streams, 2048), 2048);
  hipLaunchKernelGGL(page_copy_listed_kernel, dim3(grid), dim3(256), 0, stream, static_cast<u32x4*>(pages_k),
                     static_cast<u32x4*>(pages_v), n_streams, n_pages * page16, (int32_t)page16,
                     reinterpret_cast<const int2*>(pairs), cap, (int32_t)n_pages);
  return hipGetLastError();
}

}  // namespace pic
