// Page copies of a paged cache: page dst = page src in every (layer, kv head) stream of K and V.
//
// The streams lie n_pages * page_bytes apart, so one page copy is 2 * streams pieces of page_bytes
// (16 KB at 64 tokens of head_dim 128 in bf16) at one offset; nothing is computed, and the bound is
// the rate of a large copy (4.8 TB/s read and written for a library copy of 4 GB).  A workgroup takes one
// piece, each thread with four 16-byte loads before its first store.  Stores are non-temporal: what they
// write is not read soon, and reads keep the caches (15 pages of 64 tokens in 32 layers, 252 MB: 52.2 ->
// 44.4 us, 5.7 TB/s; 208 pages of 128 tokens in 28 layers, 3.05 GB: 590 -> 575).  Loads are too where a call
// reads more than the 256 MB last-level cache could have kept from before (575 -> 554, 5.5 TB/s; the
// 252 MB call, which reads 126, would go from 44.4 to 47.5).
#include "pic_internal.h"

namespace pic {
namespace {

// The pairs travel as kernel arguments (argument blocks hold 4 KB): a list on the device would
// cost the caller an upload and the kernel a dependent load before its first page.
constexpr int kPairs = 256;
struct Pairs {
  int2 p[kPairs];
};

typedef uint32_t u32x4 __attribute__((ext_vector_type(4)));

// grid (pairs, min(pieces, 65535)), 256 threads
template <bool kStream>
__global__ void __launch_bounds__(256) page_copy_kernel(u32x4* k, u32x4* v, int64_t n_streams, int64_t stream16,
                                                        int32_t page16, Pairs pairs) {
  constexpr int kAhead = 4;
  const int2 p = pairs.p[blockIdx.x];
  for (int64_t st = blockIdx.y; st < 2 * n_streams; st += gridDim.y) {
    u32x4* base = st < n_streams ? k + st * stream16 : v + (st - n_streams) * stream16;
    const u32x4* src = base + (int64_t)p.x * page16;
    u32x4* dst = base + (int64_t)p.y * page16;
    for (int i = threadIdx.x; i < page16; i += 256 * kAhead) {
      u32x4 x[kAhead];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i + 256 * u < page16) x[u] = kStream ? __builtin_nontemporal_load(src + i + 256 * u) : src[i + 256 * u];
#pragma unroll
      for (int u = 0; u < kAhead; ++u)
        if (i + 256 * u < page16) __builtin_nontemporal_store(x[u], dst + i + 256 * u);
    }
  }
}

}  // namespace

hipError_t launch_page_copy(void* pages_k, void* pages_v, int64_t n_streams, int64_t n_pages, int64_t page_bytes,
                            const int32_t* pairs, int32_t n_pairs, hipStream_t stream) {
  const int64_t page16 = page_bytes / 16;
  const bool stream_loads = (double)n_pairs * 2.0 * (double)n_streams * (double)page_bytes > 256e6;
  const unsigned gy = (unsigned)(2 * n_streams < 65535 ? 2 * n_streams : 65535);
  for (int32_t i0 = 0; i0 < n_pairs; i0 += kPairs) {
    const int n = n_pairs - i0 < kPairs ? n_pairs - i0 : kPairs;
    Pairs p = {};
    for (int i = 0; i < n; ++i) p.p[i] = make_int2(pairs[2 * (i0 + i)], pairs[2 * (i0 + i) + 1]);
    hipLaunchKernelGGL(stream_loads ? page_copy_kernel<true> : page_copy_kernel<false>, dim3(n, gy), dim3(256), 0, stream,
                       static_cast<u32x4*>(pages_k), static_cast<u32x4*>(pages_v), n_streams, n_pages * page16,
                       (int32_t)page16, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pic
