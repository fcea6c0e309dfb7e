// Page copies of a paged cache: page dst = page src in every (layer, kv head) stream of K and V.
//
// The streams lie n_pages * page_bytes apart, so one page copy is 2 * streams pieces of page_bytes
// (16 KB at 64 tokens of head_dim 128 in bf16) at one offset; nothing is computed, and the bound is
// the rate of a large copy.  A workgroup takes one piece.
#include "pic_internal.h"

namespace pic {
namespace {

// The pairs travel as kernel arguments (argument blocks hold 4 KB): a list on the device would
// cost the caller an upload and the kernel a dependent load before its first page.
constexpr int kPairs = 256;
struct Pairs {
  int2 p[kPairs];
};

// grid (pairs, min(streams, 65535)), 256 threads
__global__ void __launch_bounds__(256) page_copy_kernel(uint4* k, uint4* v, int64_t n_streams, int64_t stream16,
                                                        int32_t page16, Pairs pairs) {
  const int2 p = pairs.p[blockIdx.x];
  for (int64_t st = blockIdx.y; st < 2 * n_streams; st += gridDim.y) {
    uint4* base = (st < n_streams ? k + st * stream16 : v + (st - n_streams) * stream16);
    const uint4* src = base + (int64_t)p.x * page16;
    uint4* dst = base + (int64_t)p.y * page16;
    for (int i = threadIdx.x; i < page16; i += 256) dst[i] = src[i];
  }
}

}  // namespace

hipError_t launch_page_copy(void* pages_k, void* pages_v, int64_t n_streams, int64_t n_pages, int64_t page_bytes,
                            const int32_t* pairs, int32_t n_pairs, hipStream_t stream) {
  const int64_t page16 = page_bytes / 16;
  const unsigned gy = (unsigned)(2 * n_streams < 65535 ? 2 * n_streams : 65535);
  for (int32_t i0 = 0; i0 < n_pairs; i0 += kPairs) {
    const int n = n_pairs - i0 < kPairs ? n_pairs - i0 : kPairs;
    Pairs p = {};
    for (int i = 0; i < n; ++i) p.p[i] = make_int2(pairs[2 * (i0 + i)], pairs[2 * (i0 + i) + 1]);
    hipLaunchKernelGGL(page_copy_kernel, dim3(n, gy), dim3(256), 0, stream, static_cast<uint4*>(pages_k),
                       static_cast<uint4*>(pages_v), n_streams, n_pages * page16, (int32_t)page16, p);
    const hipError_t e = hipGetLastError();
    if (e != hipSuccess) return e;
  }
  return hipSuccess;
}

}  // namespace pic
