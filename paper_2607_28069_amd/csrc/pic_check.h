// What the files of the C ABI share: the thread-local error, argument checks and launch decisions
// (defined in pic_api.cpp).
#pragma once

#include "pic.h"
#include "pic_internal.h"

#define PIC_API extern "C" __attribute__((visibility("default")))

#define PIC_CHECK(expr)              \
  do {                               \
    pic_status _s = (expr);          \
    if (_s != PIC_OK) return _s;     \
  } while (0)

namespace pic {

// Largest position shift (and rotary position) of a table.
constexpr int32_t kMaxAbsDelta = 1 << 20;
// The bf16 attention kernels address a cache stream (one layer, request and kv head), one
// request's suffix rows and a pool head (one layer and kv head) with 32-bit byte offsets from
// a buffer base: each must stay under 2^32 bytes (rows of 256 bytes).
constexpr int64_t kMaxRows32 = (int64_t(1) << 32) / 256 - 1;

// fail() leaves the message for pic_last_error and returns `st`; ok() clears it.
pic_status fail(pic_status st, const char* fmt, ...);
pic_status ok();
pic_status hip_status(hipError_t e, const char* what);
bool aligned16(const void* p);
pic_status check_ptr(const void* p, const char* name);
pic_status check_model(const pic_model* m);
pic_status check_rows32(int64_t cache_cap, int64_t suffix_rows, int64_t pool_tokens);
int32_t n_tables(const pic_model* m);
AttnShape shape_of(const pic_model* m, int32_t batch, int32_t cache_cap, float scale);
pic_status check_prefill_workspace(const pic_model* m, int32_t batch, int32_t n_suffix, int32_t max_ctx,
                                   const void* workspace, size_t* ws_bytes);
pic_status plan_decode_call(const pic_model* model, const AttnShape& s, int32_t max_len, bool use_scratch,
                            int32_t* n_splits_io, void** workspace_io, size_t* ws_bytes_io);

}  // namespace pic
