// Handle of the paged KV$ operators, shared by kv.cu and attention.cu.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include "smetric_impl.cuh"

namespace smetric {

// Where a planned token goes. slot: page * page_size + place in the page, or
// -1 for a token that is left out; pos: its position in its request.
struct KvToken {
  int64_t slot;
  int32_t pos;
  int32_t req;
};

// The plan's device-side summary.
struct KvPlan {
  int64_t first, last;  // tokens [first, last) belong to requests
  int32_t window;       // keys a query sees at most (INT32_MAX: all)
  int32_t valid;        // 0: the batch's offsets or lengths were refused
  int32_t reserved[2];
};

}  // namespace smetric

struct smetric_kv {
  smetric_kv_config cfg;
  int device;
  int num_sms;
  int group;        // query heads per key head
  int32_t* status;  // device: first latched error
  smetric::KvPlan* plan;
  smetric::KvToken* tokens;  // max_batch_tokens
  // of the last plan
  bool planned;
  int32_t n_requests;
  int64_t n_tokens;
  const int64_t* offsets;
  const int32_t* kv_lens;
  const int32_t* pages;
  int64_t pages_stride;
  int32_t max_pages;
  int64_t launches;
};

namespace smetric {
// Returns SMETRIC_OK if the handle is usable from the current device.
int check_device(const smetric_kv* kv);
// A row of heads that a kernel can address: 16-byte aligned, strides of whole
// 16-byte pieces.
inline bool heads_ok(const smetric_heads& h, int64_t n_tokens) {
  return n_tokens == 0 || (h.d_data && !(reinterpret_cast<uintptr_t>(h.d_data) & 15) && h.token_stride >= 0 &&
                           h.head_stride >= 0 && h.token_stride % 8 == 0 && h.head_stride % 8 == 0);
}
inline bool cache_ok(const smetric_kv_cache& c) {
  return c.d_k && c.d_v && !((reinterpret_cast<uintptr_t>(c.d_k) | reinterpret_cast<uintptr_t>(c.d_v)) & 15) &&
         c.page_stride >= 0 && c.token_stride >= 0 && c.head_stride >= 0 && c.page_stride % 8 == 0 &&
         c.token_stride % 8 == 0 && c.head_stride % 8 == 0;
}
}  // namespace smetric
