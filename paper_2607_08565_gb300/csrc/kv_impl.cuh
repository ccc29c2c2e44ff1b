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
  int32_t reserved;
};

// The plan's device-side summary.
struct KvPlan {
  int64_t first, last;  // tokens [first, last) belong to requests
  int32_t valid;        // 0: the batch's offsets or lengths were refused
  int32_t n_split;      // units that several CTAs share
  int32_t reserved[2];
};

// Keys go through the attention in tiles of kTile, queries in tiles of kTile
// rows (a row is a token and one of the query heads that share a key head).
constexpr int kTile = 128;

// Up to two query tiles of one request's consecutive tokens, for one key head
// at a time: the attention's unit of work.
struct __align__(16) KvUnit {
  int32_t token;   // its first token's row in q
  int32_t tokens;
  int32_t pos;     // its first token's position
  int32_t req;
  int32_t tb, te;  // key tiles that it sees
  int32_t reserved[2];
};

// A CTA's share: the key tiles of (unit u0, key head h0) from t0, the units
// and heads that follow, and (u1, h1) up to t1, exclusive. A unit that several
// CTAs share has pieces: the first is the end of a CTA's share, the others the
// starts of the next CTAs'.
struct __align__(16) KvShare {
  int32_t u0, h0, t0;  // u0 < 0: nothing
  int32_t u1, h1, t1;
  int32_t n_last;      // pieces of the last unit, where the share starts it
  int32_t reserved;
  KvUnit first, last;  // units u0 and u1
};

}  // namespace smetric

struct smetric_kv {
  smetric_kv_config cfg;
  int device;
  int num_sms;
  int group;        // query heads per key head
  int tile_tokens;  // tokens of a query tile: kTile / group
  int32_t* status;  // device: first latched error
  smetric::KvPlan* plan;
  smetric::KvToken* tokens;  // max_batch_tokens
  smetric::KvUnit* units;    // max_batch_tokens / (2 * tile_tokens) + max_batch_requests
  int64_t* unit_cost;        // as many + 1: cost of the units before, for one key head
  int32_t* unit_base;        // max_batch_requests + 1: a request's first unit
  smetric::KvShare* shares;  // num_sms
  int32_t* split;            // num_sms: the CTAs that start a unit which others go on with
  float* part;               // 2 * num_sms slots of partial sums: a CTA's first unit's, its last's
  float2* part_ml;           // and their rows' (reference exponent, sum of weights)
  // of the last plan
  bool planned;
  int64_t n_tokens;
  const int32_t* pages;
  int64_t pages_stride;
  int32_t window;  // keys a query sees at most (INT32_MAX: all)
  int64_t launches;
};

namespace smetric {
// Returns SMETRIC_OK if the handle is usable from the current device.
int check_device(const smetric_kv* kv);
// Sets the attention kernels' shared-memory limits; false on a CUDA error.
bool attention_limits();
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
