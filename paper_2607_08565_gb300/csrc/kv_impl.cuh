// Handle of the paged KV$ operators, shared by kv.cu and attention.cu.
#pragma once

#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cfloat>
#include <cmath>

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
  int32_t n_split_few;  // the same of the units of few rows
  int32_t reserved;
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

// Caches in 4 bits: requests whose new tokens have at most `rows` query rows for
// a key head are the share of a kernel of their own (kv4.cu), in units of their
// tokens and one of `blocks` blocks of `heads` key heads each, and in tiles of
// kFewTile keys.
constexpr int kFewTile = 32;
// Its warps, and so the key heads of a block at most.
constexpr int kFewWarps = 12;
struct KvFew {
  int rows;    // 8, 16, or 0: no such kernel (more than 16 query heads per key head)
  int tokens;  // rows / group
  int heads, blocks;
  KvUnit* units;       // 2 * max_batch_requests
  int64_t* unit_cost;  // as many + 1
  int32_t* unit_base;  // max_batch_requests + 1
  KvShare* shares;     // num_sms
  int32_t* split;      // num_sms
  float* part;         // 2 * num_sms slots of heads * rows * head_dim partial sums
  float2* part_ml;     // and their rows' (reference exponent, sum of weights)
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
  smetric::KvFew few;
  // of the last plan
  bool planned;
  bool all_few;   // every unit is the few-row kernel's
  bool one_join;  // its join is the chunks' kernel's too
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
bool attention_limits(bool four);
bool few_limits();
// Attention over caches in 4 bits of the plan's requests of more rows than few.rows; with
// one_join its shared units are left to the few-row kernel's join.
int attention_many_rows(smetric_kv* kv, const smetric_kvq_cache& k_cache, const smetric_kvq_cache& v_cache,
                        const smetric_heads& q, float scale, const smetric_heads& out, float* d_lse,
                        smetric_stream_t stream);
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
// What scores are multiplied by, of a row that was divided by a power of two: a normal
// number, as 0 times the -inf of a key that is not seen is NaN, and infinity times the
// score 0 is. (A row of zeros has the power 2^-126. Scores are below 2^35 before, so that
// those below 2^-91 after it may be any so small.)
__device__ __forceinline__ float score_factor(float c) { return fminf(fmaxf(c, FLT_MIN), FLT_MAX); }
// A reference exponent, score * factor - lift rounded up, so that no weight passes
// 2^(lift + slack): weights are of exactly this reference, and the largest one's is
// 2^lift / 2^ulp(reference) or more. That is a number above 0 of the weights' type while
// the reference is below 2^28 (half precision, a lift of 7) or 2^30 (bf16, none).
__device__ __forceinline__ float reference(float score, float factor, float lift) { return __fmaf_ru(score, factor, -lift); }
__device__ __forceinline__ bool too_far(float reference, float lift) {
  return fabsf(reference) >= (lift > 0.f ? 0x1p28f : 0x1p30f) && fabsf(reference) < INFINITY;
}
// Bytes of a head's scales: head_dim / 16, to a whole load.
__host__ __device__ constexpr int scale_bytes(int head_dim) { return head_dim <= 64 ? 4 : 8; }
inline bool cache4_ok(const smetric_kvq_cache& c, int head_dim) {
  const int s = scale_bytes(head_dim);
  return c.d_codes && c.d_scales && !(reinterpret_cast<uintptr_t>(c.d_codes) & 15) &&
         reinterpret_cast<uintptr_t>(c.d_scales) % s == 0 && c.page_stride >= 0 && c.token_stride >= 0 &&
         c.head_stride >= 0 && c.scale_page_stride >= 0 && c.scale_token_stride >= 0 && c.scale_head_stride >= 0 &&
         c.page_stride % 16 == 0 && c.token_stride % 16 == 0 && c.head_stride % 16 == 0 &&
         c.scale_page_stride % s == 0 && c.scale_token_stride % s == 0 && c.scale_head_stride % s == 0 &&
         std::max({c.page_stride, c.token_stride, c.scale_page_stride, c.scale_token_stride}) <= UINT32_MAX &&
         c.exp >= -SMETRIC_KVQ_MAX_EXP && c.exp <= SMETRIC_KVQ_MAX_EXP && !c.reserved;
}
// At a whole number of its elements, as loads need.
template <typename E>
bool aligned(const E* p) {
  return reinterpret_cast<uintptr_t>(p) % sizeof(E) == 0;
}
// A scale of scores that the kernels can multiply by, as exponents of 2.
inline bool scale_ok(float scale) { return scale > 0.f && std::isfinite(scale * 1.4426950408889634f); }
inline bool four_bits(const smetric_kv* kv) { return kv->cfg.flags & SMETRIC_KV_4BIT; }
}  // namespace smetric
