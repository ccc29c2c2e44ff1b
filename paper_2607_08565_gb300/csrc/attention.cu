// Attention of a planned batch's queries over the paged cache.
//
//   k_paged_attention  a warp for each (token, query head): the keys one after
//                      another, the running maximum and sum of the softmax and
//                      the output in registers, lane l holding elements
//                      l, l + 32, ... of the head.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <cmath>

#include "call_range.cuh"
#include "kv_impl.cuh"
#include "launch.cuh"
#include "smetric_impl.cuh"

using namespace smetric;

namespace {

struct AttentionArgs {
  smetric_kv_cache cache;
  smetric_heads q, out;
  float* lse;
  const KvPlan* plan;
  const KvToken* tokens;
  const int32_t* pages;
  int64_t pages_stride, num_pages, n_tokens;
  int32_t hq, group, D, page_size;
  float scale;
  int32_t* status;
};

__device__ __forceinline__ float to_f(__nv_bfloat16 x) { return __bfloat162float(x); }
__device__ __forceinline__ float to_f(__half x) { return __half2float(x); }
__device__ __forceinline__ void from_f(float x, __nv_bfloat16& y) { y = __float2bfloat16_rn(x); }
__device__ __forceinline__ void from_f(float x, __half& y) { y = __float2half_rn(x); }

template <typename T>
__global__ void __launch_bounds__(256) k_paged_attention(const __grid_constant__ AttentionArgs a) {
  pdl_enter();
  constexpr int E = SMETRIC_KV_MAX_HEAD_DIM / 32;
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int64_t t = w / a.hq;
  const int h = (int)(w - t * a.hq);
  if (t >= a.n_tokens) return;
  const KvToken tok = a.tokens[t];
  float o[E] = {}, q[E], m = -INFINITY, l = 0.f;
  if (a.plan->valid && tok.req >= 0) {
    const T* qp = static_cast<const T*>(a.q.d_data) + t * a.q.token_stride + h * a.q.head_stride;
#pragma unroll
    for (int i = 0; i < E; ++i) q[i] = lane + 32 * i < a.D ? to_f(qp[lane + 32 * i]) * a.scale : 0.f;
    const int64_t head = (int64_t)(h / a.group) * a.cache.head_stride;
    const int32_t from = tok.pos >= a.plan->window ? tok.pos - a.plan->window + 1 : 0;
    for (int32_t j = from; j <= tok.pos; ++j) {
      const int32_t page = a.pages[tok.req * a.pages_stride + j / a.page_size];
      const bool held = page >= 0 && page < a.num_pages;
      if (!held && lane == 0) latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
      const int64_t at = (int64_t)page * a.cache.page_stride + (j % a.page_size) * a.cache.token_stride + head;
      const T* kp = static_cast<const T*>(a.cache.d_k) + at;
      const T* vp = static_cast<const T*>(a.cache.d_v) + at;
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < E; ++i)
        if (held && lane + 32 * i < a.D) x = fmaf(q[i], to_f(kp[lane + 32 * i]), x);
      for (int s = 16; s; s >>= 1) x += __shfl_xor_sync(0xffffffffu, x, s);
      const float top = fmaxf(m, x);
      const float back = expf(m - top), p = expf(x - top);
      l = l * back + p;
      m = top;
#pragma unroll
      for (int i = 0; i < E; ++i)
        o[i] = o[i] * back + (held && lane + 32 * i < a.D ? p * to_f(vp[lane + 32 * i]) : 0.f);
    }
  }
  T* op = static_cast<T*>(a.out.d_data) + t * a.out.token_stride + h * a.out.head_stride;
#pragma unroll
  for (int i = 0; i < E; ++i)
    if (lane + 32 * i < a.D) from_f(l == 0.f ? 0.f : o[i] / l, op[lane + 32 * i]);
  if (a.lse && lane == 0) a.lse[t * a.hq + h] = l == 0.f ? -INFINITY : m + logf(l);
}

}  // namespace

extern "C" {

int smetric_paged_attention(smetric_kv* kv, smetric_kv_cache cache, smetric_heads q, float scale, smetric_heads out,
                            float* d_lse, smetric_stream_t stream) {
  CallRange range("smetric_paged_attention");
  int rc = check_device(kv);
  if (rc) return rc;
  if (!kv->planned || !std::isfinite(scale) || !(scale > 0.f) || !cache_ok(cache) || !heads_ok(q, kv->n_tokens) ||
      !heads_ok(out, kv->n_tokens) || (reinterpret_cast<uintptr_t>(d_lse) & 3))
    return SMETRIC_ERR_INVALID_ARG;
  if (kv->n_tokens == 0) return SMETRIC_OK;
  AttentionArgs a = {};
  a.cache = cache;
  a.q = q;
  a.out = out;
  a.lse = d_lse;
  a.plan = kv->plan;
  a.tokens = kv->tokens;
  a.pages = kv->pages;
  a.pages_stride = kv->pages_stride;
  a.num_pages = kv->cfg.num_pages;
  a.n_tokens = kv->n_tokens;
  a.hq = kv->cfg.num_q_heads;
  a.group = kv->group;
  a.D = kv->cfg.head_dim;
  a.page_size = kv->cfg.page_size;
  a.scale = scale;
  a.status = kv->status;
  kv->launches++;
  auto kern = kv->cfg.dtype == SMETRIC_BF16 ? k_paged_attention<__nv_bfloat16> : k_paged_attention<__half>;
  const int64_t grid = (kv->n_tokens * a.hq + 7) / 8;
  if (grid > INT32_MAX) return SMETRIC_ERR_INVALID_ARG;
  return launch_k(kern, dim3((unsigned)grid), dim3(256), 0, reinterpret_cast<cudaStream_t>(stream), true, a);
}

}  // extern "C"
