// The paged KV$ operators over caches in 4 bits: reading back, and attention.
//
//   k_kv4_read       rows of positions in 16 bits.
//   k_kv4_attention  a warp for each query row.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>

#include "call_range.cuh"
#include "kv_impl.cuh"
#include "launch.cuh"
#include "smetric_impl.cuh"

using namespace smetric;

namespace {

constexpr unsigned kFull = 0xffffffffu;

// ---- codes and scales ----

// The two elements of byte B of a word of codes.
template <int B>
__device__ __forceinline__ uint32_t pair_of(uint32_t codes) {
  uint32_t r;
  if constexpr (B == 0)
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %1;\n cvt.rn.f16x2.e2m1x2 %0, a;\n}\n" : "=r"(r) : "r"(codes));
  else if constexpr (B == 1)
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %1;\n cvt.rn.f16x2.e2m1x2 %0, b;\n}\n" : "=r"(r) : "r"(codes));
  else if constexpr (B == 2)
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %1;\n cvt.rn.f16x2.e2m1x2 %0, c;\n}\n" : "=r"(r) : "r"(codes));
  else
    asm("{\n .reg .b8 a, b, c, d;\n mov.b32 {a, b, c, d}, %1;\n cvt.rn.f16x2.e2m1x2 %0, d;\n}\n" : "=r"(r) : "r"(codes));
  return r;
}
// Two scales (in the low 16 bits).
__device__ __forceinline__ uint32_t scales_of(uint32_t bits) {
  uint32_t r;
  asm("{\n .reg .b16 a, b;\n mov.b32 {a, b}, %1;\n cvt.rn.f16x2.e4m3x2 %0, a;\n}\n" : "=r"(r) : "r"(bits));
  return r;
}
__device__ __forceinline__ float2 floats(uint32_t h2) { return __half22float2(*reinterpret_cast<const __half2*>(&h2)); }

template <typename T>
__device__ __forceinline__ uint32_t round2(float2 x);
template <>
__device__ __forceinline__ uint32_t round2<__nv_bfloat16>(float2 x) {
  const __nv_bfloat162 p = __floats2bfloat162_rn(x.x, x.y);
  return *reinterpret_cast<const uint32_t*>(&p);
}
template <>
__device__ __forceinline__ uint32_t round2<__half>(float2 x) {
  const __half2 p = __floats2half2_rn(x.x, x.y);
  return *reinterpret_cast<const uint32_t*>(&p);
}

// ---- reading back ----

struct ReadArgs {
  smetric_kvq_cache c[2];
  smetric_heads out[2];  // absent: d_data NULL
  const int64_t* off;
  const int32_t* first;
  const int32_t* pages;
  int64_t pages_stride, n_rows, num_pages;
  int32_t n, max_pages, page_shift, D, hk, rows;  // rows of a block
  int32_t* status;
};

constexpr int kReadThreads = 128;

// A block takes `rows` rows: a thread each finds their slots, then all copy, 16
// elements (a group, whole sectors of the output) a thread at a time.
template <typename T>
__global__ void __launch_bounds__(kReadThreads) k_kv4_read(const __grid_constant__ ReadArgs a) {
  __shared__ int64_t slots[kReadThreads];  // -1: left as it is, -2: zeros
  pdl_enter();
  const int64_t row0 = (int64_t)blockIdx.x * a.rows;
  const int rows = (int)min((int64_t)a.rows, a.n_rows - row0);
  if ((int)threadIdx.x < rows) {
    const int64_t i = row0 + threadIdx.x;
    // the last request that starts at or before i (bad offsets may mislead the
    // bisection, not past the array: the request's own bounds decide)
    int32_t lo = 0, hi = a.n;
    while (hi - lo > 1) {
      const int32_t mid = lo + ((hi - lo) >> 1);
      if (a.off[mid] <= i)
        lo = mid;
      else
        hi = mid;
    }
    const int64_t begin = a.off[lo], end = a.off[lo + 1];
    int64_t slot = -1;
    if (begin < 0 || end < begin || end > a.n_rows) {
      latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
    } else if (begin <= i && i < end) {
      const int64_t pos = (a.first ? a.first[lo] : 0) + (i - begin), at = pos >> a.page_shift;
      const int32_t page = pos >= 0 && at < a.max_pages ? a.pages[lo * a.pages_stride + at] : -1;
      slot = page >= 0 && page < a.num_pages ? ((int64_t)page << a.page_shift) + (pos & ((1 << a.page_shift) - 1)) : -2;
      if (slot < 0) latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
    }
    slots[threadIdx.x] = slot;
  }
  __syncthreads();
  const int groups = a.D / 16, per = a.hk * groups;  // of a row, for keys or values
  for (int x = threadIdx.x; x < rows * 2 * per; x += kReadThreads) {
    const int row = x / (2 * per), y = x - row * 2 * per, which = y >= per;
    const int z = y - which * per, h = z / groups, g = z - h * groups;
    const int64_t slot = slots[row];
    const smetric_heads& out = a.out[which];
    if (slot == -1 || !out.d_data) continue;
    uint2 w = make_uint2(0, 0);
    uint32_t scale = 0;
    const smetric_kvq_cache& c = a.c[which];
    if (slot >= 0) {
      const int64_t page = slot >> a.page_shift, in = slot & ((1 << a.page_shift) - 1);
      w = *reinterpret_cast<const uint2*>(static_cast<const uint8_t*>(c.d_codes) + page * c.page_stride +
                                          in * c.token_stride + h * c.head_stride + 8 * g);
      scale = static_cast<const uint8_t*>(c.d_scales)[page * c.scale_page_stride + in * c.scale_token_stride +
                                                      h * c.scale_head_stride + g];
    }
    const float s = floats(scales_of(scale)).x * exp2f((float)c.exp);
    uint32_t r[8];
    const auto four = [&](uint32_t codes, uint32_t* to) {
      const uint32_t p[4] = {pair_of<0>(codes), pair_of<1>(codes), pair_of<2>(codes), pair_of<3>(codes)};
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const float2 f = floats(p[k]);
        to[k] = round2<T>(make_float2(f.x * s, f.y * s));
      }
    };
    four(w.x, r), four(w.y, r + 4);
    uint4* to = reinterpret_cast<uint4*>(static_cast<T*>(out.d_data) + (row0 + row) * out.token_stride + h * out.head_stride + 16 * g);
    to[0] = make_uint4(r[0], r[1], r[2], r[3]);
    to[1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
}

// ---- attention ----

struct Attention4Args {
  smetric_kvq_cache k, v;
  smetric_heads q, out;
  float* lse;
  const KvPlan* plan;
  const KvUnit* units;
  const int32_t* pages;
  int64_t pages_stride, n_tokens;
  int32_t num_pages, hq, kv_heads, group, D, page_shift, window;
  float scale;
  int32_t* status;
};

template <typename T>
__device__ __forceinline__ float to_float(T x);
template <>
__device__ __forceinline__ float to_float(__nv_bfloat16 x) { return __bfloat162float(x); }
template <>
__device__ __forceinline__ float to_float(__half x) { return __half2float(x); }

template <typename T>
__global__ void __launch_bounds__(128) k_kv4_attention(const __grid_constant__ Attention4Args a) {
  pdl_enter();
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int E = a.D / 32;  // elements a lane
  const float ks = exp2f((float)a.k.exp), vs = exp2f((float)a.v.exp);
  for (int64_t x = blockIdx.x; x < (int64_t)a.plan->n_units * a.kv_heads; x += gridDim.x) {
    const KvUnit u = a.units[x / a.kv_heads];
    const int h = (int)(x % a.kv_heads);
    const int32_t* pages = a.pages + u.req * a.pages_stride;
    for (int row = warp; row < u.tokens * a.group; row += 4) {
      const int64_t token = u.token + row / a.group;
      const int head = h * a.group + row % a.group;
      const int32_t pos = u.pos + row / a.group;
      float q[4] = {}, o[4] = {};
      for (int e = 0; e < E; ++e)
        q[e] = to_float(static_cast<const T*>(a.q.d_data)[token * a.q.token_stride + head * a.q.head_stride + lane * E + e]);
      float top = -INFINITY, l = 0.f;
      for (int32_t j = pos >= a.window ? pos - a.window + 1 : 0; j <= pos; ++j) {
        const int32_t page = pages[j >> a.page_shift];
        const bool held = page >= 0 && page < a.num_pages;
        if (!held) latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
        const int64_t in = j & ((1 << a.page_shift) - 1);
        const auto element = [&](const smetric_kvq_cache& c, int d) {
          if (!held) return 0.f;
          const uint8_t b = static_cast<const uint8_t*>(c.d_codes)[page * c.page_stride + in * c.token_stride + h * c.head_stride + d / 2];
          const uint8_t s = static_cast<const uint8_t*>(c.d_scales)[page * c.scale_page_stride + in * c.scale_token_stride +
                                                                    h * c.scale_head_stride + d / 16];
          const float2 f = floats(pair_of<0>(b));
          return (d & 1 ? f.y : f.x) * floats(scales_of(s)).x;
        };
        float s = 0.f;
        for (int e = 0; e < E; ++e) s += q[e] * element(a.k, lane * E + e);
        for (int i = 16; i; i >>= 1) s += __shfl_xor_sync(kFull, s, i);
        s *= a.scale * ks;
        const float next = fmaxf(top, s);
        const float f = expf(top - next), p = expf(s - next);
        top = next;
        l = l * f + p;
        for (int e = 0; e < E; ++e) o[e] = o[e] * f + p * element(a.v, lane * E + e);
      }
      for (int e = 0; e < E; ++e) {
        const uint32_t y = round2<T>(make_float2(o[e] / l * vs, 0.f));
        reinterpret_cast<uint16_t*>(a.out.d_data)[token * a.out.token_stride + head * a.out.head_stride + lane * E + e] = (uint16_t)y;
      }
      if (a.lse && lane == 0) a.lse[token * a.hq + head] = top + logf(l);
    }
  }
  // tokens of no request
  const int64_t first = a.plan->first, last = a.plan->last, none = first + a.n_tokens - last;
  for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < none * a.hq * a.D; i += (int64_t)gridDim.x * blockDim.x) {
    const int64_t x = i / a.D, h = x % a.hq;
    int64_t t = x / a.hq;
    if (t >= first) t += last - first;
    reinterpret_cast<uint16_t*>(a.out.d_data)[t * a.out.token_stride + h * a.out.head_stride + i % a.D] = 0;
    if (a.lse) a.lse[t * a.hq + h] = -INFINITY;
  }
}

}  // namespace

extern "C" {

int smetric_kvq_read(smetric_kv* kv, smetric_kvq_cache k_cache, smetric_kvq_cache v_cache, const int64_t* d_offsets,
                     int32_t n_requests, int64_t n_rows, const int32_t* d_first, const int32_t* d_pages,
                     int32_t max_pages, int64_t pages_stride, smetric_heads k, smetric_heads v,
                     smetric_stream_t stream) {
  CallRange range("smetric_kvq_read");
  int rc = check_device(kv);
  if (rc) return rc;
  const smetric_kv_config& c = kv->cfg;
  if (!four_bits(kv) || n_requests < 0 || n_requests > SMETRIC_KV_MAX_REQUESTS || n_rows < 0 || n_rows > SMETRIC_KVQ_MAX_ROWS ||
      max_pages < 0 || pages_stride < max_pages ||
      (n_requests > 0 && (!d_offsets || (max_pages > 0 && !d_pages))) || !aligned(d_offsets) || !aligned(d_first) ||
      !aligned(d_pages) || (k.d_data && (!heads_ok(k, n_rows) || !cache4_ok(k_cache, c.head_dim))) ||
      (v.d_data && (!heads_ok(v, n_rows) || !cache4_ok(v_cache, c.head_dim))))
    return SMETRIC_ERR_INVALID_ARG;
  if (n_rows == 0 || n_requests == 0 || (!k.d_data && !v.d_data)) return SMETRIC_OK;
  ReadArgs a = {};
  a.c[0] = k_cache, a.c[1] = v_cache;
  a.out[0] = k, a.out[1] = v;
  a.off = d_offsets;
  a.first = d_first;
  a.pages = d_pages;
  a.pages_stride = pages_stride;
  a.n_rows = n_rows;
  a.num_pages = c.num_pages;
  a.n = n_requests;
  a.max_pages = max_pages;
  a.page_shift = __builtin_ctz((unsigned)c.page_size);
  a.D = c.head_dim;
  a.hk = c.num_kv_heads;
  a.rows = 8;
  a.status = kv->status;
  const int64_t grid = (n_rows + a.rows - 1) / a.rows;
  kv->launches++;
  return launch_k(c.dtype == SMETRIC_BF16 ? k_kv4_read<__nv_bfloat16> : k_kv4_read<__half>, dim3((unsigned)grid),
                  dim3(kReadThreads), 0, reinterpret_cast<cudaStream_t>(stream), true, a);
}

int smetric_kvq_attention(smetric_kv* kv, smetric_kvq_cache k_cache, smetric_kvq_cache v_cache, smetric_heads q,
                          float scale, smetric_heads out, float* d_lse, smetric_stream_t stream) {
  CallRange range("smetric_kvq_attention");
  int rc = check_device(kv);
  if (rc) return rc;
  const smetric_kv_config& c = kv->cfg;
  if (!four_bits(kv) || !kv->planned || !cache4_ok(k_cache, c.head_dim) || !cache4_ok(v_cache, c.head_dim) ||
      !std::isfinite(std::ldexp(scale, k_cache.exp)) || !(std::ldexp(scale, k_cache.exp) > 0.f) ||
      !heads_ok(q, kv->n_tokens) || !heads_ok(out, kv->n_tokens) || (reinterpret_cast<uintptr_t>(d_lse) & 3))
    return SMETRIC_ERR_INVALID_ARG;
  if (kv->n_tokens == 0) return SMETRIC_OK;
  Attention4Args a = {};
  a.k = k_cache;
  a.v = v_cache;
  a.q = q;
  a.out = out;
  a.lse = d_lse;
  a.plan = kv->plan;
  a.units = kv->units;
  a.pages = kv->pages;
  a.pages_stride = kv->pages_stride;
  a.n_tokens = kv->n_tokens;
  a.num_pages = (int32_t)c.num_pages;
  a.hq = c.num_q_heads;
  a.kv_heads = c.num_kv_heads;
  a.group = kv->group;
  a.D = c.head_dim;
  a.page_shift = __builtin_ctz((unsigned)c.page_size);
  a.window = kv->window;
  a.scale = scale;
  a.status = kv->status;
  kv->launches++;
  return launch_k(c.dtype == SMETRIC_BF16 ? k_kv4_attention<__nv_bfloat16> : k_kv4_attention<__half>,
                  dim3((unsigned)kv->num_sms * 8), dim3(128), 0, reinterpret_cast<cudaStream_t>(stream), true, a);
}

}  // extern "C"
