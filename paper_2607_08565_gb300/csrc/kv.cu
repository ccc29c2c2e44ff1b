// The paged KV$ operators around the attention: the handle, the plan of a
// batch, and the norm + rotation + append pass.
//
//   k_kv_plan      block 0 checks the batch and shares its attention out;
//                  the other blocks find each new token's request by bisection
//                  of the offsets, its position and its slot in the cache.
//                  Bound by latency: 5 to 8 us from one request to 86,000
//                  tokens, once for all layers of a step.
//   k_kv_heads     one pass over the new tokens' heads: queries and keys are
//                  normed and rotated in registers, keys and values go to
//                  their slots (or, for the transform alone, to rows). Bound by
//                  memory: 35,862 tokens of 32 + 2 x 4 heads of 128 (753 MB) 127
//                  us, 87 % of a copy; 16,001 of 64 + 4 (565 MB) 95 us; 86,444 of
//                  2 x 8 of 64 (366 MB) 70 us, 77 %, as a warp has 2 KB to copy
//                  and two dependent reads to make first. Few tokens: 2 us.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <new>
#include <type_traits>

#include "call_range.cuh"
#include "kv_impl.cuh"
#include "launch.cuh"
#include "smetric_impl.cuh"

using namespace smetric;

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr int kPlanThreads = 1024;
constexpr int kMaxCtas = 1024;  // attention CTAs that a plan shares work out to

// A unit's cost, in 1,000 cycles as measured with heads of 128 elements (shorter
// ones, whose tiles cost less, have the same proportions by assumption): for each
// key tile, where it has two query tiles or one, and for what it does once (its
// queries' load, the first scores, its output). A CTA takes at least kMinCost, and a unit is cut
// at least kMinTiles from its ends.
__device__ __forceinline__ int tile_cost(const KvUnit& u, int tile_tokens) { return u.tokens > tile_tokens ? 3 : 2; }
__device__ __forceinline__ int once_cost(const KvUnit& u, int tile_tokens) { return u.tokens > tile_tokens ? 6 : 4; }
constexpr int kMinCost = 8;
constexpr int kMinTiles = 2;

struct PlanArgs {
  const int64_t* off;
  int32_t n;
  int64_t n_tokens;
  const int32_t* kv_lens;
  const int32_t* pages;
  int32_t max_pages, page_size;
  int64_t pages_stride, num_pages;
  int32_t window, tile_tokens, kv_heads, ctas;
  KvPlan* plan;
  KvToken* tokens;
  KvUnit* units;
  int64_t* unit_cost;
  int32_t* unit_base;
  KvShare* shares;
  int32_t* split;
  int32_t* status;
};

// Exclusive prefix sum over the block; total receives the sum.
template <typename S>
__device__ S block_scan(S x, S* warp_sums, S& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  S y = x;
  for (int o = 1; o < 32; o <<= 1) {
    const S z = __shfl_up_sync(kFull, y, o);
    if (lane >= o) y += z;
  }
  if (lane == 31) warp_sums[warp] = y;
  __syncthreads();
  if (warp == 0) {
    S v = warp_sums[lane];
    for (int o = 1; o < 32; o <<= 1) {
      const S z = __shfl_up_sync(kFull, v, o);
      if (lane >= o) v += z;
    }
    warp_sums[lane] = v;
  }
  __syncthreads();
  total = warp_sums[31];
  const S before = warp ? warp_sums[warp - 1] : 0;
  __syncthreads();
  return before + y - x;
}

// Largest i in [0, n) with a[i] * scale <= x (a non-decreasing, a[0] = 0, x >= 0).
template <typename S>
__device__ int32_t last_at_most(const S* a, int32_t n, int64_t x, int64_t scale) {
  int32_t lo = 0, hi = n;
  while (hi - lo > 1) {
    const int32_t mid = lo + ((hi - lo) >> 1);
    if ((int64_t)a[mid] * scale <= x)
      lo = mid;
    else
      hi = mid;
  }
  return lo;
}

// Shares the batch's attention out: the key tiles of all (unit, key head)
// pairs in a row, cut into one stretch of equal cost for each CTA, so that one
// long sequence and many short ones load the SMs alike.
__device__ void plan_units(const PlanArgs& a) {
  __shared__ int64_t sums[32];
  __shared__ int32_t su[kMaxCtas + 1], sh[kMaxCtas + 1], st[kMaxCtas + 1];
  __shared__ int32_t n_split;
  const int per = 2 * a.tile_tokens;
  int64_t base = 0;
  for (int32_t r0 = 0; r0 < a.n; r0 += kPlanThreads) {
    const int32_t r = r0 + threadIdx.x;
    const int64_t mine = r < a.n ? (a.off[r + 1] - a.off[r] + per - 1) / per : 0;
    int64_t total;
    const int64_t at = block_scan(mine, sums, total);
    if (r < a.n) a.unit_base[r] = (int32_t)(base + at);
    base += total;
  }
  const int32_t U = (int32_t)base;
  __syncthreads();
  int64_t cost = 0;
  for (int32_t u0 = 0; u0 < U; u0 += kPlanThreads) {
    const int32_t u = u0 + threadIdx.x;
    int64_t mine = 0;
    if (u < U) {
      const int32_t r = last_at_most(a.unit_base, a.n, u, 1);
      const int64_t first = (int64_t)(u - a.unit_base[r]) * per, lq = a.off[r + 1] - a.off[r];
      KvUnit x = {};
      x.token = (int32_t)(a.off[r] + first);
      x.tokens = (int32_t)min((int64_t)per, lq - first);
      x.pos = (int32_t)(a.kv_lens[r] - lq + first);
      x.req = r;
      x.tb = x.pos >= a.window ? (x.pos - a.window + 1) / kTile : 0;
      x.te = (x.pos + x.tokens - 1) / kTile + 1;
      a.units[u] = x;
      mine = (x.te - x.tb) * tile_cost(x, a.tile_tokens) + once_cost(x, a.tile_tokens);
    }
    int64_t total;
    const int64_t at = block_scan(mine, sums, total);
    if (u < U) a.unit_cost[u] = cost + at;
    cost += total;
  }
  __syncthreads();
  cost *= a.kv_heads;
  const int ctas = (int)max((int64_t)1, min((int64_t)a.ctas, cost / kMinCost));
  for (int c = threadIdx.x; c <= ctas; c += kPlanThreads) {
    int32_t u = U, h = 0, t = 0;
    if (c < ctas && U > 0) {
      const int64_t x = cost / ctas * c + cost % ctas * c / ctas;
      u = last_at_most(a.unit_cost, U, x, a.kv_heads);
      const KvUnit unit = a.units[u];
      const int per_tile = tile_cost(unit, a.tile_tokens), once = once_cost(unit, a.tile_tokens);
      const int64_t one = (int64_t)(unit.te - unit.tb) * per_tile + once, in = x - a.unit_cost[u] * a.kv_heads;
      h = (int32_t)(in / one);
      t = unit.tb + (int32_t)(max((int64_t)0, in % one - once) / per_tile);
      if (t - unit.tb < kMinTiles) {
        t = unit.tb;
      } else if (unit.te - t < kMinTiles) {
        if (++h == a.kv_heads) h = 0, ++u;
        t = u < U ? a.units[u].tb : 0;
      }
    }
    su[c] = u, sh[c] = h, st[c] = t;
  }
  if (threadIdx.x == 0) n_split = 0;
  __syncthreads();
  for (int c = threadIdx.x; c < a.ctas; c += kPlanThreads) {
    KvShare s = {};
    s.u0 = -1;
    if (c < ctas && (su[c] != su[c + 1] || sh[c] != sh[c + 1] || st[c] != st[c + 1])) {
      s.u0 = su[c], s.h0 = sh[c], s.t0 = st[c];
      s.first = a.units[s.u0];
      s.u1 = su[c + 1], s.h1 = sh[c + 1], s.t1 = st[c + 1];
      const bool cut = s.u1 < U && s.t1 > a.units[s.u1].tb;
      if (!cut) {
        if (--s.h1 < 0) s.h1 = a.kv_heads - 1, --s.u1;
        s.t1 = a.units[s.u1].te;
      }
      const auto same = [&](int i, int32_t u, int32_t h) {
        return i <= ctas && su[i] == u && sh[i] == h && u < U && st[i] > a.units[u].tb;
      };
      s.last = a.units[s.u1];
      s.n_last = 1;
      while (same(c + s.n_last, s.u1, s.h1)) ++s.n_last;
      // (their order decides which blocks join them, not how)
      if (s.n_last > 1 && !same(c, s.u1, s.h1)) a.split[atomicAdd(&n_split, 1)] = c;
    }
    a.shares[c] = s;
  }
  __syncthreads();
  if (threadIdx.x == 0) a.plan->n_split = n_split;
}

__global__ void __launch_bounds__(kPlanThreads) k_kv_plan(const __grid_constant__ PlanArgs a) {
  pdl_enter();
  if (blockIdx.x == 0) {
    int bad = 0;
    for (int32_t r = threadIdx.x; r < a.n; r += blockDim.x) {
      const int64_t lo = a.off[r], hi = a.off[r + 1], kv = a.kv_lens[r];
      bad |= lo < 0 || hi < lo || hi > a.n_tokens || kv < hi - lo || kv > (int64_t)a.max_pages * a.page_size;
    }
    bad = __syncthreads_or(bad);
    if (threadIdx.x == 0) {
      if (bad) latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
      a.plan->first = bad || a.n == 0 ? a.n_tokens : a.off[0];
      a.plan->last = bad || a.n == 0 ? a.n_tokens : a.off[a.n];
      a.plan->valid = !bad;
    }
    if (!bad) {
      plan_units(a);
    } else {
      for (int i = threadIdx.x; i < a.ctas; i += kPlanThreads) a.shares[i].u0 = -1;
      if (threadIdx.x == 0) a.plan->n_split = 0;
    }
    return;
  }
  const int64_t t = (int64_t)(blockIdx.x - 1) * blockDim.x + threadIdx.x;
  if (t >= a.n_tokens) return;
  KvToken tok = {-1, -1, 0};
  if (a.n > 0) {
    // the last request that starts at or before t (bad offsets may mislead the
    // bisection, not past the array: the request's own bounds decide)
    const int32_t r = last_at_most(a.off, a.n, t, 1);
    const int64_t lo = a.off[r], hi = a.off[r + 1], kv = a.kv_lens[r];
    if (lo >= 0 && lo <= t && t < hi && kv >= hi - lo && kv <= (int64_t)a.max_pages * a.page_size) {
      tok.pos = (int32_t)(kv - (hi - t));
      const int32_t page = a.pages[r * a.pages_stride + tok.pos / a.page_size];
      if (page >= 0 && page < a.num_pages)
        tok.slot = (int64_t)page * a.page_size + tok.pos % a.page_size;
      else
        latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
    }
  }
  a.tokens[t] = tok;
}

template <typename T>
struct Pair;
template <>
struct Pair<__nv_bfloat16> {
  static __device__ __forceinline__ float2 get(uint32_t x) {
    return make_float2(__uint_as_float(x << 16), __uint_as_float(x & 0xffff0000u));
  }
  static __device__ __forceinline__ uint32_t put(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
};
template <>
struct Pair<__half> {
  static __device__ __forceinline__ float2 get(uint32_t x) { return __half22float2(*reinterpret_cast<__half2*>(&x)); }
  static __device__ __forceinline__ uint32_t put(float a, float b) {
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
};

template <typename T>
__device__ __forceinline__ void unpack(uint4 x, float* f) {
  const uint32_t w[4] = {x.x, x.y, x.z, x.w};
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const float2 p = Pair<T>::get(w[i]);
    f[2 * i] = p.x;
    f[2 * i + 1] = p.y;
  }
}
template <typename T>
__device__ __forceinline__ uint4 pack(const float* f) {
  return make_uint4(Pair<T>::put(f[0], f[1]), Pair<T>::put(f[2], f[3]), Pair<T>::put(f[4], f[5]),
                    Pair<T>::put(f[6], f[7]));
}

struct HeadsArgs {
  smetric_heads q, k, v, q_out, k_out;  // absent: 0 heads
  int32_t hq, hk, hv;
  smetric_kv_cache cache;    // keys and values go here when tokens is not NULL
  const KvToken* tokens;     // the plan's, or NULL: d_positions and k_out
  const KvPlan* plan;
  const int32_t* positions;
  int64_t n_tokens;
  int32_t D, page_shift, rot, lanes_shift, splits;
  uint32_t rows;  // positions below it are taken: the table's rows, all that are not negative without one
  const float* table;
  const void* q_norm;
  const void* k_norm;
  float eps;
  int32_t* status;
};

// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
  float2 r;
  asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
      " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y), "f"(z.x), "f"(z.y));
  return r;
}
__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
  float2 r;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mul.rn.f32x2 d, a, b;\n"
      " mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
  return r;
}

// A lane's part of the transform: 16 elements in two pieces of 8.
struct Lane {
  bool held, turned;  // it has elements of a head; they are rotated
  int e0, e1;         // the pieces' first elements
  int lanes_shift, D;
  float eps;
  float2 cs[4], sn[4];  // of its 8 pairs
};

// A lane's two pieces of head h of a token (src is at that head).
template <typename T>
__device__ __forceinline__ void load_head(const Lane& l, const T* src, int h, int heads, uint4 (&x)[2]) {
  if (l.held && h < heads) {
    x[0] = *reinterpret_cast<const uint4*>(src + l.e0);
    x[1] = *reinterpret_cast<const uint4*>(src + l.e1);
  }
}

// heads h, h + step, ... < heads of a token, from src to dst (both at head h);
// x: the first of them. (A round's heads are loaded while the round before is
// computed.)
template <typename T, bool kInterleaved>
__device__ __forceinline__ void transform_heads(const Lane& l, const T* src, int64_t src_step, T* dst, int64_t dst_step,
                                                int h, int step, int heads, int rounds, const T* norm, uint4 (&x)[2]) {
  for (int r = 0; r < rounds; ++r, h += step, dst += dst_step) {
    const bool on = l.held && h < heads;
    const uint4 y[2] = {x[0], x[1]};
    src += src_step;
    load_head(l, src, h + step, heads, x);
    if (!norm && !l.turned) {  // (nothing changes: its bits are kept, a NaN's among them)
      if (on) {
        *reinterpret_cast<uint4*>(dst + l.e0) = y[0];
        *reinterpret_cast<uint4*>(dst + l.e1) = y[1];
      }
      continue;
    }
    float2 f[8];
#pragma unroll
    for (int e = 0; e < 2; ++e) unpack<T>(y[e], &f[4 * e].x);
    if (norm) {  // (the same for the warp: its lanes take part in the sum)
      float2 s2 = make_float2(0.f, 0.f);
#pragma unroll
      for (int k = 0; k < 8; ++k) s2 = fma2(f[k], f[k], s2);
      float ss = on ? s2.x + s2.y : 0.f;
      for (int o = 1; o < 1 << l.lanes_shift; o <<= 1) ss += __shfl_xor_sync(kFull, ss, o);
      if (on) {
        const float inv = 1.0f / sqrtf(ss / (float)l.D + l.eps);
#pragma unroll
        for (int e = 0; e < 2; ++e) {
          float2 g[4];
          unpack<T>(*reinterpret_cast<const uint4*>(norm + (e ? l.e1 : l.e0)), &g[0].x);
#pragma unroll
          for (int k = 0; k < 4; ++k) f[4 * e + k] = mul2(mul2(f[4 * e + k], make_float2(inv, inv)), g[k]);
        }
      }
    }
    if (l.turned) {
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        if (kInterleaved) {  // pairs 2k and 2k + 1, as (a, b) each
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const float c = i ? l.cs[k].y : l.cs[k].x, s = i ? l.sn[k].y : l.sn[k].x;
            const float2 u = f[2 * k + i];
            f[2 * k + i] = make_float2(u.x * c - u.y * s, u.y * c + u.x * s);
          }
        } else {
          const float2 u = f[k], v = f[4 + k];
          f[k] = fma2(u, l.cs[k], mul2(v, make_float2(-l.sn[k].x, -l.sn[k].y)));
          f[4 + k] = fma2(v, l.cs[k], mul2(u, l.sn[k]));
        }
      }
    }
    if (on) {
      *reinterpret_cast<uint4*>(dst + l.e0) = pack<T>(&f[0].x);
      *reinterpret_cast<uint4*>(dst + l.e1) = pack<T>(&f[4].x);
    }
  }
}

// A warp takes a token (or one of `splits` shares of its heads) and a group of
// 2^lanes_shift lanes a head at a time, 16 elements a lane in two 16-byte
// pieces: the two halves of 8 rotation pairs (i, i + rot/2), 8 interleaved
// pairs, or 16 elements past rot. So a rotation never leaves the lane, a norm
// is a sum over the group's lanes, and the token's cosines and sines are
// loaded once for all its heads. Bound by memory; the registers of 28 warps an
// SM hold the bytes in flight: 72 a thread, with 44 to 60 bytes spilled (24 warps
// of 80 took 101 us for 16,001 tokens of 64 + 4 heads, where these take 96).
template <typename T, bool kInterleaved>
__global__ void __launch_bounds__(128, 7) k_kv_heads(const __grid_constant__ HeadsArgs a) {
  pdl_enter();
  const int lane = threadIdx.x & 31;
  const int64_t w = (int64_t)blockIdx.x * (blockDim.x >> 5) + (threadIdx.x >> 5);
  const int64_t t = w / a.splits;
  const int share = (int)(w - t * a.splits);
  if (t >= a.n_tokens) return;
  Lane l;
  const int c = lane & ((1 << a.lanes_shift) - 1);
  l.held = 16 * c < a.D;  // (groups of 8 lanes hold heads of 96 elements)
  l.turned = l.held && a.table && 16 * c < a.rot;
  l.e0 = l.turned && !kInterleaved ? 8 * c : 16 * c;
  l.e1 = l.turned && !kInterleaved ? 8 * c + a.rot / 2 : 16 * c + 8;
  l.lanes_shift = a.lanes_shift;
  l.D = a.D;
  l.eps = a.eps;
  const int per = 32 >> a.lanes_shift;  // heads a warp takes at a time
  const int step = per * a.splits, first = lane >> a.lanes_shift;
  // rounds of heads: the keys', then the values', then the queries'; the share
  // has every splits-th, from rounds k0, v0, q0 of each
  const int rk = (a.hk + per - 1) / per, rv = (a.hv + per - 1) / per, rq = (a.hq + per - 1) / per;
  const auto start = [&](int before) { return (share - before % a.splits + a.splits) % a.splits; };
  const int k0 = share, v0 = start(rk), q0 = start(rk + rv);
  const auto source = [&](const smetric_heads& src, int r) {
    return static_cast<const T*>(src.d_data) + t * src.token_stride + (r * per + first) * src.head_stride;
  };
  // (the first loads run while the token's place is found)
  uint4 x[2] = {make_uint4(0, 0, 0, 0), make_uint4(0, 0, 0, 0)}, y[2] = {x[0], x[1]};
  if (v0 < rv) load_head(l, source(a.v, v0), v0 * per + first, a.hv, y);
  if (k0 < rk) load_head(l, source(a.k, k0), k0 * per + first, a.hk, x);
  int64_t slot = 0;
  int32_t pos;
  if (a.tokens) {
    const KvToken tok = a.tokens[t];
    if (!a.plan->valid || tok.slot < 0) return;
    slot = tok.slot;
    pos = tok.pos;
  } else {
    pos = a.positions[t];
  }
  if ((uint32_t)pos >= a.rows) {
    if (lane == 0 && share == 0) latch_error(a.status, SMETRIC_ERR_OVERFLOW);
    return;
  }
  const bool turned = l.turned;
  if (turned) {
    const float4* row = reinterpret_cast<const float4*>(a.table + (int64_t)pos * a.rot + 8 * c);
    const float4* row2 = reinterpret_cast<const float4*>(a.table + (int64_t)pos * a.rot + a.rot / 2 + 8 * c);
#pragma unroll
    for (int i = 0; i < 2; ++i) {
      const float4 u = row[i], v = row2[i];
      l.cs[2 * i] = make_float2(u.x, u.y), l.cs[2 * i + 1] = make_float2(u.z, u.w);
      l.sn[2 * i] = make_float2(v.x, v.y), l.sn[2 * i + 1] = make_float2(v.z, v.w);
    }
  }
  const auto heads = [&](const smetric_heads& src, T* dst, int64_t head_stride, int r, int rounds, int n_heads,
                         const void* norm, uint4(&z)[2]) {
    if (r < rounds)
      transform_heads<T, kInterleaved>(l, source(src, r), step * src.head_stride,
                                       dst + (r * per + first) * head_stride, step * head_stride, r * per + first, step,
                                       n_heads, (rounds - r + a.splits - 1) / a.splits, static_cast<const T*>(norm), z);
  };
  const int64_t at = (slot >> a.page_shift) * a.cache.page_stride +
                     (slot & ((1 << a.page_shift) - 1)) * a.cache.token_stride;
  l.turned = false;
  heads(a.v, static_cast<T*>(a.cache.d_v) + at, a.cache.head_stride, v0, rv, a.hv, nullptr, y);
  l.turned = turned;
  if (q0 < rq) load_head(l, source(a.q, q0), q0 * per + first, a.hq, y);
  if (a.tokens)
    heads(a.k, static_cast<T*>(a.cache.d_k) + at, a.cache.head_stride, k0, rk, a.hk, a.k_norm, x);
  else
    heads(a.k, static_cast<T*>(a.k_out.d_data) + t * a.k_out.token_stride, a.k_out.head_stride, k0, rk, a.hk, a.k_norm, x);
  heads(a.q, static_cast<T*>(a.q_out.d_data) + t * a.q_out.token_stride, a.q_out.head_stride, q0, rq, a.hq, a.q_norm, y);
}

// At a whole number of its elements, as loads need.
template <typename E>
bool aligned(const E* p) {
  return reinterpret_cast<uintptr_t>(p) % sizeof(E) == 0;
}

bool transform_ok(const smetric_kv* kv, const smetric_kv_transform& t) {
  if (t.reserved || (t.flags & ~SMETRIC_KV_INTERLEAVED) || t.rot_dim < 0 || t.rot_dim > kv->cfg.head_dim ||
      t.rot_dim % 16 || t.table_rows < 0)
    return false;
  if (t.d_cos_sin && (t.rot_dim == 0 || (reinterpret_cast<uintptr_t>(t.d_cos_sin) & 15))) return false;
  if ((reinterpret_cast<uintptr_t>(t.d_q_norm) | reinterpret_cast<uintptr_t>(t.d_k_norm)) & 15) return false;
  return (!t.d_q_norm && !t.d_k_norm) || (std::isfinite(t.eps) && t.eps >= 0.f);
}

int launch_heads(smetric_kv* kv, HeadsArgs& a, const smetric_kv_transform& t, cudaStream_t s) {
  a.D = kv->cfg.head_dim;
  a.page_shift = __builtin_ctz((unsigned)kv->cfg.page_size);
  a.rot = t.rot_dim;
  a.table = t.rot_dim ? t.d_cos_sin : nullptr;
  a.rows = (uint32_t)(a.table ? std::min<int64_t>(t.table_rows, 1ll << 31) : 1ll << 31);
  a.q_norm = a.hq ? t.d_q_norm : nullptr;
  a.k_norm = a.hk ? t.d_k_norm : nullptr;
  a.eps = t.eps;
  a.status = kv->status;
  a.lanes_shift = 0;
  while (16 << a.lanes_shift < a.D) a.lanes_shift++;
  // Warps that share a token's heads: as many as it has rounds of heads while
  // there are too few tokens to fill the SMs (28 warps an SM), else one.
  const int rounds = (a.hq + a.hk + a.hv + (32 >> a.lanes_shift) - 1) / (32 >> a.lanes_shift);
  const int64_t room = (int64_t)kv->num_sms * 28 / std::max<int64_t>(1, a.n_tokens);
  a.splits = (int32_t)std::max<int64_t>(1, std::min<int64_t>(rounds, room));
  const int64_t grid = (a.n_tokens * a.splits + 3) / 4;
  const bool il = t.flags & SMETRIC_KV_INTERLEAVED;
  const bool bf = kv->cfg.dtype == SMETRIC_BF16;
  auto kern = bf ? (il ? k_kv_heads<__nv_bfloat16, true> : k_kv_heads<__nv_bfloat16, false>)
                 : (il ? k_kv_heads<__half, true> : k_kv_heads<__half, false>);
  kv->launches++;
  return launch_k(kern, dim3((unsigned)grid), dim3(128), 0, s, true, a);
}

// Device memory of a handle: one allocation (each costs the host some 30 us),
// its parts 256-byte aligned. Sets the parts' pointers within `mem` (NULL: only
// counts) and returns its size.
size_t lay_out(smetric_kv* kv, unsigned char* mem) {
  const size_t tokens = (size_t)kv->cfg.max_batch_tokens, requests = (size_t)kv->cfg.max_batch_requests;
  const size_t units = tokens / (2 * kv->tile_tokens) + requests + 1;
  const size_t slots = 2 * (size_t)kv->num_sms * 2 * kTile;
  size_t at = 0;
  const auto part = [&](auto*& p, size_t n) {
    p = reinterpret_cast<std::remove_reference_t<decltype(p)>>(mem ? mem + at : nullptr);
    at += (n * sizeof(*p) + 255) / 256 * 256;
  };
  part(kv->status, 1);
  part(kv->plan, 1);
  part(kv->tokens, tokens + 1);
  part(kv->units, units);
  part(kv->unit_cost, units + 1);
  part(kv->unit_base, requests + 1);
  part(kv->shares, kv->num_sms);
  part(kv->split, kv->num_sms);
  part(kv->part, slots * kv->cfg.head_dim);
  part(kv->part_ml, slots);
  return at;
}

}  // namespace

int smetric::check_device(const smetric_kv* kv) {
  if (!kv) return SMETRIC_ERR_INVALID_ARG;
  int dev = -1;
  if (cudaGetDevice(&dev) != cudaSuccess) return cuda_status(cudaErrorUnknown);
  return dev == kv->device ? SMETRIC_OK : SMETRIC_ERR_INVALID_ARG;
}

extern "C" {

int smetric_kv_create(const smetric_kv_config* cfg, smetric_kv** out) {
  CallRange range("smetric_kv_create");
  if (!cfg || !out) return SMETRIC_ERR_INVALID_ARG;
  *out = nullptr;
  const smetric_kv_config& c = *cfg;
  if (c.head_dim < 16 || c.head_dim > SMETRIC_KV_MAX_HEAD_DIM || c.head_dim % 16 || c.num_kv_heads < 1 ||
      c.num_kv_heads > 4096 || c.num_q_heads < c.num_kv_heads || c.num_q_heads % c.num_kv_heads ||
      c.num_q_heads / c.num_kv_heads > SMETRIC_KV_MAX_GROUP || c.page_size < 16 || c.page_size > 256 ||
      (c.page_size & (c.page_size - 1)) || (c.dtype != SMETRIC_BF16 && c.dtype != SMETRIC_F16) || c.flags ||
      c.num_pages < 1 || c.num_pages > INT32_MAX || c.max_batch_requests < 0 ||
      c.max_batch_requests > SMETRIC_KV_MAX_REQUESTS || c.max_batch_tokens < 0 ||
      c.max_batch_tokens > SMETRIC_KV_MAX_TOKENS)
    return SMETRIC_ERR_INVALID_ARG;
  smetric_kv* kv = new (std::nothrow) smetric_kv{};
  if (!kv) return SMETRIC_ERR_OOM;
  kv->cfg = c;
  kv->group = c.num_q_heads / c.num_kv_heads;
  kv->tile_tokens = kTile / kv->group;
  unsigned char* mem = nullptr;
  bool ok = cudaGetDevice(&kv->device) == cudaSuccess &&
            cudaDeviceGetAttribute(&kv->num_sms, cudaDevAttrMultiProcessorCount, kv->device) == cudaSuccess;
  if (ok) {
    kv->num_sms = std::min(kv->num_sms, kMaxCtas);
    ok = cudaMalloc(&mem, lay_out(kv, nullptr)) == cudaSuccess;
  }
  if (ok) {
    lay_out(kv, mem);
    ok = attention_limits() && cudaMemset(kv->status, 0, sizeof(int32_t)) == cudaSuccess &&
         cudaDeviceSynchronize() == cudaSuccess;
  }
  if (!ok) {
    (void)cudaGetLastError();
    cudaFree(mem);
    delete kv;
    return SMETRIC_ERR_OOM;
  }
  *out = kv;
  return SMETRIC_OK;
}

int smetric_kv_destroy(smetric_kv* kv) {
  CallRange range("smetric_kv_destroy");
  if (!kv) return SMETRIC_OK;
  int dev = -1;
  cudaGetDevice(&dev);
  if (dev != kv->device) cudaSetDevice(kv->device);
  cudaDeviceSynchronize();
  cudaFree(kv->status);  // (the first part: the whole)
  int rc = cuda_status(cudaGetLastError());
  if (dev >= 0 && dev != kv->device) cudaSetDevice(dev);
  delete kv;
  return rc;
}

int smetric_kv_plan(smetric_kv* kv, const int64_t* d_offsets, int32_t n_requests, int64_t n_tokens,
                    const int32_t* d_kv_lens, const int32_t* d_pages, int32_t max_pages, int64_t pages_stride,
                    int32_t window, smetric_stream_t stream) {
  CallRange range("smetric_kv_plan");
  int rc = check_device(kv);
  if (rc) return rc;
  if (n_requests < 0 || n_requests > kv->cfg.max_batch_requests || n_tokens < 0 ||
      n_tokens > kv->cfg.max_batch_tokens || max_pages < 0 || pages_stride < max_pages || window < 0 ||
      (n_requests > 0 && (!d_offsets || !d_kv_lens || (max_pages > 0 && !d_pages))) || !aligned(d_offsets) ||
      !aligned(d_kv_lens) || !aligned(d_pages))
    return SMETRIC_ERR_INVALID_ARG;
  kv->planned = false;
  PlanArgs a = {};
  a.off = d_offsets;
  a.n = n_requests;
  a.n_tokens = n_tokens;
  a.kv_lens = d_kv_lens;
  a.pages = d_pages;
  a.max_pages = max_pages;
  a.page_size = kv->cfg.page_size;
  a.pages_stride = pages_stride;
  a.num_pages = kv->cfg.num_pages;
  a.window = window > 0 ? window : INT32_MAX;
  a.tile_tokens = kv->tile_tokens;
  a.kv_heads = kv->cfg.num_kv_heads;
  a.ctas = kv->num_sms;
  a.plan = kv->plan;
  a.tokens = kv->tokens;
  a.units = kv->units;
  a.unit_cost = kv->unit_cost;
  a.unit_base = kv->unit_base;
  a.shares = kv->shares;
  a.split = kv->split;
  a.status = kv->status;
  const unsigned grid = 1 + (unsigned)((n_tokens + kPlanThreads - 1) / kPlanThreads);
  kv->launches++;
  rc = launch_k(k_kv_plan, dim3(grid), dim3(kPlanThreads), 0, reinterpret_cast<cudaStream_t>(stream), true, a);
  if (rc) return rc;
  kv->planned = true;
  kv->n_tokens = n_tokens;
  kv->pages = d_pages;
  kv->pages_stride = pages_stride;
  kv->window = a.window;
  return SMETRIC_OK;
}

int smetric_kv_append(smetric_kv* kv, smetric_kv_cache cache, smetric_heads k, smetric_heads v, smetric_heads q,
                      smetric_heads q_out, smetric_kv_transform t, smetric_stream_t stream) {
  CallRange range("smetric_kv_append");
  int rc = check_device(kv);
  if (rc) return rc;
  if (!kv->planned || !transform_ok(kv, t) || !heads_ok(k, kv->n_tokens) || !heads_ok(v, kv->n_tokens) ||
      (q.d_data && (!heads_ok(q, kv->n_tokens) || !heads_ok(q_out, kv->n_tokens))) || !cache_ok(cache))
    return SMETRIC_ERR_INVALID_ARG;
  if (kv->n_tokens == 0) return SMETRIC_OK;
  HeadsArgs a = {};
  a.k = k;
  a.v = v;
  a.q = q;
  a.q_out = q_out;
  a.hk = a.hv = kv->cfg.num_kv_heads;
  a.hq = q.d_data ? kv->cfg.num_q_heads : 0;
  a.cache = cache;
  a.tokens = kv->tokens;
  a.plan = kv->plan;
  a.n_tokens = kv->n_tokens;
  return launch_heads(kv, a, t, reinterpret_cast<cudaStream_t>(stream));
}

int smetric_qk_norm_rope(smetric_kv* kv, smetric_heads q, smetric_heads k, const int32_t* d_positions,
                         int64_t n_tokens, smetric_kv_transform t, smetric_heads q_out, smetric_heads k_out,
                         smetric_stream_t stream) {
  CallRange range("smetric_qk_norm_rope");
  int rc = check_device(kv);
  if (rc) return rc;
  if (n_tokens < 0 || n_tokens > SMETRIC_KV_MAX_TOKENS || !transform_ok(kv, t) ||
      (q.d_data && (!heads_ok(q, n_tokens) || !heads_ok(q_out, n_tokens))) ||
      (k.d_data && (!heads_ok(k, n_tokens) || !heads_ok(k_out, n_tokens))) || (n_tokens > 0 && !d_positions) ||
      !aligned(d_positions))
    return SMETRIC_ERR_INVALID_ARG;
  if (n_tokens == 0 || (!q.d_data && !k.d_data)) return SMETRIC_OK;
  HeadsArgs a = {};
  a.k = k;
  a.q = q;
  a.k_out = k_out;
  a.q_out = q_out;
  a.hk = k.d_data ? kv->cfg.num_kv_heads : 0;
  a.hq = q.d_data ? kv->cfg.num_q_heads : 0;
  a.positions = d_positions;
  a.n_tokens = n_tokens;
  return launch_heads(kv, a, t, reinterpret_cast<cudaStream_t>(stream));
}

int smetric_kv_status(smetric_kv* kv, smetric_stream_t stream) {
  CallRange range("smetric_kv_status");
  int rc = check_device(kv);
  if (rc) return rc;
  if (cudaStreamSynchronize(reinterpret_cast<cudaStream_t>(stream)) != cudaSuccess)
    return cuda_status(cudaErrorUnknown);
  int32_t h = 0;
  if (cudaMemcpy(&h, kv->status, sizeof(h), cudaMemcpyDeviceToHost) != cudaSuccess)
    return cuda_status(cudaErrorUnknown);
  if (h != 0 && cudaMemset(kv->status, 0, sizeof(int32_t)) != cudaSuccess) return cuda_status(cudaErrorUnknown);
  return h;
}

int64_t smetric_kv_launch_count(const smetric_kv* kv) { return kv ? kv->launches : 0; }

}  // extern "C"
