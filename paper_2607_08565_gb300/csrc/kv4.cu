// The paged KV$ operators over caches in 4 bits: reading back, and the attention of
// requests with few query rows (single tokens; others are attention.cu's). Appending
// is kv.cu's.
//
//   k_kv4_read      rows of positions in 16 bits.
//   k_kv4_few       one CTA an SM, each with the share of the batch that the plan gave
//                   it.
//   k_kv4_join      joins the pieces of the units that several CTAs share (and those of
//                   the chunks' kernel, where it probably has none).
//
// An element is code * scale * 2^exp: 4 bits (e2m1) and, for 16 of them, 8 (e4m3). Code
// times scale has 6 bits and lies within 2^-10 .. 2,688: exact in half precision, in
// which the products are. The exponents go into the scores' factor and the output's.

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include <algorithm>
#include <cmath>
#include <type_traits>

#include "attention_join.cuh"
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

// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 mul2(float2 x, float2 y) {
  float2 r;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mul.rn.f32x2 d, a, b;\n"
      " mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
  return r;
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
  bool wide[2];  // outputs can be stored in pieces of 32 bytes
  int32_t* status;
};

constexpr int kReadThreads = 128;
constexpr int kReadRows = 32;  // of a block, at most: a warp's lanes

// A block takes some rows: a thread each finds where they are, then all copy, 16
// elements (a group, whole sectors of the output) a thread at a time; a thread has the
// same group of the same head for every row that it takes, four rows on their way.
// Bound by memory (the output is 3.6 times the input): 148,000 rows of 2 x 4 heads of 128,
// 474 MB, take 77 us, 92 % of a copy. With a row and a column found by divisions for every
// 16 elements 87 us, at 268 instructions for each; blocks of 16 and 64 rows 79 and 80 us.
template <typename T>
__global__ void __launch_bounds__(kReadThreads) k_kv4_read(const __grid_constant__ ReadArgs a) {
  __shared__ int64_t codes_at[kReadRows][2], scales_at[kReadRows][2];  // -1: left as it is, -2: zeros
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
    int32_t page = -1, in = -1;
    if (begin < 0 || end < begin || end > a.n_rows) {
      latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
    } else if (begin <= i && i < end) {
      const int64_t pos = (a.first ? a.first[lo] : 0) + (i - begin), at = pos >> a.page_shift;
      page = pos >= 0 && at < a.max_pages ? a.pages[lo * a.pages_stride + at] : -1;
      in = page >= 0 && page < a.num_pages ? (int32_t)(pos & ((1 << a.page_shift) - 1)) : -2;
      if (in < 0) latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
    }
#pragma unroll
    for (int w = 0; w < 2; ++w) {
      codes_at[threadIdx.x][w] = in < 0 ? in : page * a.c[w].page_stride + in * a.c[w].token_stride;
      scales_at[threadIdx.x][w] = page * a.c[w].scale_page_stride + in * a.c[w].scale_token_stride;
    }
  } else if (threadIdx.x >= 32) {  // meanwhile: offsets that no row leads to
    constexpr int kRest = kReadThreads - 32;
    for (int64_t r = (int64_t)blockIdx.x * kRest + threadIdx.x - 32; r < a.n; r += (int64_t)gridDim.x * kRest) {
      const int64_t begin = a.off[r], end = a.off[r + 1];
      if (begin < 0 || end < begin || end > a.n_rows) latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
    }
  }
  __syncthreads();
  // columns: a group of a head's keys or values each; `width` of them at a time
  const int groups = a.D / 16, per = a.hk * groups, width = min(2 * per, kReadThreads);
  const int stride = kReadThreads / width, first = threadIdx.x / width;
  if (first >= stride) return;
  for (int column = threadIdx.x - first * width; column < 2 * per; column += width) {
    const int which = column >= per, z = column - which * per, h = z / groups, g = z - h * groups;
    const smetric_heads& out = a.out[which];
    if (!out.d_data) continue;
    const smetric_kvq_cache& c = a.c[which];
    const uint8_t* const codes = static_cast<const uint8_t*>(c.d_codes) + h * c.head_stride + 8 * g;
    const uint8_t* const scales = static_cast<const uint8_t*>(c.d_scales) + h * c.scale_head_stride + g;
    T* to = static_cast<T*>(out.d_data) + (row0 + first) * out.token_stride + h * out.head_stride + 16 * g;
    const float unit = exp2f((float)c.exp);
    constexpr int P = 4;  // rows on their way
    for (int row0 = first; row0 < rows; row0 += P * stride) {
      int64_t at[P];
      uint2 w[P];
      uint32_t scale[P];
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const int row = row0 + k * stride;
        at[k] = row < rows ? codes_at[row][which] : -1;
        w[k] = make_uint2(0, 0);
        scale[k] = 0;
        if (at[k] >= 0) {
          w[k] = *reinterpret_cast<const uint2*>(codes + at[k]);
          scale[k] = scales[scales_at[row][which]];
        }
      }
#pragma unroll
      for (int k = 0; k < P; ++k, to += stride * out.token_stride) {
        if (at[k] == -1) continue;
        const float s = floats(scales_of(scale[k])).x * unit;
        uint32_t r[8];
        const auto four = [&](uint32_t x, uint32_t* y) {
          const uint32_t p[4] = {pair_of<0>(x), pair_of<1>(x), pair_of<2>(x), pair_of<3>(x)};
#pragma unroll
          for (int i = 0; i < 4; ++i) y[i] = round2<T>(mul2(floats(p[i]), make_float2(s, s)));
        };
        four(w[k].x, r), four(w[k].y, r + 4);
        // (a whole sector in one store: two halves took 97 us for 148,000 rows of 2 x 4 heads
        // of 128, as every sector went to the L2 cache twice)
        if (a.wide[which]) {
          asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"l"(to), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                       "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
        } else {
          uint4* q = reinterpret_cast<uint4*>(to);
          q[0] = make_uint4(r[0], r[1], r[2], r[3]);
          q[1] = make_uint4(r[4], r[5], r[6], r[7]);
        }
      }
    }
  }
}

// ---- attention of few rows ----

// The pieces of the chunks' kernel, for the join.
struct ManyJoin {
  smetric_heads out;
  float* lse;
  const KvShare* shares;
  const int32_t* split;
  float* part;
  float2* part_ml;
  int32_t hq, group, tile_tokens, D;
  float v_scale;
  bool wide;  // outputs can be stored in pieces of 32 bytes
};

struct FewArgs {
  ManyJoin many;
  smetric_kvq_cache k, v;
  smetric_heads q, out;
  float* lse;
  const KvPlan* plan;
  const KvUnit* units;
  const KvShare* shares;
  const int32_t* split;
  float* part;
  float2* part_ml;
  const int32_t* pages;
  int64_t pages_stride, n_tokens;
  int32_t num_pages, hq, hk, group, heads, blocks, page_shift, window;
  float scale;  // of scores in powers of 2
  float v_scale;
  bool bf16;
  int32_t* status;
};

// (as the attention of 16-bit caches has them in half precision)
constexpr float kLift = 7.f;   // weights up to 2^(kLift + kSlack): half precision ends at 65,504
constexpr float kSlack = 8.f;  // log2 of how far scores may pass the reference

__host__ __device__ constexpr int stage_bytes(int D) { return 2 * kFewTile * (D / 2 + scale_bytes(D)); }
__host__ __device__ constexpr int stages(int D) {
  return 225 * 1024 / (kFewWarps * stage_bytes(D)) < 8 ? 225 * 1024 / (kFewWarps * stage_bytes(D)) : 8;
}
__host__ __device__ constexpr int ring_bytes(int D) { return kFewWarps * stages(D) * stage_bytes(D); }
// A row of a warp's sums in shared memory, in floats: 4 past a multiple of 32, so that
// the rows of the lanes that store together lie in other banks.
__host__ __device__ constexpr int sum_row(int D) { return D + 4; }
__host__ __device__ constexpr int few_smem(int D, int rows) {
  const int sums = kFewWarps * rows * (sum_row(D) + 2) * 4;
  return ring_bytes(D) > sums ? ring_bytes(D) : sums;
}
static_assert(few_smem(128, 8) <= 232448 && few_smem(128, 16) <= 232448 && few_smem(32, 8) <= 232448, "227 KB");

struct FewItem {
  KvUnit unit;
  int32_t hb, tb, te;  // block of key heads, its key tiles in this CTA
  bool whole;          // nobody else has key tiles of it
  int32_t slot;        // of its partial sums, where !whole
};

// The CTA's share, item by item.
struct FewWalk {
  KvUnit unit;
  int32_t u, h, t0, u1, h1, t1;
  bool first, done;
  __device__ __forceinline__ void start(const FewArgs& a) {
    const KvShare& s = a.shares[blockIdx.x];
    unit = s.first;
    u = s.u0, h = s.h0, t0 = s.t0, u1 = s.u1, h1 = s.h1, t1 = s.t1;
    first = true;
    done = u < 0;
  }
  __device__ __forceinline__ bool next(const FewArgs& a, FewItem& it) {
    if (done) return false;
    const bool last = u == u1 && h == h1;
    it.unit = unit;
    it.hb = h;
    it.tb = first ? t0 : unit.tb;
    it.te = last ? t1 : unit.te;
    it.whole = it.tb == unit.tb && it.te == unit.te;
    it.slot = 2 * (int32_t)blockIdx.x + (it.tb == unit.tb);
    first = false;
    done = last;
    if (++h == a.blocks && !done) {
      h = 0;
      unit = a.units[++u];
    }
    return true;
  }
};

__device__ __forceinline__ uint32_t mul_h2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("mul.rn.f16x2 %0, %1, %2;\n" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
// D (16 x 8, 32 bits) += A (16 x 16) B (16 x 8).
__device__ __forceinline__ void mma(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%0, %1, %2, %3};\n"
               : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1));
}
// D = A B.
__device__ __forceinline__ void mma_first(float (&d)[4], const uint32_t (&a)[4], uint32_t b0, uint32_t b1) {
  asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0, %1, %2, %3}, {%4, %5, %6, %7}, {%8, %9}, {%10, %10, %10, %10};\n"
               : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3])
               : "r"(a[0]), "r"(a[1]), "r"(a[2]), "r"(a[3]), "r"(b0), "r"(b1), "f"(0.f));
}
// The low four bits of each byte of x, the high four of y.
__device__ __forceinline__ uint32_t low_nibbles(uint32_t x, uint32_t y) {
  uint32_t r;
  asm("lop3.b32 %0, %1, %2, 0x0f0f0f0f, 0xe4;\n" : "=r"(r) : "r"(x), "r"(y));
  return r;
}
// Two 32-bit operations in one instruction.
__device__ __forceinline__ float2 fma2(float2 x, float2 y, float2 z) {
  float2 r;
  asm("{\n .reg .b64 a, b, c, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n mov.b64 c, {%6, %7};\n"
      " fma.rn.f32x2 d, a, b, c;\n mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y), "f"(z.x), "f"(z.y));
  return r;
}
__device__ __forceinline__ float2 add2(float2 x, float2 y) {
  float2 r;
  asm("{\n .reg .b64 a, b, d;\n mov.b64 a, {%2, %3};\n mov.b64 b, {%4, %5};\n add.rn.f32x2 d, a, b;\n"
      " mov.b64 {%0, %1}, d;\n}\n"
      : "=f"(r.x), "=f"(r.y) : "f"(x.x), "f"(x.y), "f"(y.x), "f"(y.y));
  return r;
}
__device__ __forceinline__ uint32_t transposed(uint32_t x) {
  uint32_t r;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;\n" : "=r"(r) : "r"(x));
  return r;
}
// N bytes; zeros where !held.
template <int N, bool kWhole>
__device__ __forceinline__ void copy_async(uint32_t dst, const void* src, bool held) {
  if constexpr (kWhole && N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16;\n" ::"r"(dst), "l"(src) : "memory");
  else if constexpr (kWhole)
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2;\n" ::"r"(dst), "l"(src), "n"(N) : "memory");
  else if constexpr (N == 16)
    asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;\n" ::"r"(dst), "l"(src), "r"(held ? 16 : 0) : "memory");
  else
    asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;\n" ::"r"(dst), "l"(src), "n"(N), "r"(held ? N : 0) : "memory");
}

// Query rows n0 .. n0 + 7 of a key head as the products' B operand, and their powers of
// 2. Lane (g, c) = (lane / 4, lane % 4) has row g's elements [c D/4, (c+1) D/4). A row in
// bf16 goes to half precision divided by the power of two of its largest element: its 8
// bits fit where an element is 2^-17 of the largest or more, and smaller ones are rounded
// to multiples of 2^-24 of it. (Where the largest meets codes of 0 they can count.)
template <int D>
__device__ __forceinline__ void load_rows(const FewArgs& a, const KvUnit& u, int head, int n0, uint4 (&x)[D / 32]) {
  const int lane = threadIdx.x & 31, n = n0 + (lane >> 2);
#pragma unroll
  for (int i = 0; i < D / 32; ++i) x[i] = make_uint4(0, 0, 0, 0);
  if (n >= u.tokens * a.group) return;
  const int64_t at = (int64_t)(u.token + n / a.group) * a.q.token_stride + (int64_t)(head * a.group + n % a.group) * a.q.head_stride;
  const uint4* p = reinterpret_cast<const uint4*>(static_cast<const uint16_t*>(a.q.d_data) + at + (lane & 3) * (D / 4));
#pragma unroll
  for (int i = 0; i < D / 32; ++i) x[i] = p[i];
}
template <int D>
__device__ __forceinline__ void convert_rows(const uint4 (&x)[D / 32], bool bf16, uint32_t (&qf)[D / 16][2], float& power) {
  float f[D / 4];
#pragma unroll
  for (int i = 0; i < D / 32; ++i) {
    const uint32_t w[4] = {x[i].x, x[i].y, x[i].z, x[i].w};
#pragma unroll
    for (int k = 0; k < 4; ++k) {
      const float2 y = bf16 ? make_float2(__uint_as_float(w[k] << 16), __uint_as_float(w[k] & 0xffff0000u)) : floats(w[k]);
      f[8 * i + 2 * k] = y.x, f[8 * i + 2 * k + 1] = y.y;
    }
  }
  float top = 0.f;
#pragma unroll
  for (int i = 0; i < D / 4; ++i) top = fmaxf(top, fabsf(f[i]));
  top = fmaxf(top, __shfl_xor_sync(kFull, top, 1));
  top = fmaxf(top, __shfl_xor_sync(kFull, top, 2));
  // 2^(E - 127) <= top, its reciprocal a number; infinities keep their row as it is, and half precision is it
  uint32_t E = __float_as_uint(top) >> 23;
  E = !bf16 || E == 255 ? 127 : min(max(E, 1u), 253u);
  const float down = __uint_as_float((254 - E) << 23);
  power = __uint_as_float(E << 23);
#pragma unroll
  for (int i = 0; i < D / 16; ++i)
#pragma unroll
    for (int k = 0; k < 2; ++k) qf[i][k] = round2<__half>(make_float2(f[4 * i + 2 * k] * down, f[4 * i + 2 * k + 1] * down));
}

// Elements 4 lane .. 4 lane + 3 of a row.
template <int D>
__device__ __forceinline__ void write_row(const FewArgs& a, const KvUnit& u, int head, int row, float4 f, float top, float l) {
  const int lane = threadIdx.x & 31;
  const int64_t token = u.token + row / a.group;
  const int qh = head * a.group + row % a.group;
  const float inv = (l > 0.f ? 1.f / l : l) * a.v_scale;  // (NaN stays)
  if (lane < D / 4) {
    uint16_t* to = static_cast<uint16_t*>(a.out.d_data) + token * a.out.token_stride + qh * a.out.head_stride + 4 * lane;
    const float2 e = make_float2(f.x * inv, f.y * inv), q = make_float2(f.z * inv, f.w * inv);
    *reinterpret_cast<uint2*>(to) = a.bf16 ? make_uint2(round2<__nv_bfloat16>(e), round2<__nv_bfloat16>(q))
                                           : make_uint2(round2<__half>(e), round2<__half>(q));
  }
  if (a.lse && lane == 0) a.lse[token * a.hq + qh] = l == 0.f ? -INFINITY : (top + log2f(l)) * 0.6931471805599453f;
}

// Attention of up to NB * 8 query rows (a token's heads of one key head, or a few
// tokens') at a time. Every warp has a key head and every `streams`-th tile of 32
// keys of the CTA's share, copies it for itself into a ring of its own (no barriers
// between warps), and joins its sums with the head's other warps' at the item's end.
// All key heads of a tile are read by one CTA at about the same time: a token's scales
// are 8 bytes a head, a quarter of what memory delivers.
//
// Tokens are the long side of both products: S^T = K Q^T and O^T = V^T P^T, in
// mma.sync of 16 x 8 x 16, so that a code goes from shared memory to a register of the
// operand with one conversion (two codes) and one product with its scale. P^T is S^T's
// registers after a transposition of 8 x 8 blocks. (tcgen05 takes its operands from
// shared memory or TMEM: the same conversions, and a way there and back. At 8 rows the
// products need a third of mma.sync's rate, 1,012 multiply-adds a cycle and SM.)
//
// What bounds it: 32 keys of a head are 4.6 KB, 200 cycles of an SM's share of memory,
// and 555 instructions, 139 cycles of issue slots; conversions and their products take
// half of theirs (64 lanes a cycle each). Both together come to 234 cycles, at 56 % of
// the issue slots: 64 single tokens over 2k to 48k keys (4 key heads of 128, 896 MB) take
// 171 us, 5.2 TB/s, 78 % of a copy's rate, where the copies alone take 148 and the
// arithmetic alone 137, and 12 of them are the start, the item's end and the join. 37
// tokens of 16 rows (347 MB) take 98 us, with twice the products. One token over 24,577
// keys takes 12.4 us on the device: share, pages and first tile 3.5, tiles 2, the
// item's end 2, the join 3, launches.
//
// 12 warps of 168 registers: 16 of 128 took 178 us for the 64 tokens, 20 of 96 239, 8 of
// 255 205. The next tile's scores computed beside this tile's weights took 186.
template <int D, int NB>
__global__ void __launch_bounds__(kFewWarps * 32, 1) k_kv4_few(const __grid_constant__ FewArgs a) {
  constexpr int kWarps = kFewWarps, kRows = 8 * NB, kStages = stages(D), kStage = stage_bytes(D);
  constexpr int W = D / 32;               // words of codes a lane has of a key, and half words of a value
  constexpr int kCodes = kFewTile * D / 2, kScales = kFewTile * scale_bytes(D), SB = scale_bytes(D);
  extern __shared__ __align__(128) unsigned char smem[];
  pdl_enter();
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");  // (the join's blocks, which wait for this kernel's end)
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, g = lane >> 2, c = lane & 3;
  // tokens of no request
  {
    const int64_t first = a.plan->first, last = a.plan->last, none = first + a.n_tokens - last, pieces = none * a.hq * (D / 8);
    for (int64_t i = (int64_t)blockIdx.x * blockDim.x + threadIdx.x; i < pieces; i += (int64_t)gridDim.x * blockDim.x) {
      const int64_t x = i / (D / 8), h = x % a.hq;
      int64_t t = x / a.hq;
      if (t >= first) t += last - first;
      *reinterpret_cast<uint4*>(static_cast<uint16_t*>(a.out.d_data) + t * a.out.token_stride + h * a.out.head_stride + i % (D / 8) * 8) =
          make_uint4(0, 0, 0, 0);
      if (a.lse) a.lse[t * a.hq + h] = -INFINITY;
    }
  }
  const uint32_t ring = (uint32_t)__cvta_generic_to_shared(smem) + warp * kStages * kStage;
  const int page_size = 1 << a.page_shift;
  // Row r of a tile's keys in shared memory (the product's row) is token 2 c -> c, 2 c + 1
  // -> 4 + c of each 8: so lane (g, c)'s values, of the product's inner places 2 c, 2 c +
  // 1, are tokens c and 4 + c, whose rows lie in other banks for other c.
  const auto row_of = [](int token) { return (token & ~7) | (token & 3) << 1 | (token >> 2 & 1); };
  const auto token_of = [](int row) { return (row & ~7) | (row & 1) << 2 | (row >> 1 & 3); };
  FewWalk w;
  w.start(a);
  FewItem it;
  while (w.next(a, it)) {
    const int heads = min(a.heads, a.hk - it.hb * a.heads);
    const int streams = kWarps / heads;
    const int my_head = warp % heads, stream = warp / heads;
    const bool busy = stream < streams;
    const int head = it.hb * a.heads + my_head;
    const KvUnit& u = it.unit;
    const int32_t seen_lo = u.pos >= a.window ? u.pos - a.window + 1 : 0, seen_hi = u.pos + u.tokens;  // keys that some row sees
    const int n = busy ? max(0, (it.te - it.tb - stream + streams - 1) / streams) : 0;
    float o[D / 16][NB][4], ref[NB][2], lim[NB][2], l[NB][2];
#pragma unroll
    for (int b = 0; b < NB; ++b) {
#pragma unroll
      for (int m = 0; m < D / 16; ++m)
#pragma unroll
        for (int i = 0; i < 4; ++i) o[m][b][i] = 0.f;
#pragma unroll
      for (int i = 0; i < 2; ++i) ref[b][i] = 0.f, lim[b][i] = -INFINITY, l[b][i] = 0.f;
    }
    if (n > 0) {
      const int32_t* pages = a.pages + u.req * a.pages_stride;
      const uint32_t key0 = (uint32_t)(it.tb + stream) * kFewTile, key_step = (uint32_t)streams * kFewTile;
      // Pages of 16 tiles' halves, a lane each: of the tiles now copied, and of the next
      // 16. Bits of the halves that are in the cache, and of those without a key that nobody sees.
      uint32_t pages_now = 0, in_cache = 0, in_whole = 0;
      int32_t pages_next;
      const auto look_up = [&](int j) {  // of tiles j..
        const int x = j + (lane >> 1);
        const uint32_t key = key0 + (uint32_t)x * key_step + 16 * (lane & 1);
        pages_next = x < n && key < (uint32_t)seen_hi && key + 16 > (uint32_t)seen_lo ? pages[key >> a.page_shift] : -1;
      };
      const auto turn = [&](int j) {  // to tiles j..
        const bool held = (uint32_t)pages_next < (uint32_t)a.num_pages;
        pages_now = held ? pages_next : 0;
        const uint32_t key = key0 + (uint32_t)(j + (lane >> 1)) * key_step + 16 * (lane & 1);
        if (!held && j + (lane >> 1) < n && key < (uint32_t)seen_hi && key + 16 > (uint32_t)seen_lo)
          latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
        in_cache = __ballot_sync(kFull, held);
        in_whole = __ballot_sync(kFull, held && key >= (uint32_t)seen_lo && key + 16 <= (uint32_t)seen_hi);
        if (j + 16 < n) look_up(j + 16);
      };
      look_up(0);
      // (on their way with the pages)
      uint4 queries[NB][D / 32];
#pragma unroll
      for (int b = 0; b < NB; ++b) load_rows<D>(a, u, head, 8 * b, queries[b]);
      uint32_t copy_key = key0, copy_to = ring;
      // A lane copies pieces (lane & 1) and 2 + (lane & 1) of token lane / 2 of each half,
      // the last piece of heads of 32 or 96 of token `lane`, and that token's scales.
      // Places in pages of 16 tokens are the lane's own, in larger ones the tile's are added.
      const bool small = page_size == 16;
      const uint32_t half_token = lane >> 1, own_token = small ? lane & 15 : lane, own_to = row_of(lane);
      const uint32_t k_page = (uint32_t)a.k.page_stride, k_token = (uint32_t)a.k.token_stride;  // (all below 2^32)
      const uint32_t v_page = (uint32_t)a.v.page_stride, v_token = (uint32_t)a.v.token_stride;
      const uint32_t ks_page = (uint32_t)a.k.scale_page_stride, ks_token = (uint32_t)a.k.scale_token_stride;
      const uint32_t vs_page = (uint32_t)a.v.scale_page_stride, vs_token = (uint32_t)a.v.scale_token_stride;
      const auto times = [](uint32_t x, uint32_t y) { return (uint64_t)x * y; };
      const uint8_t* const kh = static_cast<const uint8_t*>(a.k.d_codes) + head * a.k.head_stride;
      const uint8_t* const vh = static_cast<const uint8_t*>(a.v.d_codes) + head * a.v.head_stride;
      const uint8_t* const kp = kh + 16 * (lane & 1) + times(half_token, k_token);
      const uint8_t* const vp = vh + 16 * (lane & 1) + times(half_token, v_token);
      const uint8_t* const kl = kh + 16 * (W - 1) + times(own_token, k_token);
      const uint8_t* const vl = vh + 16 * (W - 1) + times(own_token, v_token);
      const uint8_t* const ks = static_cast<const uint8_t*>(a.k.d_scales) + head * a.k.scale_head_stride + times(own_token, ks_token);
      const uint8_t* const vs = static_cast<const uint8_t*>(a.v.d_scales) + head * a.v.scale_head_stride + times(own_token, vs_token);
      const uint32_t k_to = row_of(half_token) * (D / 2) + 16 * (lane & 1);
      // (128 elements: tokens 2, 3 of each 4 have their halves changed over, for the banks)
      const uint32_t v_to = kCodes + half_token * (D / 2) + 16 * (lane & 1) + (D == 128 ? (half_token & 2) << 4 : 0);
      // the tile's copies; kWhole: all of it is in the cache and seen
      const auto copy_tile = [&](auto whole, int shift, uint32_t key, uint32_t at) {
        constexpr bool kWhole = decltype(whole)::value;
        bool held[2] = {true, true}, held_own = true;
        if (!kWhole) {
#pragma unroll
          for (int h = 0; h < 2; ++h) {
            const uint32_t x = key + 16 * h + half_token;
            held[h] = (in_cache >> (shift + h) & 1) && x >= (uint32_t)seen_lo && x < (uint32_t)seen_hi;
          }
          const uint32_t x = key + lane;
          held_own = (in_cache >> (shift + (lane >> 4)) & 1) && x >= (uint32_t)seen_lo && x < (uint32_t)seen_hi;
        }
        const auto codes = [&](const uint8_t* k, const uint8_t* v, int h) {
          copy_async<16, kWhole>(at + k_to + 16 * h * (D / 2), k, held[h]);
          copy_async<16, kWhole>(at + v_to + 16 * h * (D / 2), v, held[h]);
          if constexpr (W == 4) {
            copy_async<16, kWhole>(at + k_to + 16 * h * (D / 2) + 32, k + 32, held[h]);
            copy_async<16, kWhole>(at + (v_to ^ 32) + 16 * h * (D / 2), v + 32, held[h]);
          }
        };
        const auto rest = [&](const uint8_t* k, const uint8_t* v, const uint8_t* k_scale, const uint8_t* v_scale) {
          if constexpr (W & 1) {
            copy_async<16, kWhole>(at + own_to * (D / 2) + 16 * (W - 1), k, held_own);
            copy_async<16, kWhole>(at + kCodes + lane * (D / 2) + 16 * (W - 1), v, held_own);
          }
          copy_async<SB, kWhole>(at + 2 * kCodes + own_to * SB, k_scale, held_own);
          copy_async<SB, kWhole>(at + 2 * kCodes + kScales + lane * SB, v_scale, held_own);
        };
        if (small) {
          const uint32_t page0 = __shfl_sync(kFull, pages_now, shift), page1 = __shfl_sync(kFull, pages_now, shift + 1);
          const uint32_t own = lane < 16 ? page0 : page1;
          if constexpr (W >= 2) {
            codes(kp + times(page0, k_page), vp + times(page0, v_page), 0);
            codes(kp + times(page1, k_page), vp + times(page1, v_page), 1);
          }
          rest(kl + times(own, k_page), vl + times(own, v_page), ks + times(own, ks_page), vs + times(own, vs_page));
        } else {
          // (one page; where only the second half is in the cache, it is the second's)
          const uint32_t page = __shfl_sync(kFull, pages_now, kWhole || (in_cache >> shift & 1) ? shift : shift + 1);
          const uint32_t in = key & (page_size - 1);
          const uint8_t* k = kp + times(page, k_page) + times(in, k_token);
          const uint8_t* v = vp + times(page, v_page) + times(in, v_token);
          if constexpr (W >= 2) {
            codes(k, v, 0);
            codes(k + times(16, k_token), v + times(16, v_token), 1);
          }
          rest(kl + times(page, k_page) + times(in, k_token), vl + times(page, v_page) + times(in, v_token),
               ks + times(page, ks_page) + times(in, ks_token), vs + times(page, vs_page) + times(in, vs_token));
        }
      };
      const auto copy = [&](int j) {
        if ((j & 15) == 0) turn(j);
        const int shift = 2 * (j & 15);
        if ((in_whole >> shift & 3) == 3)
          copy_tile(std::true_type(), shift, copy_key, copy_to);
        else
          copy_tile(std::false_type(), shift, copy_key, copy_to);
        copy_key += key_step;
        copy_to = copy_to + kStage == ring + kStages * kStage ? ring : copy_to + kStage;
      };
#pragma unroll
      for (int j = 0; j < kStages - 1; ++j) {
        if (j < n) copy(j);
        asm volatile("cp.async.commit_group;\n" ::: "memory");
      }
      uint32_t qf[NB][D / 16][2];
      float cs[NB][2];
#pragma unroll
      for (int b = 0; b < NB; ++b) {
        float power;
        convert_rows<D>(queries[b], a.bf16, qf[b], power);
#pragma unroll
        for (int i = 0; i < 2; ++i) cs[b][i] = score_factor(__shfl_sync(kFull, power, 4 * (2 * c + i)) * a.scale);
      }
      uint32_t at = warp * kStages * kStage;  // in smem
      uint32_t key = key0;
      // tiles that every row sees whole begin within
      const uint32_t whole_lo = (uint32_t)max((int64_t)seen_hi - a.window, (int64_t)0);
      const int32_t whole_hi = u.pos - (kFewTile - 1);
      for (int j = 0; j < n; ++j) {
        asm volatile("cp.async.wait_group %0;\n" ::"n"(kStages - 2) : "memory");
        __syncwarp();
        if (j + kStages - 1 < n) copy(j + kStages - 1);
        asm volatile("cp.async.commit_group;\n" ::: "memory");
        // scores: S[half][block][...] of tokens token_of(g), token_of(g + 8) and rows 2c, 2c + 1
        float s[2][NB][4];
        uint32_t codes[2][2][W], k_scales[2][2][W];
#pragma unroll
        for (int t = 0; t < 2; ++t) {
#pragma unroll
          for (int i = 0; i < 2; ++i) {
            const int row = 16 * t + 8 * i + g;
            const unsigned char* p = smem + (at + row * (D / 2) + 4 * W * c);
            uint32_t(&x)[W] = codes[t][i];
            uint32_t(&scale)[W] = k_scales[t][i];
            if constexpr (W == 4) {
              const uint4 y = *reinterpret_cast<const uint4*>(p);
              x[0] = y.x, x[1] = y.y, x[2] = y.z, x[3] = y.w;
            } else if constexpr (W == 2) {
              const uint2 y = *reinterpret_cast<const uint2*>(p);
              x[0] = y.x, x[1] = y.y;
            } else {
#pragma unroll
              for (int k = 0; k < W; ++k) x[k] = reinterpret_cast<const uint32_t*>(p)[k];
            }
            // each word's group's scale, twice
            const unsigned char* sp = smem + (at + 2 * kCodes + row * SB);
            if constexpr (W == 4) {
              const uint32_t two = scales_of(reinterpret_cast<const uint16_t*>(sp)[c]);
              scale[0] = scale[1] = __byte_perm(two, 0, 0x1010);
              scale[2] = scale[3] = __byte_perm(two, 0, 0x3232);
            } else if constexpr (W == 3) {  // (12 words of 6 groups: the middle word goes with the first or the last)
              const uint32_t y = sp[3 * c / 2], z = sp[3 * c / 2 + 1];
              scale[0] = scales_of(y * 0x101), scale[2] = scales_of(z * 0x101);
              scale[1] = c & 1 ? scale[2] : scale[0];
            } else {
              const uint32_t y = sp[W * c / 2];
#pragma unroll
              for (int k = 0; k < W; ++k) scale[k] = scales_of(y * 0x101);
            }
          }
        }
        // (the halves in turn: a product takes longer than the conversions for the next)
#pragma unroll
        for (int k = 0; k < W; ++k) {
#pragma unroll
          for (int t = 0; t < 2; ++t) {
            uint32_t x[4], y[4];  // the word's pairs: rows g, g + 8
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              x[i] = mul_h2(pair_of<0>(codes[t][i][k]), k_scales[t][i][k]);
              x[2 + i] = mul_h2(pair_of<1>(codes[t][i][k]), k_scales[t][i][k]);
              y[i] = mul_h2(pair_of<2>(codes[t][i][k]), k_scales[t][i][k]);
              y[2 + i] = mul_h2(pair_of<3>(codes[t][i][k]), k_scales[t][i][k]);
            }
#pragma unroll
            for (int b = 0; b < NB; ++b) {
              if (k == 0)
                mma_first(s[t][b], x, qf[b][0][0], qf[b][0][1]);
              else
                mma(s[t][b], x, qf[b][2 * k][0], qf[b][2 * k][1]);
              mma(s[t][b], y, qf[b][2 * k + 1][0], qf[b][2 * k + 1][1]);
            }
          }
        }
        if ((int32_t)key > whole_hi || key < whole_lo) {  // some row does not see some key
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int64_t hi = u.pos + (8 * b + 2 * c + i) / a.group;
#pragma unroll
              for (int t = 0; t < 2; ++t)
#pragma unroll
                for (int k = 0; k < 2; ++k) {
                  const int64_t x = (int64_t)key + 16 * t + token_of(8 * k + g);
                  if (x > hi || x <= hi - a.window) s[t][b][2 * k + i] = -INFINITY;
                }
            }
        }
        bool move = false;
#pragma unroll
        for (int b = 0; b < NB; ++b)
#pragma unroll
          for (int i = 0; i < 2; ++i)
            move |= fmaxf(fmaxf(s[0][b][i], s[0][b][i + 2]), fmaxf(s[1][b][i], s[1][b][i + 2])) > lim[b][i];
        if (__any_sync(kFull, move)) {
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              float top = fmaxf(fmaxf(s[0][b][i], s[0][b][i + 2]), fmaxf(s[1][b][i], s[1][b][i + 2]));
#pragma unroll
              for (int x = 4; x < 32; x <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, x));
              if (top > lim[b][i]) {
                const float to = reference(top, cs[b][i], kLift), back = lim[b][i] == -INFINITY ? 0.f : ex2(ref[b][i] - to);
                ref[b][i] = to, lim[b][i] = __fadd_rd(top, kSlack / cs[b][i]);
                l[b][i] *= back;
#pragma unroll
                for (int m = 0; m < D / 16; ++m) o[m][b][i] *= back, o[m][b][i + 2] *= back;
              }
            }
        }
        uint32_t p[2][NB][2];  // weights, as the second product's operand
#pragma unroll
        for (int t = 0; t < 2; ++t)
#pragma unroll
          for (int b = 0; b < NB; ++b)
#pragma unroll
            for (int k = 0; k < 2; ++k) {
              float2 x = fma2(make_float2(s[t][b][2 * k], s[t][b][2 * k + 1]), make_float2(cs[b][0], cs[b][1]),
                              make_float2(-ref[b][0], -ref[b][1]));
              x = make_float2(ex2(x.x), ex2(x.y));
              const float2 sum = add2(make_float2(l[b][0], l[b][1]), x);
              l[b][0] = sum.x, l[b][1] = sum.y;
              p[t][b][k] = transposed(round2<__half>(x));
            }
#pragma unroll
        for (int t = 0; t < 2; ++t) {
          // values of tokens c, 4 + c, 8 + c, 12 + c of the half, elements [g D/8, (g+1) D/8)
          uint32_t even[2][(W + 1) / 2], odd[2][(W + 1) / 2], scales[2][2];
#pragma unroll
          for (int k = 0; k < 2; ++k) {
            uint32_t x[2][(W + 1) / 2], sb[2][2];
#pragma unroll
            for (int i = 0; i < 2; ++i) {
              const int token = 16 * t + 8 * k + 4 * i + c;
              const unsigned char* row = smem + (at + kCodes + token * (D / 2));
              if constexpr (W == 4) {
                const uint2 y = *reinterpret_cast<const uint2*>(row + 16 * ((g >> 1) ^ (c & 2)) + 8 * (g & 1));
                x[i][0] = y.x, x[i][1] = y.y;
              } else if constexpr (W == 2) {
                x[i][0] = *reinterpret_cast<const uint32_t*>(row + 4 * g);
              } else {
                const uint16_t* y = reinterpret_cast<const uint16_t*>(row + 2 * W * g);
                x[i][0] = y[0];
                if constexpr (W == 3) x[i][0] |= (uint32_t)y[1] << 16, x[i][1] = y[2];
              }
              const unsigned char* sp = smem + (at + 2 * kCodes + kScales + token * SB);
              sb[i][0] = sp[W * g / 4];
              sb[i][1] = W == 3 ? sp[min((W * g / 4) + 1, D / 16 - 1)] : 0;
            }
#pragma unroll
            for (int q = 0; q < (W + 1) / 2; ++q) {
              const uint32_t y = x[0][q], z = x[1][q];
              even[k][q] = low_nibbles(y, z << 4);
              odd[k][q] = low_nibbles(y >> 4, z);
            }
            scales[k][0] = scales_of(sb[0][0] | sb[1][0] << 8);
            scales[k][1] = W == 3 ? scales_of(sb[0][1] | sb[1][1] << 8) : 0;
          }
#pragma unroll
          for (int m = 0; m < D / 16; ++m) {
            const auto byte = [&](uint32_t x) {
              return m % 4 == 0 ? pair_of<0>(x) : m % 4 == 1 ? pair_of<1>(x) : m % 4 == 2 ? pair_of<2>(x) : pair_of<3>(x);
            };
            // (heads of 96: a lane's 12 elements lie in two groups)
            const bool second = W == 3 && (12 * g + 2 * m) / 16 > 12 * g / 16;
            const uint32_t s0 = second ? scales[0][1] : scales[0][0], s1 = second ? scales[1][1] : scales[1][0];
            const uint32_t x[4] = {mul_h2(byte(even[0][m / 4]), s0), mul_h2(byte(odd[0][m / 4]), s0),
                                   mul_h2(byte(even[1][m / 4]), s1), mul_h2(byte(odd[1][m / 4]), s1)};
#pragma unroll
            for (int b = 0; b < NB; ++b) mma(o[m][b], x, p[t][b][0], p[t][b][1]);
          }
        }
        at = at + kStage == (warp + 1) * kStages * kStage ? warp * kStages * kStage : at + kStage;
        key += key_step;
      }
      asm volatile("cp.async.wait_group 0;\n" ::: "memory");
    }
    // the item's sums: warps of a head side by side in shared memory
#pragma unroll
    for (int b = 0; b < NB; ++b)
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int x = 4; x < 32; x <<= 1) l[b][i] += __shfl_xor_sync(kFull, l[b][i], x);
      }
    __syncthreads();  // (the rings are done with)
    float* const sums = reinterpret_cast<float*>(smem);
    float2* const stats = reinterpret_cast<float2*>(sums + kWarps * kRows * sum_row(D));
    if (busy) {
#pragma unroll
      for (int b = 0; b < NB; ++b)
#pragma unroll
        for (int i = 0; i < 2; ++i) {
          const int row = warp * kRows + 8 * b + 2 * c + i;
#pragma unroll
          for (int m = 0; m < D / 16; ++m)  // (elements g D/8 + 2m, + 1)
            *reinterpret_cast<float2*>(sums + row * sum_row(D) + 16 * m + 2 * g) = make_float2(o[m][b][i], o[m][b][i + 2]);
          if (g == 0 && 8 * b + 2 * c + i < u.tokens * a.group && too_far(ref[b][i], kLift)) latch_error(a.status, SMETRIC_ERR_OVERFLOW);
          if (g == 0) stats[row] = make_float2(lim[b][i] == -INFINITY && l[b][i] == 0.f ? -INFINITY : ref[b][i], l[b][i]);
        }
    }
    __syncthreads();
    const int rows = u.tokens * a.group;
    for (int y = warp; y < heads * rows; y += kWarps) {  // a row a warp
      const int h = y / rows, row = y - h * rows, d = 4 * lane, q = d / (D / 8), m = d % (D / 8) / 2;
      float top = -INFINITY;
      for (int k = 0; k < streams; ++k) top = fmaxf(top, stats[(k * heads + h) * kRows + row].x);
      float sum = 0.f;
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
      for (int k = 0; k < streams; ++k) {
        const int at = (k * heads + h) * kRows + row;
        const float2 st = stats[at];
        const float e = st.x == -INFINITY ? 0.f : ex2(st.x - top);
        sum += st.y * e;
        if (D == 128 || d < D) {
          const float2 p0 = *reinterpret_cast<const float2*>(sums + at * sum_row(D) + 16 * m + 2 * q);
          const float2 p1 = *reinterpret_cast<const float2*>(sums + at * sum_row(D) + 16 * (m + 1) + 2 * q);
          f.x += p0.x * e, f.y += p0.y * e, f.z += p1.x * e, f.w += p1.y * e;
        }
      }
      if (it.whole) {
        write_row<D>(a, u, it.hb * a.heads + h, row, f, top, sum);
      } else {
        const int64_t at = ((int64_t)it.slot * a.heads + h) * kRows + row;
        if (D == 128 || d < D) *reinterpret_cast<float4*>(a.part + at * D + d) = f;
        if (lane == 0) a.part_ml[at] = make_float2(top, sum);
      }
    }
    __syncthreads();  // (the sums' memory is the rings')
  }
}

// out = sum_i 2^(ref_i - top) O_i / sum_i 2^(ref_i - top) l_i over a unit's pieces, the
// pieces in an order that depends on their number alone. The blocks in turn for the
// units that are shared. A row of few pieces has a warp, one of many (a long sequence
// alone) a block. Bound by latency: 3 to 5 us.
constexpr int kFewJoin = 512;
constexpr int kFewPieces = 8;

template <int D, int NB>
__device__ __forceinline__ void join_few(const FewArgs& a, const KvShare& s, int c1, int block, int blocks) {
  constexpr int kRows = 8 * NB, kWarps = kFewJoin / 32;
  __shared__ float4 sums[kWarps][D / 4];
  __shared__ float2 stats[kWarps];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const KvUnit& u = s.last;
  const int unit_rows = u.tokens * a.group, rows = min(a.heads, a.hk - s.h1 * a.heads) * unit_rows, n = s.n_last;
  const bool holds = lane < D / 4;
  if (n <= kFewPieces) {
    for (int x = block * kWarps + warp; x < rows; x += blocks * kWarps) {
      const int h = x / unit_rows, row = x - h * unit_rows;
      const auto at = [&](int i) { return ((int64_t)(2 * (c1 + i) + (i == 0)) * a.heads + h) * kRows + row; };
      float2 ml[kFewPieces];
      float4 p[kFewPieces];
#pragma unroll
      for (int i = 0; i < kFewPieces; ++i) {
        ml[i] = make_float2(-INFINITY, 0.f);
        p[i] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < n) {
          ml[i] = a.part_ml[at(i)];
          if (holds) p[i] = *reinterpret_cast<const float4*>(a.part + at(i) * D + 4 * lane);
        }
      }
      float top = -INFINITY, l = 0.f;
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int i = 0; i < kFewPieces; ++i) top = fmaxf(top, ml[i].x);
#pragma unroll
      for (int i = 0; i < kFewPieces; ++i) {
        const float e = ml[i].x == -INFINITY ? 0.f : ex2(ml[i].x - top);  // (no key of it is seen)
        l += ml[i].y * e;
        f.x += p[i].x * e, f.y += p[i].y * e, f.z += p[i].z * e, f.w += p[i].w * e;
      }
      write_row<D>(a, u, s.h1 * a.heads + h, row, f, top, l);
    }
    return;
  }
  for (int x = block; x < rows; x += blocks) {
    const int h = x / unit_rows, row = x - h * unit_rows;
    const auto at = [&](int i) { return ((int64_t)(2 * (c1 + i) + (i == 0)) * a.heads + h) * kRows + row; };
    constexpr int P = 5;  // pieces a warp has on their way
    float top = -INFINITY, l = 0.f;
    float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
    for (int i0 = warp; i0 < n; i0 += P * kWarps) {
      float2 ml[P];
      float4 p[P];
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const int i = i0 + k * kWarps;
        ml[k] = make_float2(-INFINITY, 0.f);
        p[k] = make_float4(0.f, 0.f, 0.f, 0.f);
        if (i < n) {
          ml[k] = a.part_ml[at(i)];
          if (holds) p[k] = *reinterpret_cast<const float4*>(a.part + at(i) * D + 4 * lane);
        }
      }
      float to = top;
#pragma unroll
      for (int k = 0; k < P; ++k) to = fmaxf(to, ml[k].x);
      const float back = top == -INFINITY ? 0.f : ex2(top - to);
      top = to;
      l *= back;
      f.x *= back, f.y *= back, f.z *= back, f.w *= back;
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const float e = ml[k].x == -INFINITY ? 0.f : ex2(ml[k].x - to);
        l += ml[k].y * e;
        f.x += p[k].x * e, f.y += p[k].y * e, f.z += p[k].z * e, f.w += p[k].w * e;
      }
    }
    if (holds) sums[warp][lane] = f;
    if (lane == 0) stats[warp] = make_float2(top, l);
    __syncthreads();
    if (warp == 0) {
      float all = -INFINITY;
      l = 0.f;
      f = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll
      for (int k = 0; k < kWarps; ++k) all = fmaxf(all, stats[k].x);
#pragma unroll
      for (int k = 0; k < kWarps; ++k) {
        const float e = stats[k].x == -INFINITY ? 0.f : ex2(stats[k].x - all);
        l += stats[k].y * e;
        if (holds) {
          const float4 p = sums[k][lane];
          f.x += p.x * e, f.y += p.y * e, f.z += p.z * e, f.w += p.w * e;
        }
      }
      write_row<D>(a, u, s.h1 * a.heads + h, row, f, all, l);
    }
    __syncthreads();
  }
}

// The units that several CTAs share; with kMany those of the chunks' kernel too.
template <int D, int NB, bool kMany>
__global__ void __launch_bounds__(kFewJoin) k_kv4_join(const __grid_constant__ FewArgs a) {
  // (the plan was done before the kernel that this one waits for)
  const auto find = [](int units, const int32_t* split, const KvShare* shares, int at, int n, KvShare& s, int& c1, int& block, int& blocks) {
    blocks = units ? n / units : 0, block = units ? at / units : 0;
    if (block >= blocks) return;
    c1 = split[at % units];
    s = shares[c1];
  };
  constexpr int kParts = kFewJoin / kJoinThreads;  // a block is as many for the units of many rows
  KvShare few = {}, many = {};
  int few_c1 = 0, few_block, few_blocks, many_c1 = 0, many_block = 0, many_blocks = 0;
  find(a.plan->n_split_few, a.split, a.shares, blockIdx.x, gridDim.x, few, few_c1, few_block, few_blocks);
  if (kMany)
    find(a.plan->n_split, a.many.split, a.many.shares, blockIdx.x * kParts + threadIdx.x / kJoinThreads, gridDim.x * kParts, many, many_c1,
         many_block, many_blocks);
  pdl_enter();
  if (few_block < few_blocks) join_few<D, NB>(a, few, few_c1, few_block, few_blocks);
  if (kMany && many_block < many_blocks) {
    if (a.bf16)
      join_unit<__nv_bfloat16>(a.many, many, many_c1, many_block, many_blocks, threadIdx.x % kJoinThreads);
    else
      join_unit<__half>(a.many, many, many_c1, many_block, many_blocks, threadIdx.x % kJoinThreads);
  }
}

template <int D, int NB>
bool few_limit() {
  return cudaFuncSetAttribute((const void*)k_kv4_few<D, NB>, cudaFuncAttributeMaxDynamicSharedMemorySize, few_smem(D, 8 * NB)) ==
         cudaSuccess;
}
template <int D, int NB>
int launch_few(smetric_kv* kv, const FewArgs& a, cudaStream_t s) {
  int rc = launch_k(k_kv4_few<D, NB>, dim3((unsigned)kv->num_sms), dim3(kFewWarps * 32), (size_t)few_smem(D, 8 * NB), s, true, a);
  if (rc) return rc;
  kv->launches += 2;
  return launch_k(kv->one_join ? k_kv4_join<D, NB, true> : k_kv4_join<D, NB, false>, dim3((unsigned)kv->num_sms * 2), dim3(kFewJoin), 0, s, true, a);
}

}  // namespace

bool smetric::few_limits() {
  return few_limit<32, 1>() && few_limit<32, 2>() && few_limit<64, 1>() && few_limit<64, 2>() && few_limit<96, 1>() &&
         few_limit<96, 2>() && few_limit<128, 1>() && few_limit<128, 2>();
}

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
  // (few rows: enough blocks for the SMs first)
  a.rows = (int32_t)std::min<int64_t>(kReadRows, std::max<int64_t>(1, n_rows / (8 * kv->num_sms)));
  for (int w = 0; w < 2; ++w)
    a.wide[w] = !(reinterpret_cast<uintptr_t>(a.out[w].d_data) & 31) && a.out[w].token_stride % 16 == 0 && a.out[w].head_stride % 16 == 0;
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
      !scale_ok(std::ldexp(scale, k_cache.exp)) || !heads_ok(q, kv->n_tokens) || !heads_ok(out, kv->n_tokens) || (reinterpret_cast<uintptr_t>(d_lse) & 3))
    return SMETRIC_ERR_INVALID_ARG;
  if (kv->n_tokens == 0) return SMETRIC_OK;
  if (!kv->all_few) {
    rc = attention_many_rows(kv, k_cache, v_cache, q, scale, out, d_lse, stream);
    if (rc || !kv->few.rows) return rc;
  }
  FewArgs a = {};
  a.k = k_cache;
  a.v = v_cache;
  a.q = q;
  a.out = out;
  a.lse = d_lse;
  a.plan = kv->plan;
  a.units = kv->few.units;
  a.shares = kv->few.shares;
  a.split = kv->few.split;
  a.part = kv->few.part;
  a.part_ml = kv->few.part_ml;
  a.pages = kv->pages;
  a.pages_stride = kv->pages_stride;
  a.n_tokens = kv->n_tokens;
  a.num_pages = (int32_t)c.num_pages;
  a.hq = c.num_q_heads;
  a.hk = c.num_kv_heads;
  a.group = kv->group;
  a.heads = kv->few.heads;
  a.blocks = kv->few.blocks;
  a.page_shift = __builtin_ctz((unsigned)c.page_size);
  a.window = kv->window;
  a.scale = std::ldexp(scale, k_cache.exp) * 1.4426950408889634f;
  a.v_scale = std::ldexp(1.f, v_cache.exp);
  a.bf16 = c.dtype == SMETRIC_BF16;
  a.status = kv->status;
  a.many.out = out;
  a.many.lse = d_lse;
  a.many.shares = kv->shares;
  a.many.split = kv->split;
  a.many.part = kv->part;
  a.many.part_ml = kv->part_ml;
  a.many.hq = a.hq;
  a.many.group = kv->group;
  a.many.tile_tokens = kv->tile_tokens;
  a.many.D = c.head_dim;
  a.many.v_scale = a.v_scale;
  a.many.wide = !(reinterpret_cast<uintptr_t>(out.d_data) & 31) && out.token_stride % 16 == 0 && out.head_stride % 16 == 0;
  const cudaStream_t s = reinterpret_cast<cudaStream_t>(stream);
  const bool one = kv->few.rows == 8;
  switch (c.head_dim) {
    case 32: return one ? launch_few<32, 1>(kv, a, s) : launch_few<32, 2>(kv, a, s);
    case 64: return one ? launch_few<64, 1>(kv, a, s) : launch_few<64, 2>(kv, a, s);
    case 96: return one ? launch_few<96, 1>(kv, a, s) : launch_few<96, 2>(kv, a, s);
    default: return one ? launch_few<128, 1>(kv, a, s) : launch_few<128, 2>(kv, a, s);
  }
}

}  // extern "C"
