// The join of the pieces of a unit that several CTAs share (attention.cu), and what it
// shares with the attention itself.
#pragma once

#include <cuda_bf16.h>
#include <cuda_fp16.h>
#include <cuda_runtime.h>
#include <stdint.h>

#include "kv_impl.cuh"

namespace smetric {

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}

template <typename T>
struct Type;
template <>
struct Type<__nv_bfloat16> {
  static constexpr uint32_t kFormat = 1;  // of the tensor cores' operands
  static constexpr float kLift = 0.f;
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __nv_bfloat162 p = __floats2bfloat162_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
};
template <>
struct Type<__half> {
  static constexpr uint32_t kFormat = 0;
  // Weights up to 2^(kLift + kSlack) = 2^15: half precision's range ends at
  // 65,504, and the small weights of long rows stay normal numbers longer.
  static constexpr float kLift = 7.f;
  static __device__ __forceinline__ uint32_t pack(float a, float b) {
    const __half2 p = __floats2half2_rn(a, b);
    return *reinterpret_cast<const uint32_t*>(&p);
  }
};

// Partial sums: a slot's two query tiles, each D/4 columns of kTile rows of four
// sums, so that the threads of a warp (a row each) store in whole lines. The
// place of a column's first row, in units of four sums.
__device__ __forceinline__ int64_t part_at(int D, int64_t slot, int tile, int column) {
  return ((slot * 2 + tile) * (D / 4) + column) * kTile;
}

// 16 elements of an output.
__device__ __forceinline__ void store16(bool wide, void* p, const uint32_t* r) {
  if (wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(r[0], r[1], r[2], r[3]);
    static_cast<uint4*>(p)[1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
}

// The pieces of 16 elements of a row, so far.
struct Joined {
  float top = -INFINITY, l = 0.f;  // largest reference exponent; sum of weights, to it
  float4 o[4] = {};
  __device__ __forceinline__ void add(float ref, float weights, const float4 (&p)[4]) {
    const float next = fmaxf(top, ref);
    if (next == -INFINITY) return;  // no key so far
    const float f = ex2(top - next), g = ex2(ref - next);
    top = next;
    l = l * f + weights * g;
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      o[i].x = o[i].x * f + p[i].x * g, o[i].y = o[i].y * f + p[i].y * g;
      o[i].z = o[i].z * f + p[i].z * g, o[i].w = o[i].w * f + p[i].w * g;
    }
  }
};

// out = sum_i 2^(ref_i - top) O_i / sum_i 2^(ref_i - top) l_i over a unit's
// pieces. G threads share 16 elements of a row (a whole sector of the output),
// thread g taking pieces g, g + G, ..., two of them in flight: the order of the
// sums depends on the number of pieces alone.
// CTA c1's share starts the unit; the block is one of `blocks` for it.
constexpr int kJoinThreads = 128;
template <typename T, int G, typename Args>
__device__ __forceinline__ void join(const Args& a, const KvUnit& unit, int h, int c1, int pieces, int block, int blocks,
                                     int thread) {
  const int n_rows = unit.tokens * a.group, full_rows = a.tile_tokens * a.group;
  constexpr int P = 2;
  const int n = n_rows * (a.D / 16), g = thread % G, step = blocks * (kJoinThreads / G);
  for (int x = block * (kJoinThreads / G) + thread / G; x - (thread % 32) / G < n; x += step) {
    const int column = min(x, n - 1) / n_rows, r = min(x, n - 1) - column * n_rows;
    const int tile = r >= full_rows, row = r - tile * full_rows;
    Joined s;
    for (int i0 = g; i0 < pieces; i0 += P * G) {
      float2 ml[P];
      float4 p[P][4];
#pragma unroll
      for (int k = 0; k < P; ++k) {
        const int i = i0 + k * G;
        if (i >= pieces) continue;
        const int64_t slot = 2 * ((int64_t)c1 + i) + (i == 0);
        ml[k] = a.part_ml[slot * 2 * kTile + tile * kTile + row];
        const float4* from = reinterpret_cast<const float4*>(a.part) + part_at(a.D, slot, tile, 4 * column) + row;
#pragma unroll
        for (int q = 0; q < 4; ++q) p[k][q] = from[q * kTile];
      }
#pragma unroll
      for (int k = 0; k < P; ++k)
        if (i0 + k * G < pieces) s.add(ml[k].x, ml[k].y, p[k]);
    }
    // The G threads' sums: their exponents to the largest, then in pairs, each of
    // a pair going on with half of the elements: 15 to 16 exchanges of elements
    // instead of 16 a step, and the stores spread over the threads (18.6 us against
    // 19.3 for single tokens of 19 sequences of up to 900 keys, 192 against 196 for
    // chunks in a window).
    float top = s.top;
#pragma unroll
    for (int o = 1; o < G; o <<= 1) top = fmaxf(top, __shfl_xor_sync(0xffffffffu, top, o));
    const float f = s.top == -INFINITY ? 0.f : ex2(s.top - top);
    float l = s.l * f, v[16];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      v[4 * q] = s.o[q].x * f, v[4 * q + 1] = s.o[q].y * f, v[4 * q + 2] = s.o[q].z * f, v[4 * q + 3] = s.o[q].w * f;
    int first = 0;  // of the elements that the thread has
#pragma unroll
    for (int o = 1; o < G; o <<= 1) {
      l += __shfl_xor_sync(0xffffffffu, l, o);
      const bool high = g & o;
      const int m = 8 / o;  // elements to go on with
      if (m > 0) {
#pragma unroll
        for (int i = 0; i < m; ++i) v[i] = (high ? v[i + m] : v[i]) + __shfl_xor_sync(0xffffffffu, high ? v[i] : v[i + m], o);
        first += high ? m : 0;
      } else {
        v[0] += __shfl_xor_sync(0xffffffffu, v[0], o);
      }
    }
    if (x >= n) continue;
    const float inv = (l > 0.f ? 1.f / l : l) * a.v_scale;  // (NaN stays)
    const int64_t token = unit.token + r / a.group;
    const int head = h * a.group + r % a.group;
    T* out = static_cast<T*>(a.out.d_data) + token * a.out.token_stride + head * a.out.head_stride + 16 * column;
    if constexpr (G == 1) {
      uint32_t y[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) y[q] = Type<T>::pack(v[2 * q] * inv, v[2 * q + 1] * inv);
      store16(a.wide, out, y);
    } else if constexpr (G <= 8) {
#pragma unroll
      for (int q = 0; q < 8 / G; ++q)
        reinterpret_cast<uint32_t*>(out + first)[q] = Type<T>::pack(v[2 * q] * inv, v[2 * q + 1] * inv);
    } else if (g < 16) {
      // (element 0 is the low half)
      reinterpret_cast<uint16_t*>(out)[first] = (uint16_t)Type<T>::pack(v[0] * inv, 0.f);
    }
    if (a.lse && column == 0 && g == 0)
      a.lse[token * a.hq + head] = l == 0.f ? -INFINITY : (top + log2f(l)) * 0.6931471805599453f;
  }
}

// Pieces of every shared unit, by blocks in turn for the units, so that one such unit (a
// chunk over a long sequence: 9 MB of pieces) has them all. `share` and `c1` are of the
// block's unit.
template <typename T, typename Args>
__device__ __forceinline__ void join_unit(const Args& a, const KvShare& share, int c1, int block, int blocks, int thread) {
  // Chunks have two or three pieces of many rows, single tokens many of few.
  if (share.n_last <= 4)
    join<T, 1>(a, share.last, share.h1, c1, share.n_last, block, blocks, thread);
  else if (share.n_last <= 16)
    join<T, 8>(a, share.last, share.h1, c1, share.n_last, block, blocks, thread);
  else
    join<T, 32>(a, share.last, share.h1, c1, share.n_last, block, blocks, thread);
}

}  // namespace smetric
