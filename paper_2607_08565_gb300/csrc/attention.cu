// Attention of a planned batch's queries over the paged cache.
//
//   k_paged_attention  one CTA an SM, each with the share of the batch that the
//                      plan gave it.
//   k_paged_join       joins the pieces of the units that several CTAs share.
//
// For a tile of 128 query rows (a row is a token and one of the query heads of
// a key head) and a tile of 128 keys: S = Q K^T and O += P V on the tensor
// cores (tcgen05, sums in TMEM), P = exp2(c S - ref) in between, c = scale *
// log2(e). ref is the row's reference exponent: its largest c S when it was
// last moved. It moves only when a score exceeds it by 2^kSlack, since a common
// factor of P and its sum l cancels in O / l: so O is seldom rescaled.
//
// Two query tiles are in flight, so that one's softmax runs while the tensor
// cores work on the other: a unit of more than 128 rows has its two halves
// (both read the same keys), a smaller one has the even and the odd key tiles
// of its rows, whose sums are joined at the end.
//
// Warps: 0 and 2 copy tiles with TMA (keys and values alternate in one ring of
// buffers, query tiles in one of two), 1 issues the matrix products, 3 writes
// zeros for tokens of no request, 4-7 and 8-11 are the two tiles' softmax (a
// thread a row), 12-15 write a unit's output while the softmax of the next one
// runs.
//
// Scores, statistics, sums and the join are in 32 bits. P is rounded to the
// type of the values, as the tensor cores multiply operands of one type of 16
// bits (its sum l is taken before that): against 64 bits the output's error is
// 1.2 to 1.5 times that of its own rounding.
//
// Single tokens are bound by memory: 64 of them over 2k to 48k keys (4 key heads
// of 128, 3.2 GB) take 464 us, 6.9 TB/s, the rate of a copy. Chunks are bound by
// the power cap and by the chain of a tile's softmax (1,300 cycles), its product
// with the values and its half's next scores (2 x 512 on the tensor cores), 2,840
// cycles for two query tiles and a key tile: 2,048 tokens over 65,000 (32 query
// heads) take 1,566 us, 1,415 TFLOP/s, with the cap, and 1,360 to 1,440 us in
// runs too short for it. A thread spills 108 bytes and loads 152 (of all roles:
// 60 and 56 without the softmax, 88 and 120 without the issuing warp).

#include <cuda.h>
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
#include "tensor_map.cuh"

using namespace smetric;

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr long long kWaitCycles = 1ll << 32;  // bounded mbarrier waits: about 2 s
constexpr uint32_t kNap = 20000;  // ns that a waiting warp sleeps between looks at most
constexpr int kThreads = 512;
constexpr float kSlack = 8.f;     // log2 of how far scores may pass the reference
constexpr uint32_t kHalf = 16384;  // bytes of 128 rows of 64 elements

// Buffers of the ring: what 227 KB hold beside the two query tiles.
__host__ __device__ constexpr int stages(int halves) { return halves == 2 ? 5 : 11; }

struct AttentionArgs {
  CUtensorMap q, k, v;
  smetric_heads out;
  float* lse;
  const KvPlan* plan;
  const KvUnit* units;
  const KvShare* shares;
  const int32_t* split;
  float* part;
  float2* part_ml;
  const int32_t* pages;
  int64_t pages_stride, n_tokens;
  int32_t num_pages, hq, kv_heads, group, tile_tokens, D, page_size, window;
  float scale;
  bool wide;  // outputs can be stored in pieces of 32 bytes
  int32_t* status;
};

// ---- shared memory, TMA, tensor cores ----

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }

struct __align__(8) Barriers {
  uint64_t full[11], empty[11];   // the ring's
  uint64_t q_full[2], q_empty[2];
  uint64_t s_full[2];  // scores in TMEM (and the products before them done)
  uint64_t p_full[2];  // weights in TMEM, O rescaled
  uint64_t o_full[2];  // the unit's last product with the values done
  uint64_t o_free[2];  // its sums and statistics read
  uint64_t stat_full[2];
  uint64_t drain;
};

struct Shared {
  Barriers bar;
  float2 stat[2][kTile];  // a unit's (reference exponent, sum of weights), rows of the two tiles
  uint32_t tmem;
  int32_t abort;          // a wait ran out: everybody stops waiting
};

__device__ __forceinline__ void mbar_init(uint64_t* b, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;\n" ::"r"(smem_u32(b)), "r"(count) : "memory");
}
__device__ __forceinline__ void mbar_arrive(uint64_t* b) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];\n" ::"r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void mbar_expect(uint64_t* b, uint32_t bytes) {
  asm volatile("mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n" ::"r"(smem_u32(b)), "r"(bytes) : "memory");
}
// One try for the phase of the given parity, asleep for up to kNap ns: four
// warps that only polled for a unit's end took a tenth of the softmax's speed.
__device__ __forceinline__ bool mbar_try(uint64_t* b, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2, %3;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(done) : "r"(smem_u32(b)), "r"(parity), "r"(kNap) : "memory");
  return done != 0;
}
// One look.
__device__ __forceinline__ bool mbar_test(uint64_t* b, uint32_t parity) {
  uint32_t done;
  asm volatile(
      "{\n .reg .pred p;\n mbarrier.test_wait.parity.shared::cta.b64 p, [%1], %2;\n selp.u32 %0, 1, 0, p;\n}\n"
      : "=r"(done) : "r"(smem_u32(b)), "r"(parity) : "memory");
  return done != 0;
}
// Whether a wait of the CTA has run out. The warp votes: its lanes may read the
// flag before and after another warp sets it, and have to go the same way.
__device__ __forceinline__ bool stopped(const Shared* sh) {
  return __any_sync(kFull, *(const volatile int32_t*)&sh->abort != 0);
}
// The warp waits for the phase of the given parity; gives up after kWaitCycles,
// or when another wait of the CTA has. Callers go on either way (every loop is
// bounded by the plan); outputs are then undefined and the error is latched.
__device__ __forceinline__ void mbar_wait(uint64_t* b, uint32_t parity, Shared* sh, int32_t* status) {
  if (!mbar_test(b, parity)) {
    const long long start = clock64();
    while (!mbar_try(b, parity)) {
      if (*(const volatile int32_t*)&sh->abort != 0) break;
      if (clock64() - start > kWaitCycles) {
        *(volatile int32_t*)&sh->abort = 1;
        latch_error(status, SMETRIC_ERR_CUDA);
        break;
      }
    }
  }
  __syncwarp();
}
// The same for the products in flight when the CTA gives up.
__device__ __forceinline__ void mbar_drain(uint64_t* b, uint32_t parity) {
  const long long start = clock64();
  while (!mbar_try(b, parity) && clock64() - start < kWaitCycles) {
  }
}

__device__ __forceinline__ void tma_3d(uint32_t dst, const CUtensorMap* m, int32_t x, int32_t y, int32_t z, uint64_t* b) {
  asm volatile(
      "cp.async.bulk.tensor.3d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4}], [%5];\n" ::
          "r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z), "r"(smem_u32(b)) : "memory");
}
__device__ __forceinline__ void tma_4d(uint32_t dst, const CUtensorMap* m, int32_t x, int32_t y, int32_t z, int32_t w,
                                       uint64_t* b) {
  asm volatile(
      "cp.async.bulk.tensor.4d.shared::cluster.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3, %4, %5}],"
      " [%6];\n" ::"r"(dst), "l"(reinterpret_cast<uint64_t>(m)), "r"(x), "r"(y), "r"(z), "r"(w), "r"(smem_u32(b))
      : "memory");
}

// One lane of a converged warp, the same one each time. (Under a condition on
// the lane number the compiler cannot tell that one thread issues, and a matrix
// product took 120 cycles to issue.)
__device__ __forceinline__ bool elect() {
  uint32_t p;
  asm volatile("{\n .reg .pred p;\n elect.sync _|p, 0xffffffff;\n selp.u32 %0, 1, 0, p;\n}\n" : "=r"(p) : : "memory");
  return p != 0;
}

// Shared-memory descriptors of operands in rows of 128 bytes with the 128-byte
// swizzle: groups of 8 rows 1,024 bytes apart (the high half says that). The
// low half has the address in units of 16 bytes and lbo, the bytes between the
// 64-element halves where the rows run along the product's inner dimension
// (the values).
constexpr uint32_t kDescHigh = 1024 >> 4 | 1u << 14 | 2u << 29;
__device__ __forceinline__ uint32_t desc_low(uint32_t addr, uint32_t lbo) {
  return (addr & 0x3ffff) >> 4 | lbo >> 4 << 16;
}
__device__ __forceinline__ void mma_ss(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 a, b;\n setp.ne.u32 p, %4, 0;\n mov.b64 a, {%1, %5};\n mov.b64 b, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], a, b, %3, p;\n}\n" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(add),
      "n"(kDescHigh) : "memory");
}
__device__ __forceinline__ void mma_ts(uint32_t d, uint32_t a, uint32_t b, uint32_t idesc, uint32_t add) {
  asm volatile(
      "{\n .reg .pred p;\n .reg .b64 b;\n setp.ne.u32 p, %4, 0;\n mov.b64 b, {%2, %5};\n"
      " tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], b, %3, p;\n}\n" ::"r"(d), "r"(a), "r"(b), "r"(idesc), "r"(add),
      "n"(kDescHigh) : "memory");
}
__device__ __forceinline__ void zero16(uint32_t addr) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %1, %1, %1};\n" ::"r"(addr), "r"(0) : "memory");
}
// Arrives at b when the products issued so far are done.
__device__ __forceinline__ void mma_commit(uint64_t* b) {
  asm volatile("tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n" ::"r"(smem_u32(b))
               : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;\n" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;\n" ::: "memory"); }
// Waits for the warp's loads from TMEM; their registers are read after it.
template <int N>
__device__ __forceinline__ void wait_ld(uint32_t (&r)[N]) {
  asm volatile("tcgen05.wait::ld.sync.aligned;\n" ::: "memory");
#pragma unroll
  for (int i = 0; i < N; ++i) asm volatile("" : "+r"(r[i]));
}
__device__ __forceinline__ void wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;\n" ::: "memory"); }

// 32 columns of the warp's 32 lanes (a row a thread).
__device__ __forceinline__ void tmem_ld32(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]), "=r"(r[16]),
        "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]), "=r"(r[24]),
        "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_ld16(uint32_t addr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x16.b32 {%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15}, "
      "[%16];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]), "=r"(r[8]),
        "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15])
      : "r"(addr) : "memory");
}
__device__ __forceinline__ void tmem_st16(uint32_t addr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x16.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16};\n" ::"r"(addr), "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
      "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]) : "memory");
}

__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;\n" : "=f"(y) : "f"(x));
  return y;
}

__device__ __forceinline__ float max3(float x, float y, float z) {
  float m;
  asm("max.f32 %0, %1, %2, %3;\n" : "=f"(m) : "f"(x), "f"(y), "f"(z));
  return m;
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

// ---- a CTA's share ----

struct Item {
  KvUnit unit;
  int32_t h, tb, te;  // key head, its key tiles in this CTA
  bool whole;         // nobody else has key tiles of it
  bool pair;          // two query tiles (else the even and the odd key tiles)
  int32_t slot;       // of its partial sums, where !whole
};

struct Walk {
  KvUnit unit;  // the next item's
  int32_t u, h, t0, u1, h1, t1;
  bool first, done;
  __device__ __forceinline__ void load(const KvUnit* p) {
    const int4 x = reinterpret_cast<const int4*>(p)[0];
    const int2 y = reinterpret_cast<const int2*>(p)[2];
    unit.token = x.x, unit.tokens = x.y, unit.pos = x.z, unit.req = x.w, unit.tb = y.x, unit.te = y.y;
  }
  __device__ __forceinline__ void start(const AttentionArgs& a) {
    const KvShare* s = a.shares + blockIdx.x;
    const int4 x = reinterpret_cast<const int4*>(s)[0];
    const int2 y = reinterpret_cast<const int2*>(s)[2];
    load(&s->first);
    u = x.x, h = x.y, t0 = x.z, u1 = x.w, h1 = y.x, t1 = y.y;
    first = true;
    done = u < 0;
  }
  __device__ __forceinline__ bool next(const AttentionArgs& a, Item& it) {
    if (done) return false;
    const bool last = u == u1 && h == h1;
    it.unit = unit;
    it.h = h;
    it.tb = first ? t0 : unit.tb;
    it.te = last ? t1 : unit.te;
    it.pair = unit.tokens > a.tile_tokens;
    it.whole = it.tb == unit.tb && it.te == unit.te;
    it.slot = 2 * (int32_t)blockIdx.x + (it.tb == unit.tb);
    first = false;
    done = last;
    if (++h == a.kv_heads && !done) {
      h = 0;
      load(a.units + ++u);  // (ahead of its use)
    }
    return true;
  }
};

// Partial sums: a slot's two query tiles, each D/4 columns of kTile rows of four
// sums, so that the threads of a warp (a row each) store in whole lines. The
// place of a column's first row, in units of four sums.
__device__ __forceinline__ int64_t part_at(int D, int64_t slot, int tile, int column) {
  return ((slot * 2 + tile) * (D / 4) + column) * kTile;
}

// Places of an item's tiles in the ring, of n key tiles: K0 K1 V0 K2 V1 K3 ...
__device__ __forceinline__ uint32_t place_k(int j) { return j < 2 ? j : 2 * j - 1; }
__device__ __forceinline__ uint32_t place_v(int j, int n) { return min(2 + 2 * j, 2 * n - 1); }

// ---- the warps ----

// One warp copies the query tiles and the keys, another the values (a tile of
// 16-token pages is 16 copies, and one warp issues them no faster than memory
// delivers half of them). A lane has a page and a half of the elements.
template <int HALVES>
__device__ __forceinline__ void copy_tiles(const AttentionArgs& a, Shared* sh, Walk w, uint32_t q_smem, uint32_t ring,
                                           const bool values) {
  constexpr int S = stages(HALVES);
  Barriers& b = sh->bar;
  const int lane = threadIdx.x & 31;
  const int rows = min(kTile, a.page_size), per = kTile / rows;  // of a copy, and pages of a tile
  const int page_shift = __ffs(a.page_size) - 1;
  const int mine = lane % per, half = lane / per;
  const bool copies = half < HALVES;
  const uint32_t q_bytes = (uint32_t)a.tile_tokens * a.group * 128 * HALVES;
  const CUtensorMap* const map = values ? &a.v : &a.k;
  uint32_t base = 0, nq = 0;
  Item it;
  while (w.next(a, it)) {
    const int n = it.te - it.tb;
    // the keys that some query of the unit sees
    const int32_t lo = it.unit.pos >= a.window ? it.unit.pos - a.window + 1 : 0, hi = it.unit.pos + it.unit.tokens;
    const int32_t* pages = a.pages + it.unit.req * a.pages_stride;
    // the lane's page of a tile, INT32_MIN where nobody sees a key of it
    const auto page_of = [&](int j) {
      const int64_t key = (int64_t)(it.tb + j) * kTile + mine * rows;
      return copies && j < n && key < hi && key + rows > lo ? pages[key >> page_shift] : INT32_MIN;
    };
    int32_t next = page_of(0);
    for (int j = 0; j < n; ++j) {
      int32_t page = next;
      next = page_of(j + 1);
      const uint32_t at = base + (values ? place_v(j, n) : place_k(j)), s = at % S;
      if (at >= S) mbar_wait(&b.empty[s], (at / S - 1) & 1, sh, a.status);
      if (stopped(sh)) break;
      const bool held = page != INT32_MIN;
      const unsigned who = __ballot_sync(kFull, held);
      if (lane == 0) mbar_expect(&b.full[s], __popc(who) * rows * 128);
      __syncwarp();
      if (held) {
        if (page < 0 || page >= a.num_pages) {
          latch_error(a.status, SMETRIC_ERR_INVALID_ARG);
          page = a.num_pages;  // outside the tensor map: zeros
        }
        tma_4d(ring + (s * HALVES + half) * kHalf + mine * rows * 128, map, 64 * half,
               a.page_size > kTile ? (it.tb + j) * kTile % a.page_size : 0, it.h, page, &b.full[s]);
      }
      if (j == 0 && !values) {
        for (int t = 0; t < (it.pair ? 2 : 1); ++t, ++nq) {
          uint64_t* full = &b.q_full[nq & 1];
          if (nq > 1) mbar_wait(&b.q_empty[nq & 1], (nq / 2 - 1) & 1, sh, a.status);
          const bool stop = stopped(sh);
          if (lane == 0 && !stop) {
            mbar_expect(full, q_bytes);
#pragma unroll
            for (int e = 0; e < HALVES; ++e)
              tma_3d(q_smem + ((nq & 1) * HALVES + e) * kHalf, &a.q, 64 * e, it.h * a.group,
                     it.unit.token + t * a.tile_tokens, full);
          }
          __syncwarp();
        }
      }
    }
    base += 2 * n;
    if (stopped(sh)) break;
  }
}

// Issues the products, a step's (weights with values, then the half's next
// scores) by one elected lane in one go: this warp is close to the limit, a wait
// that is ready costs it 60 to 160 cycles. The two halves take turns.
template <typename T, int HALVES>
__device__ __forceinline__ void multiply(const AttentionArgs& a, Shared* sh, Walk w, uint32_t q_smem, uint32_t ring) {
  constexpr int S = stages(HALVES);
  Barriers& b = sh->bar;
  const int lane = threadIdx.x & 31;
  const uint32_t tmem = sh->tmem;
  constexpr uint32_t kType = 1u << 4 | Type<T>::kFormat << 7 | Type<T>::kFormat << 10 | (kTile >> 4) << 24;
  constexpr uint32_t kScores = kType | (kTile >> 3) << 17;
  const uint32_t values = kType | 1u << 16 | (uint32_t)(a.D >> 3) << 17;
  const int steps = a.D / 16;
  // (an operand's address is the descriptor's low bits, in units of 16 bytes)
  const uint32_t q_desc = desc_low(q_smem, 16), k_desc = desc_low(ring, 16), v_desc = desc_low(ring, kHalf);
  uint32_t base = 0, items = 0, nq = 0, np[2] = {0, 0};
  Item it;
  for (; w.next(a, it); ++items) {
    const int n = it.te - it.tb;
    const int32_t lo = it.unit.pos >= a.window ? it.unit.pos - a.window + 1 : 0, hi = it.unit.pos + it.unit.tokens;
    const auto stage = [&](uint32_t place) { return (base + place) % S; };
    const auto wait_full = [&](uint32_t place) {
      mbar_wait(&b.full[stage(place)], (base + place) / S & 1, sh, a.status);
    };
    const auto wait_q = [&](uint32_t i) { mbar_wait(&b.q_full[i & 1], i / 2 & 1, sh, a.status); };
    const auto release_q = [&](uint32_t i) {
      if (elect()) mma_commit(&b.q_empty[i & 1]);
    };
    // (one elected lane, from here to the commit)
    const auto issue_scores = [&](int t, uint32_t q, uint32_t at) {  // S_t = Q_q K^T
      const uint32_t qd = q_desc + (q & 1) * (HALVES * kHalf >> 4), kd = k_desc + at * (HALVES * kHalf >> 4);
#pragma unroll
      for (int k = 0; k < 4 * HALVES; ++k) {
        const uint32_t o = ((k >> 2) * kHalf + (k & 3) * 32) >> 4;
        if (k < steps) mma_ss(tmem + t * kTile, qd + o, kd + o, kScores, k > 0);
      }
      mma_commit(&b.s_full[t]);
    };
    const auto issue_products = [&](int t, uint32_t at, bool add) {  // O_t (+)= P_t V
      const uint32_t vd = v_desc + at * (HALVES * kHalf >> 4);
#pragma unroll
      for (int k = 0; k < kTile / 16; ++k)
        mma_ts(tmem + 2 * kTile + t * kTile, tmem + t * kTile + 8 * k, vd + k * (2048 >> 4), values, add || k > 0);
    };
    const auto wait_weights = [&](int t, bool first) {
      if (first && items) mbar_wait(&b.o_free[t], (items - 1) & 1, sh, a.status);
      mbar_wait(&b.p_full[t], np[t]++ & 1, sh, a.status);
      fence_after();
    };
    // Rows of a tile's values that no key lies at become zeros: a weight of
    // zero does not cancel what may lie there. (A row's 128 bytes are its own
    // under the swizzle.)
    const auto clear = [&](uint32_t place, int j) {
      const int32_t key = (it.tb + j) * kTile;
      if (key >= lo && hi - key >= kTile) return;  // (key + kTile may pass 32 bits)
      const uint32_t at = ring + stage(place) * HALVES * kHalf;
      const int before = max(lo - key, 0), after = min(hi - key, kTile);
#pragma unroll
      for (int e = 0; e < HALVES; ++e) {
        for (int i = lane * 16; i < before * 128; i += 512) zero16(at + e * kHalf + i);
        for (int i = after * 128 + lane * 16; i < kTile * 128; i += 512) zero16(at + e * kHalf + i);
      }
      asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
      __syncwarp();
    };
    wait_full(0);
    wait_q(nq);
    if (stopped(sh)) break;
    fence_after();
    if (it.pair) {
      if (elect()) issue_scores(0, nq, stage(0));
      wait_q(nq + 1);
      if (elect()) {
        issue_scores(1, nq + 1, stage(0));
        mma_commit(&b.empty[stage(0)]);
      }
      for (int j = 0; j + 1 < n; ++j) {
        const uint32_t v = place_v(j, n), k = place_k(j + 1), vs = stage(v), ks = stage(k);
        wait_full(v);
        if (j == 0) clear(v, j);
        wait_full(k);
        wait_weights(0, j == 0);
        if (elect()) {
          issue_products(0, vs, j > 0);
          issue_scores(0, nq, ks);
        }
        wait_weights(1, j == 0);
        if (elect()) {
          issue_products(1, vs, j > 0);
          mma_commit(&b.empty[vs]);
          issue_scores(1, nq + 1, ks);
          mma_commit(&b.empty[ks]);
        }
      }
      release_q(nq), release_q(nq + 1);
      const uint32_t v = place_v(n - 1, n), vs = stage(v);
      wait_full(v);
      clear(v, n - 1);
      wait_weights(0, n == 1);
      if (elect()) {
        issue_products(0, vs, n > 1);
        mma_commit(&b.o_full[0]);
      }
      wait_weights(1, n == 1);
      if (elect()) {
        issue_products(1, vs, n > 1);
        mma_commit(&b.o_full[1]);
        mma_commit(&b.empty[vs]);
      }
      nq += 2;
    } else {
      for (int j = 0; j < min(n, 2); ++j) {
        if (j) wait_full(j);
        if (elect()) {
          issue_scores(j, nq, stage(j));
          mma_commit(&b.empty[stage(j)]);
        }
      }
      if (n <= 2) release_q(nq);
      // (waited for by every unit, so that no two have one parity, and before the
      // product that lets the unit's own phase end)
      if (n == 1 && items) mbar_wait(&b.o_free[1], (items - 1) & 1, sh, a.status);
      for (int j = 0; j < n; ++j) {
        const int t = j & 1;
        const bool more = j + 2 < n;
        const uint32_t v = place_v(j, n), k = place_k(j + 2), vs = stage(v), ks = stage(k);
        wait_full(v);
        clear(v, j);
        if (more) wait_full(k);
        wait_weights(t, j < 2);
        if (elect()) {
          issue_products(t, vs, j > 1);
          mma_commit(&b.empty[vs]);
          if (more) {
            issue_scores(t, nq, ks);
            mma_commit(&b.empty[ks]);
            if (j + 3 == n) mma_commit(&b.q_empty[nq & 1]);
          } else {
            mma_commit(&b.o_full[t]);
          }
        }
      }
      nq += 1;
    }
    base += 2 * n;
    __syncwarp();
  }
  if (stopped(sh)) {  // products in flight must end before the CTA's memory goes
    if (elect()) mma_commit(&b.drain);
    mbar_drain(&b.drain, 0);
    __syncwarp();
  }
}

// 16 elements of an output.
__device__ __forceinline__ void store16(const AttentionArgs& a, void* p, const uint32_t* r) {
  if (a.wide) {
    asm volatile("st.global.v8.b32 [%0], {%1, %2, %3, %4, %5, %6, %7, %8};\n" ::"l"(p), "r"(r[0]), "r"(r[1]), "r"(r[2]),
                 "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]) : "memory");
  } else {
    static_cast<uint4*>(p)[0] = make_uint4(r[0], r[1], r[2], r[3]);
    static_cast<uint4*>(p)[1] = make_uint4(r[4], r[5], r[6], r[7]);
  }
}

// A tile's first token in its unit, and its rows.
__device__ __forceinline__ int tile_token(const AttentionArgs& a, const Item& it, int tile) {
  return it.pair ? tile * a.tile_tokens : 0;
}
__device__ __forceinline__ int tile_rows(const AttentionArgs& a, const Item& it, int tile) {
  return min(a.tile_tokens, it.unit.tokens - tile_token(a, it, tile)) * a.group;
}

// The lowest n bits, none or all where n is outside 0..32.
__device__ __forceinline__ uint32_t below(int32_t n) { return n <= 0 ? 0 : n >= 32 ? kFull : (1u << n) - 1; }

// (One code for both tiles: two copies miss the instruction cache.)
template <typename T>
__device__ __forceinline__ void softmax(const AttentionArgs& a, Shared* sh, Walk w, const int tile) {
  Barriers& b = sh->bar;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5 & 3, row = threadIdx.x & 127;
  const uint32_t lanes = (uint32_t)warp << 21;  // the warp's TMEM lanes
  const uint32_t s_at = sh->tmem + tile * kTile + lanes, o_at = sh->tmem + 2 * kTile + tile * kTile + lanes;
  const int row_token = row / a.group;
  const float c = a.scale * 1.4426950408889634f;
  uint32_t ns = 0, items = 0;
  Item it;
  for (; w.next(a, it); ++items) {
    const int n = it.te - it.tb;
    const int n_rows = tile_rows(a, it, tile);
    const bool mine = row < n_rows;
    const int32_t hi = mine ? it.unit.pos + tile_token(a, it, tile) + row_token : INT32_MAX / 2;  // last key that the row sees
    const int32_t lo = mine && hi >= a.window ? hi - a.window + 1 : 0;                        // first key
    const bool busy = 32 * warp < n_rows;
    // every row of the warp sees all keys of [all_lo, all_hi]
    const int32_t all_lo = __reduce_max_sync(kFull, lo), all_hi = __reduce_min_sync(kFull, hi);
    float top = -INFINITY;  // largest score when the reference was last moved
    float ref = 0.f;        // the reference exponent: c * top - kLift (0 before the first visible key)
    float l = 0.f;
    for (int j = it.pair ? 0 : tile; j < n; j += it.pair ? 1 : 2) {
      mbar_wait(&b.s_full[tile], ns++ & 1, sh, a.status);
      if (!busy) {
        __syncwarp();
        if (lane == 0) mbar_arrive(&b.p_full[tile]);
        continue;
      }
      fence_after();
      uint32_t r[kTile];
#pragma unroll
      for (int i = 0; i < 4; ++i) tmem_ld32(s_at + 32 * i, r + 32 * i);
      wait_ld(r);
      float s[kTile];
#pragma unroll
      for (int i = 0; i < kTile; ++i) s[i] = __uint_as_float(r[i]);
      const int32_t key = (it.tb + j) * kTile;
      if (key + kTile - 1 > all_hi || key < all_lo) {
#pragma unroll
        for (int i = 0; i < kTile; i += 32) {  // a bit a column
          const uint32_t seen = below(hi + 1 - (key + i)) & ~below(lo - (key + i));
#pragma unroll
          for (int k = 0; k < 32; ++k) s[i + k] = seen & 1u << k ? s[i + k] : -INFINITY;
        }
      }
      float m[8];
#pragma unroll
      for (int i = 0; i < 8; ++i) m[i] = s[i];
#pragma unroll
      for (int i = 8; i < kTile; i += 16)
#pragma unroll
        for (int k = 0; k < 8; ++k) m[k] = i + 8 + k < kTile ? max3(m[k], s[i + k], s[i + 8 + k]) : fmaxf(m[k], s[i + k]);
      const float most = max3(max3(m[0], m[1], m[2]), max3(m[3], m[4], m[5]), fmaxf(m[6], m[7]));
      const bool move = (most - top) * c > kSlack;  // (false for -inf - -inf)
      if (__any_sync(kFull, move)) {
        float back = 1.f;
        if (move) {
          const float next = most * c - Type<T>::kLift;
          back = top == -INFINITY ? 0.f : ex2(ref - next);
          top = most;
          ref = next;
          l *= back;
        }
        if (j > (it.pair ? 0 : tile)) {
          for (int d = 0; d < a.D; d += 16) {
            uint32_t o[16];
            tmem_ld16(o_at + d, o);
            wait_ld(o);
#pragma unroll
            for (int i = 0; i < 16; ++i) o[i] = __float_as_uint(__uint_as_float(o[i]) * back);
            tmem_st16(o_at + d, o);
          }
        }
      }
      float2 sum[4] = {};
      const float2 c2 = make_float2(c, c), ref2 = make_float2(-ref, -ref);
#pragma unroll
      for (int i = 0; i < kTile; i += 32) {
        uint32_t p[16];
#pragma unroll
        for (int k = 0; k < 16; ++k) {
          float2 x = fma2(make_float2(s[i + 2 * k], s[i + 2 * k + 1]), c2, ref2);
          x = make_float2(ex2(x.x), ex2(x.y));
          sum[k & 3] = add2(sum[k & 3], x);
          p[k] = Type<T>::pack(x.x, x.y);
        }
        tmem_st16(s_at + i / 2, p);
      }
      wait_st();
      fence_before();
      __syncwarp();
      if (lane == 0) mbar_arrive(&b.p_full[tile]);
      const float2 all = add2(add2(sum[0], sum[1]), add2(sum[2], sum[3]));
      l += all.x + all.y;
    }
    if (items) mbar_wait(&b.o_free[tile], (items - 1) & 1, sh, a.status);
    // (scores that are all NaN leave top where it was, but not l: the row is not
    // one without keys, and what joins its pieces must not pass over it)
    sh->stat[tile][row] = make_float2(top == -INFINITY && l == 0.f ? -INFINITY : ref, l);
    __syncwarp();
    if (lane == 0) mbar_arrive(&b.stat_full[tile]);
  }
}

// A unit's output: O / l, or its sums and statistics where other CTAs have
// pieces of it.
template <typename T>
__device__ __forceinline__ void write_out(const AttentionArgs& a, Shared* sh, Walk w) {
  Barriers& b = sh->bar;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5 & 3, row = threadIdx.x & 127;
  const uint32_t o_all = sh->tmem + 2 * kTile + ((uint32_t)warp << 21);
  const int row_token = row / a.group, row_head = row - row_token * a.group;
  uint32_t items = 0, no[2] = {0, 0};
  Item it;
  for (; w.next(a, it); ++items) {
    const bool two = !it.pair && it.te - it.tb > 1;  // sums of even and of odd key tiles
    for (int tile = 0; tile < (it.pair ? 2 : 1); ++tile) {
      const int n_rows = tile_rows(a, it, tile);
      mbar_wait(&b.stat_full[tile], items & 1, sh, a.status);
      float2 st = sh->stat[tile][row];
      float w1 = 1.f, w2 = 0.f;  // the even and the odd tiles' shares
      if (!it.pair) {
        mbar_wait(&b.stat_full[1], items & 1, sh, a.status);
        const float2 odd = sh->stat[1][row];
        const float both = fmaxf(st.x, odd.x);
        if (both > -INFINITY) {
          w1 = ex2(st.x - both);
          w2 = ex2(odd.x - both);
          st = make_float2(both, st.y * w1 + odd.y * w2);
        }
        if (two) mbar_wait(&b.o_full[1], no[1]++ & 1, sh, a.status);
      }
      mbar_wait(&b.o_full[tile], no[tile]++ & 1, sh, a.status);
      if (32 * warp < n_rows) {
        fence_after();
        const bool mine = row < n_rows;
        const int64_t token = it.unit.token + tile_token(a, it, tile) + row_token;
        const int head = it.h * a.group + row_head;
        const float inv = it.whole ? (st.y > 0.f ? 1.f / st.y : st.y) : 1.f;  // (NaN stays)
        w1 *= inv, w2 *= inv;
        const uint32_t o_at = o_all + tile * kTile;
        T* out = static_cast<T*>(a.out.d_data) + token * a.out.token_stride + head * a.out.head_stride;
        for (int d = 0; d < a.D; d += 16) {
          uint32_t o[16];
          float f[16];
          tmem_ld16(o_at + d, o);
          wait_ld(o);
#pragma unroll
          for (int i = 0; i < 16; ++i) f[i] = __uint_as_float(o[i]) * w1;
          if (two) {
            tmem_ld16(o_at + kTile + d, o);
            wait_ld(o);
#pragma unroll
            for (int i = 0; i < 16; ++i) f[i] += __uint_as_float(o[i]) * w2;
          }
          if (mine) {
            if (it.whole) {
              uint32_t y[8];
#pragma unroll
              for (int i = 0; i < 8; ++i) y[i] = Type<T>::pack(f[2 * i], f[2 * i + 1]);
              store16(a, out + d, y);
            } else {
              float4* p = reinterpret_cast<float4*>(a.part) + part_at(a.D, it.slot, tile, d / 4) + row;
#pragma unroll
              for (int i = 0; i < 4; ++i)
                p[i * kTile] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
            }
          }
        }
        fence_before();
        if (mine) {
          if (!it.whole)
            a.part_ml[(int64_t)it.slot * 2 * kTile + tile * kTile + row] = st;
          else if (a.lse)
            a.lse[token * a.hq + head] = st.y == 0.f ? -INFINITY : (st.x + log2f(st.y)) * 0.6931471805599453f;
        }
      }
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&b.o_free[tile]);
        if (!it.pair) mbar_arrive(&b.o_free[1]);
      }
    }
  }
}

template <typename T, int HALVES>
__global__ void __launch_bounds__(kThreads, 1) k_paged_attention(const __grid_constant__ AttentionArgs a) {
  constexpr int S = stages(HALVES);
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  Shared* sh = reinterpret_cast<Shared*>(smem_raw + (2 + S) * HALVES * kHalf);
  if (smem_u32(smem_raw) & 1023) {  // (the swizzle's groups of 8 rows)
    latch_error(a.status, SMETRIC_ERR_CUDA);
    return;
  }
  const uint32_t q_smem = smem_u32(smem_raw), ring = q_smem + 2 * HALVES * kHalf;
  const int warp = threadIdx.x >> 5;
  if (threadIdx.x == 0) {
    Barriers& b = sh->bar;
    for (int i = 0; i < S; ++i) mbar_init(&b.full[i], 1), mbar_init(&b.empty[i], 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&b.q_full[t], 1);
      mbar_init(&b.q_empty[t], 1);
      mbar_init(&b.s_full[t], 1);
      mbar_init(&b.p_full[t], 4);  // (a lane of each warp)
      mbar_init(&b.o_full[t], 1);
      mbar_init(&b.o_free[t], 4);
      mbar_init(&b.stat_full[t], 4);
    }
    mbar_init(&b.drain, 1);
    sh->abort = 0;
    asm volatile("fence.mbarrier_init.release.cluster;\n" ::: "memory");
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&a.q)) : "memory");
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&a.k)) : "memory");
    asm volatile("prefetch.tensormap [%0];\n" ::"l"(reinterpret_cast<uint64_t>(&a.v)) : "memory");
  }
  if (warp == 1) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], 512;\n" ::"r"(smem_u32(&sh->tmem))
                 : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;\n" ::: "memory");
  }
  pdl_enter();
  // The join's blocks find no room beside this CTA, but are ready when it ends.
  // Not before the wait above: they read the plan before their own.
  asm volatile("griddepcontrol.launch_dependents;\n" ::: "memory");
  Walk w;
  w.start(a);  // (its loads run while the CTA is set up)
  fence_before();
  __syncthreads();
  fence_after();
  // Registers a thread: 4 warps of 80, 8 of 176 and 4 of 80 are what the CTA was
  // launched with, 16 of 128.
  if (warp < 4) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;\n");
    if (warp == 0) {
      copy_tiles<HALVES>(a, sh, w, q_smem, ring, false);
    } else if (warp == 1) {
      multiply<T, HALVES>(a, sh, w, q_smem, ring);
    } else if (warp == 2) {
      copy_tiles<HALVES>(a, sh, w, q_smem, ring, true);
    } else {
      // tokens of no request
      const int64_t first = a.plan->first, last = a.plan->last, none = first + a.n_tokens - last;
      const int64_t pieces = none * a.hq * (a.D / 8);
      for (int64_t i = (int64_t)blockIdx.x * 32 + threadIdx.x - 96; i < pieces; i += (int64_t)gridDim.x * 32) {
        const int64_t x = i / (a.D / 8), h = x % a.hq;
        int64_t t = x / a.hq;
        if (t >= first) t += last - first;
        *reinterpret_cast<uint4*>(static_cast<T*>(a.out.d_data) + t * a.out.token_stride + h * a.out.head_stride +
                                  i % (a.D / 8) * 8) = make_uint4(0, 0, 0, 0);
        if (a.lse) a.lse[t * a.hq + h] = -INFINITY;
      }
    }
  } else if (warp < 12) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;\n");
    softmax<T>(a, sh, w, (warp >> 2) - 1);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;\n");
    write_out<T>(a, sh, w);
  }
  __syncwarp();
  fence_before();
  __syncthreads();
  if (stopped(sh)) {
    // Copies and products in flight must end before the CTA's memory goes. Which
    // are pending is for the warps to know that have given up, or have issued them
    // and gone on: a pause that is a thousand times as long as any takes.
    const long long start = clock64();
    while (clock64() - start < kWaitCycles / 1024) __nanosleep(1000);
    __syncwarp();
  }
  if (warp == 1) {
    fence_after();
    asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, 512;\n" ::"r"(sh->tmem) : "memory");
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
constexpr int kJoinBlocks = 16;  // an SM
template <typename T, int G>
__device__ __forceinline__ void join(const AttentionArgs& a, const KvUnit& unit, int h, int c1, int pieces, int block,
                                     int blocks) {
  const int n_rows = unit.tokens * a.group, full_rows = a.tile_tokens * a.group;
  constexpr int P = 2;
  const int n = n_rows * (a.D / 16), g = threadIdx.x % G, step = blocks * (kJoinThreads / G);
  for (int x = block * (kJoinThreads / G) + threadIdx.x / G; x - (int)(threadIdx.x % 32) / G < n; x += step) {
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
    for (int o = 1; o < G; o <<= 1) top = fmaxf(top, __shfl_xor_sync(kFull, top, o));
    const float f = s.top == -INFINITY ? 0.f : ex2(s.top - top);
    float l = s.l * f, v[16];
#pragma unroll
    for (int q = 0; q < 4; ++q)
      v[4 * q] = s.o[q].x * f, v[4 * q + 1] = s.o[q].y * f, v[4 * q + 2] = s.o[q].z * f, v[4 * q + 3] = s.o[q].w * f;
    int first = 0;  // of the elements that the thread has
#pragma unroll
    for (int o = 1; o < G; o <<= 1) {
      l += __shfl_xor_sync(kFull, l, o);
      const bool high = g & o;
      const int m = 8 / o;  // elements to go on with
      if (m > 0) {
#pragma unroll
        for (int i = 0; i < m; ++i) v[i] = (high ? v[i + m] : v[i]) + __shfl_xor_sync(kFull, high ? v[i] : v[i + m], o);
        first += high ? m : 0;
      } else {
        v[0] += __shfl_xor_sync(kFull, v[0], o);
      }
    }
    if (x >= n) continue;
    const float inv = l > 0.f ? 1.f / l : l;  // (NaN stays)
    const int64_t token = unit.token + r / a.group;
    const int head = h * a.group + r % a.group;
    T* out = static_cast<T*>(a.out.d_data) + token * a.out.token_stride + head * a.out.head_stride + 16 * column;
    if constexpr (G == 1) {
      uint32_t y[8];
#pragma unroll
      for (int q = 0; q < 8; ++q) y[q] = Type<T>::pack(v[2 * q] * inv, v[2 * q + 1] * inv);
      store16(a, out, y);
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

// The blocks in turn for the units that several CTAs share, so that one such
// unit (a chunk over a long sequence: 9 MB of pieces) has them all. Bound by the
// latency of its reads: 10 us for 150 units of 252 rows in two pieces (49 MB), 6
// for 4 units of 8 rows in 38, 3.5 for none.
template <typename T>
__global__ void __launch_bounds__(kJoinThreads) k_paged_join(const __grid_constant__ AttentionArgs a) {
  // (the plan was done before the kernel that this one waits for)
  const int units = a.plan->n_split, blocks = units ? gridDim.x / units : 0;
  const int block = units ? blockIdx.x / units : 0;
  KvShare s = {};
  int c1 = 0;
  if (block < blocks) {
    c1 = a.split[blockIdx.x % units];
    s = a.shares[c1];
  }
  pdl_enter();
  if (block >= blocks) return;
  // Chunks have two or three pieces of many rows, single tokens many of few.
  if (s.n_last <= 4)
    join<T, 1>(a, s.last, s.h1, c1, s.n_last, block, blocks);
  else if (s.n_last <= 16)
    join<T, 8>(a, s.last, s.h1, c1, s.n_last, block, blocks);
  else
    join<T, 32>(a, s.last, s.h1, c1, s.n_last, block, blocks);
}

constexpr size_t smem_bytes(int halves) { return (size_t)(2 + stages(halves)) * halves * kHalf + sizeof(Shared); }
static_assert(smem_bytes(1) <= 232448 && smem_bytes(2) <= 232448, "227 KB");

bool encode(CUtensorMap* m, int32_t dtype, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
            const cuuint32_t* box) {
  EncodeTiledFn enc = tensor_map_encoder();
  const cuuint32_t one[5] = {1, 1, 1, 1, 1};
  return enc && enc(m, dtype == SMETRIC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank,
                    const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Bytes of a stride; a dimension of one entry may have any.
cuuint64_t stride_of(int64_t elements, int64_t entries) { return entries > 1 ? (cuuint64_t)elements * 2 : 256; }

}  // namespace

bool smetric::attention_limits() {
  const auto set = [](const void* f, int halves) {
    return cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(halves)) == cudaSuccess;
  };
  return set((const void*)k_paged_attention<__nv_bfloat16, 1>, 1) && set((const void*)k_paged_attention<__nv_bfloat16, 2>, 2) &&
         set((const void*)k_paged_attention<__half, 1>, 1) && set((const void*)k_paged_attention<__half, 2>, 2);
}

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
  const smetric_kv_config& c = kv->cfg;
  static thread_local AttentionArgs a;
  {
    const cuuint64_t dims[3] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.num_q_heads, (cuuint64_t)kv->n_tokens};
    const cuuint64_t strides[2] = {stride_of(q.head_stride, c.num_q_heads), stride_of(q.token_stride, kv->n_tokens)};
    const cuuint32_t box[3] = {64, (cuuint32_t)kv->group, (cuuint32_t)kv->tile_tokens};
    if (!encode(&a.q, c.dtype, 3, q.d_data, dims, strides, box)) return SMETRIC_ERR_INVALID_ARG;
  }
  {
    const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.page_size, (cuuint64_t)c.num_kv_heads,
                                (cuuint64_t)c.num_pages};
    const cuuint64_t strides[3] = {stride_of(cache.token_stride, c.page_size),
                                   stride_of(cache.head_stride, c.num_kv_heads),
                                   stride_of(cache.page_stride, c.num_pages)};
    const cuuint32_t box[4] = {64, (cuuint32_t)std::min(c.page_size, kTile), 1, 1};
    if (!encode(&a.k, c.dtype, 4, cache.d_k, dims, strides, box) ||
        !encode(&a.v, c.dtype, 4, cache.d_v, dims, strides, box))
      return SMETRIC_ERR_INVALID_ARG;
  }
  a.out = out;
  a.lse = d_lse;
  a.plan = kv->plan;
  a.units = kv->units;
  a.shares = kv->shares;
  a.split = kv->split;
  a.part = kv->part;
  a.part_ml = kv->part_ml;
  a.pages = kv->pages;
  a.pages_stride = kv->pages_stride;
  a.n_tokens = kv->n_tokens;
  a.num_pages = (int32_t)c.num_pages;
  a.hq = c.num_q_heads;
  a.kv_heads = c.num_kv_heads;
  a.group = kv->group;
  a.tile_tokens = kv->tile_tokens;
  a.D = c.head_dim;
  a.page_size = c.page_size;
  a.window = kv->window;
  a.scale = scale;
  a.wide = !(reinterpret_cast<uintptr_t>(out.d_data) & 31) && out.token_stride % 16 == 0 && out.head_stride % 16 == 0;
  a.status = kv->status;
  const int halves = c.head_dim > 64 ? 2 : 1;
  auto kern = c.dtype == SMETRIC_BF16
                  ? (halves == 2 ? k_paged_attention<__nv_bfloat16, 2> : k_paged_attention<__nv_bfloat16, 1>)
                  : (halves == 2 ? k_paged_attention<__half, 2> : k_paged_attention<__half, 1>);
  kv->launches += 2;
  rc = launch_k(kern, dim3((unsigned)kv->num_sms), dim3(kThreads), smem_bytes(halves),
                reinterpret_cast<cudaStream_t>(stream), true, a);
  if (rc) return rc;
  auto join = c.dtype == SMETRIC_BF16 ? k_paged_join<__nv_bfloat16> : k_paged_join<__half>;
  return launch_k(join, dim3((unsigned)kv->num_sms * kJoinBlocks), dim3(kJoinThreads), 0,
                  reinterpret_cast<cudaStream_t>(stream), true, a);
}

}  // extern "C"
