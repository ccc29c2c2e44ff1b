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
// factor of P and its sum l cancels in O / l: so O is seldom rescaled. (Of scores past 2^27,
// 2^29 where P is in bf16, ref's rounding alone takes P out of its type's range: the
// error is latched.)
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
// runs too short for it. A thread spills 116 bytes and loads 136 (of all roles).
//
// Caches in 4 bits (kFour) go the same way with other hands: warp 0 copies tiles of codes
// with TMA, 2 their scales (8 bytes a row are too few for TMA), 3 the query tiles; 12-15
// turn codes into tiles of the ring, in half precision, which all products take; and the
// softmax's warps write the output. Queries in bf16 become half precision, divided by a
// power of two for each row, by 12-15 too. 2,048 tokens over 65,000 take 1,380 us, 1,605
// TFLOP/s (1,554 with the power cap), 3,000 cycles for two query tiles and a key tile:
// the weights have 11 bits instead of 8, memory moves a quarter. What conversions cost is
// issue slots (54 %, where 16-bit caches take 40): a tile's softmax takes 1,700 cycles
// beside them instead of 1,200, and a unit's ends 10,000 and more, as its output is not
// written beside the next unit's softmax. So 4,600 tokens of 8 turns take 429 us (as
// 16-bit caches do: 425), two prompts of 7,600 tokens 700 (641). Before, three warps
// copied and converted what they had copied: 2,369 us for the 2,048 tokens (each took
// 1,200 cycles a tile to copy its part), and 4,344 with their loads in registers, whose
// lines shared memory leaves no room for. A thread spills 208 bytes and loads 236.

#include <cuda.h>
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
#include "tensor_map.cuh"

using namespace smetric;

namespace {

constexpr unsigned kFull = 0xffffffffu;
constexpr long long kWaitCycles = 1ll << 32;  // bounded mbarrier waits: about 2 s
constexpr uint32_t kNap = 20000;  // ns that a waiting warp sleeps between looks at most
constexpr int kThreads = 512;
static_assert(kTile == 1 << 7, "shifts");
constexpr float kSlack = 8.f;     // log2 of how far scores may pass the reference
constexpr uint32_t kHalf = 16384;  // bytes of 128 rows of 64 elements

// Buffers of the ring: what 227 KB hold beside the two query tiles (and, for
// caches in 4 bits, the codes' way to the ring).
__host__ __device__ constexpr int stages(int halves, bool four) {
  return four ? (halves == 2 ? 4 : 10) : halves == 2 ? 5 : 11;
}
// Caches in 4 bits: tiles of codes and scales as they are, on their way to the ring.
constexpr int kStaged = 3;
__host__ __device__ constexpr int codes_bytes(int halves) { return kTile * 32 * halves; }
__host__ __device__ constexpr int staging_bytes(int halves, bool four) {
  return four ? kStaged * (codes_bytes(halves) + kTile * 4 * halves) : 0;
}

struct AttentionArgs {
  CUtensorMap q, k, v;
  smetric_kvq_cache k4, v4;  // (in 4 bits; k and v are of the codes)
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
  float scale, v_scale;
  bool wide;    // outputs can be stored in pieces of 32 bytes
  bool clears;  // zeros for tokens of no request are this kernel's
  int32_t* status;
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
// What caches in 4 bits need besides.
struct SharedFour : Shared {
  uint64_t staged_full[kStaged], staged_empty[kStaged];
  uint64_t q_raw[2];        // query tiles that are yet to be converted
  uint8_t power[4][kTile];  // exponents of the rows of the last query tiles, where they were converted
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

// Places of an item's tiles in the ring, of n key tiles: K0 K1 V0 K2 V1 K3 ...
__device__ __forceinline__ uint32_t place_k(int j) { return j < 2 ? j : 2 * j - 1; }
__device__ __forceinline__ uint32_t place_v(int j, int n) { return min(2 + 2 * j, 2 * n - 1); }

// ---- the warps ----

// The tiles of an item, from its first, of which some query sees a key among `rows` ones
// from row `at`: a lane's page. (A page number says nothing of that: it may be any.)
struct Tiles {
  int32_t begin, end;
  uint32_t key0;
  __device__ __forceinline__ Tiles(const Item& it, int32_t lo, int32_t hi, int at, int rows, bool any) {
    begin = ((lo - rows - at) >> 7) + 1 - it.tb;  // (kTile is 2^7)
    end = any ? min(((hi - at - 1) >> 7) + 1, it.te) - it.tb : INT32_MIN;
    key0 = (uint32_t)it.tb * kTile + at;
  }
  __device__ __forceinline__ bool operator()(int j) const { return j >= begin && j < end; }
  __device__ __forceinline__ uint32_t key(int j) const { return key0 + (uint32_t)j * kTile; }
};

// Query tile number nq of the CTA: tile t of the item's, when its buffer is free. The
// whole warp calls.
template <int HALVES>
__device__ __forceinline__ void copy_queries(const AttentionArgs& a, Shared* sh, const Item& it, int t, uint32_t nq,
                                             uint32_t q_smem, uint64_t* full) {
  Barriers& b = sh->bar;
  if (nq > 1) mbar_wait(&b.q_empty[nq & 1], (nq / 2 - 1) & 1, sh, a.status);
  const bool stop = stopped(sh);
  if ((threadIdx.x & 31) == 0 && !stop) {
    mbar_expect(full, (uint32_t)a.tile_tokens * a.group * 128 * HALVES);
#pragma unroll
    for (int e = 0; e < HALVES; ++e)
      tma_3d(q_smem + ((nq & 1) * HALVES + e) * kHalf, &a.q, 64 * e, it.h * a.group, it.unit.token + t * a.tile_tokens, full);
  }
  __syncwarp();
}

// One warp copies the query tiles and the keys, another the values (a tile of
// 16-token pages is 16 copies, and one warp issues them no faster than memory
// delivers half of them). A lane has a page and a half of the elements.
template <int HALVES>
__device__ __forceinline__ void copy_tiles(const AttentionArgs& a, Shared* sh, Walk w, uint32_t q_smem, uint32_t ring,
                                           const bool values) {
  constexpr int S = stages(HALVES, false);
  Barriers& b = sh->bar;
  const int lane = threadIdx.x & 31;
  const int rows = min(kTile, a.page_size), per = kTile / rows;  // of a copy, and pages of a tile
  const int page_shift = __ffs(a.page_size) - 1;
  const int mine = lane % per, half = lane / per;
  const bool copies = half < HALVES;
  const CUtensorMap* const map = values ? &a.v : &a.k;
  uint32_t base = 0, nq = 0;
  Item it;
  while (w.next(a, it)) {
    const int n = it.te - it.tb;
    // the keys that some query of the unit sees
    const int32_t lo = it.unit.pos >= a.window ? it.unit.pos - a.window + 1 : 0, hi = it.unit.pos + it.unit.tokens;
    const int32_t* pages = a.pages + it.unit.req * a.pages_stride;
    const Tiles seen(it, lo, hi, mine * rows, rows, copies);
    const auto page_of = [&](int j) { return seen(j) ? pages[seen.key(j) >> page_shift] : -1; };
    int32_t next = page_of(0);
    for (int j = 0; j < n; ++j) {
      int32_t page = next;
      next = page_of(j + 1);
      const uint32_t at = base + (values ? place_v(j, n) : place_k(j)), s = at % S;
      if (at >= S) mbar_wait(&b.empty[s], (at / S - 1) & 1, sh, a.status);
      if (stopped(sh)) break;
      const bool held = seen(j);
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
        for (int t = 0; t < (it.pair ? 2 : 1); ++t, ++nq) copy_queries<HALVES>(a, sh, it, t, nq, q_smem, &b.q_full[nq & 1]);
      }
    }
    base += 2 * n;
    if (stopped(sh)) break;
  }
}

// ---- caches in 4 bits ----

// An item's tiles in their order, K0 K1 V0 K2 V1 K3 ..., and the lane's page of each: a
// tile's values have the pages of its keys, two places on.
struct Order {
  int32_t n, jk, jv;         // key tiles; keys' and values' so far
  int32_t ahead, last, before;  // pages of the next keys, of the last ones, of those before
  template <typename F>
  __device__ __forceinline__ void start(int32_t tiles, F page_of) {
    n = tiles, jk = jv = 0;
    last = before = -1;
    ahead = page_of(0);
  }
  // The next tile, its page and whether it is of values; page_of(j) is the page of tile j.
  template <typename F>
  __device__ __forceinline__ int32_t next(F page_of, bool& values, int32_t& page) {
    values = jk == n || (jk > 1 && jv < jk - 1);
    if (values) {
      page = jv == jk - 1 ? last : before;
      return jv++;
    }
    page = ahead;
    before = last, last = ahead;
    ahead = jk + 1 < n ? page_of(jk + 1) : -1;
    return jk++;
  }
};

// One warp copies the tiles' codes as they are, a lane a page.
template <int HALVES>
__device__ __forceinline__ void copy_codes(const AttentionArgs& a, SharedFour* sh, Walk w, uint32_t staging) {
  const int lane = threadIdx.x & 31;
  const int rows = min(kTile, a.page_size), per = kTile / rows;  // of a copy, and pages of a tile
  const int page_shift = __ffs(a.page_size) - 1, row_bytes = a.D / 2;
  uint32_t at = 0;
  Order order;
  Item it;
  while (w.next(a, it)) {
    const int32_t lo = it.unit.pos >= a.window ? it.unit.pos - a.window + 1 : 0, hi = it.unit.pos + it.unit.tokens;
    const int32_t* pages = a.pages + it.unit.req * a.pages_stride;
    const Tiles seen(it, lo, hi, lane * rows, rows, lane < per);
    const auto page_of = [&](int j) { return seen(j) ? pages[seen.key(j) >> page_shift] : -1; };
    order.start(it.te - it.tb, page_of);
    for (int place = 0; place < 2 * order.n; ++place, ++at) {
      bool values;
      int32_t page;
      const int j = order.next(page_of, values, page);
      const uint32_t s = at % kStaged;
      if (at >= kStaged) mbar_wait(&sh->staged_empty[s], (at / kStaged - 1) & 1, sh, a.status);
      if (stopped(sh)) break;
      const bool held = (uint32_t)page < (uint32_t)a.num_pages;
      if (!held && seen(j)) latch_error(a.status, SMETRIC_ERR_INVALID_ARG);  // (its scales become zeros)
      const unsigned who = __ballot_sync(kFull, held);
      if (lane == 0) mbar_expect(&sh->staged_full[s], __popc(who) * rows * row_bytes);
      __syncwarp();
      if (held)
        tma_4d(staging + s * codes_bytes(HALVES) + lane * rows * row_bytes, values ? &a.v : &a.k, 0,
               a.page_size > kTile ? (it.tb + j) * kTile % a.page_size : 0, it.h, page, &sh->staged_full[s]);
    }
    if (stopped(sh)) break;
  }
}

// 8 bytes to shared memory, or zeros (4 for heads of at most 64 elements).
template <int N>
__device__ __forceinline__ void copy_row_scales(uint32_t dst, const void* src, bool held) {
  asm volatile("cp.async.ca.shared.global [%0], [%1], %2, %3;\n" ::"r"(dst), "l"(src), "n"(N), "r"(held ? N : 0) : "memory");
}

// Another warp copies their scales, a lane every 32nd row. Rows that nobody sees have
// scales of zero.
template <int HALVES>
__device__ __forceinline__ void copy_scales(const AttentionArgs& a, SharedFour* sh, Walk w, uint32_t staging) {
  constexpr int SB = 4 * HALVES;
  const int lane = threadIdx.x & 31, page_shift = __ffs(a.page_size) - 1;
  staging += kStaged * codes_bytes(HALVES);
  uint32_t at = 0;
  Order order;
  Item it;
  while (w.next(a, it)) {
    const int32_t lo = it.unit.pos >= a.window ? it.unit.pos - a.window + 1 : 0, hi = it.unit.pos + it.unit.tokens;
    const int32_t* pages = a.pages + it.unit.req * a.pages_stride;
    // the page of 16 rows (lane & 7) of a tile
    const auto page_of = [&](int j) {
      const int64_t key = (int64_t)(it.tb + j) * kTile + 16 * (lane & 7);
      return key < hi && key + 16 > lo ? pages[key >> page_shift] : -1;
    };
    order.start(it.te - it.tb, page_of);
    for (int place = 0; place < 2 * order.n; ++place, ++at) {
      bool values;
      int32_t page;
      const int64_t key = (int64_t)(it.tb + order.next(page_of, values, page)) * kTile + lane;
      const smetric_kvq_cache& c = values ? a.v4 : a.k4;
      const uint8_t* scales = static_cast<const uint8_t*>(c.d_scales) + it.h * c.scale_head_stride;
      const uint32_t page_stride = (uint32_t)c.scale_page_stride, token_stride = (uint32_t)c.scale_token_stride;  // (below 2^32)
      const uint32_t s = at % kStaged;
      if (at >= kStaged) mbar_wait(&sh->staged_empty[s], (at / kStaged - 1) & 1, sh, a.status);
      if (stopped(sh)) break;
#pragma unroll
      for (int i = 0; i < 4; ++i) {
        const int64_t x = key + 32 * i;
        const int32_t p = __shfl_sync(kFull, page, 2 * i + (lane >> 4));
        const bool held = (uint32_t)p < (uint32_t)a.num_pages && x >= lo && x < hi;
        const uint32_t in = (uint32_t)x & (a.page_size - 1);
        copy_row_scales<SB>(staging + (s * kTile + 32 * i + lane) * SB,
                            scales + (uint64_t)(held ? (uint32_t)p : 0u) * page_stride + (uint64_t)in * token_stride, held);
      }
      asm volatile("cp.async.mbarrier.arrive.noinc.shared.b64 [%0];\n" ::"r"(smem_u32(&sh->staged_full[s])) : "memory");
    }
    if (stopped(sh)) break;
  }
  asm volatile("cp.async.wait_all;\n" ::: "memory");
}

// A row (the thread's) of query tile number nq from bf16 to half precision, in its
// place: divided by the power of two of its largest element, so that 8 bits of elements
// of 2^-17 of it and more fit; smaller ones are rounded to multiples of 2^-24 of it.
template <int HALVES>
__device__ __forceinline__ void convert_row(SharedFour* sh, uint32_t nq, uint32_t q_smem, int row) {
  const uint32_t at = q_smem + (nq & 1) * HALVES * kHalf + row * 128;
  const auto chunk = [&](int j) { return at + (j >> 3) * kHalf + (((j & 7) ^ (row & 7)) << 4); };
  uint32_t top = 0;  // magnitudes' bits order as they do
#pragma unroll 4
  for (int j = 0; j < 8 * HALVES; ++j) {
    uint32_t x[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(chunk(j)) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i) top = __vmaxu2(top, x[i] & 0x7fff7fffu);
  }
  const uint32_t most = max(top >> 16, top & 0xffff) >> 7;
  const uint32_t E = most == 0 ? 1 : most == 255 ? 127 : min(most, 253);  // (infinities keep their row as it is)
  const float down = __uint_as_float((254 - E) << 23);
  sh->power[nq & 3][row] = (uint8_t)E;
#pragma unroll 4
  for (int j = 0; j < 8 * HALVES; ++j) {
    uint32_t x[4];
    asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n" : "=r"(x[0]), "=r"(x[1]), "=r"(x[2]), "=r"(x[3]) : "r"(chunk(j)) : "memory");
#pragma unroll
    for (int i = 0; i < 4; ++i)
      x[i] = Type<__half>::pack(__uint_as_float(x[i] << 16) * down, __uint_as_float(x[i] & 0xffff0000u) * down);
    asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(chunk(j)), "r"(x[0]), "r"(x[1]), "r"(x[2]), "r"(x[3]) : "memory");
  }
}

// Four warps turn tiles of codes into tiles of the ring in half precision, in the
// 128-byte swizzle, 32 rows each: a conversion for two codes and a product with their
// scale, both exact (2 and 4 bits). A tile's keys and values are laid out alike. They
// also convert an item's query tiles (kQueries), when they find them there between two
// of its tiles, and after as many as the ring takes (or its last) at the latest: all
// before are used up without the queries.
template <int HALVES, bool kQueries>
__device__ __forceinline__ void convert_tiles(const AttentionArgs& a, SharedFour* sh, Walk w, uint32_t q_smem, uint32_t ring,
                                              uint32_t staging) {
  constexpr int S = stages(HALVES, true), SB = 4 * HALVES;
  Barriers& b = sh->bar;
  const int lane = threadIdx.x & 31, odd = lane >> 4, row = (threadIdx.x >> 5 & 3) * 32 + (lane & 15);
  const int pieces = a.D / 32;  // of 16 bytes, in a row: a lane has piece `odd` and, of longer heads, 2 + odd
  const int row_bytes = a.D / 2;
  // (rows of 64 and of 32 bytes are swizzled, for the banks; 16 rows on, alike)
  const int swizzle = row_bytes == 64 ? row >> 1 & 3 : row_bytes == 32 ? row >> 2 & 1 : 0;
  uint32_t at = 0, nq = 0;
  Item it;
  while (w.next(a, it)) {
    const int n = it.te - it.tb;
    int queries = it.pair ? 2 : 1;  // tiles left to convert
    for (int place = 0; place < 2 * n; ++place, ++at) {
      const uint32_t s = at % S, from = at % kStaged;
      mbar_wait(&sh->staged_full[from], at / kStaged & 1, sh, a.status);
      if (stopped(sh)) break;
      uint32_t word[2][HALVES][4], two[2][HALVES];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int e = 0; e < HALVES; ++e) {
          const int piece = 2 * e + odd;
          if (piece < pieces) {
            asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];\n"
                         : "=r"(word[i][e][0]), "=r"(word[i][e][1]), "=r"(word[i][e][2]), "=r"(word[i][e][3])
                         : "r"(staging + from * codes_bytes(HALVES) + (row + 16 * i) * row_bytes + 16 * (piece ^ swizzle)) : "memory");
            asm volatile("{\n .reg .b16 x;\n ld.shared.b16 x, [%1];\n cvt.u32.u16 %0, x;\n}\n"
                         : "=r"(two[i][e])
                         : "r"(staging + kStaged * codes_bytes(HALVES) + (from * kTile + row + 16 * i) * SB + 2 * piece) : "memory");
          }
        }
      }
      if (at >= S) mbar_wait(&b.empty[s], (at / S - 1) & 1, sh, a.status);
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int e = 0; e < HALVES; ++e) {
          uint32_t h2;
          asm("{\n .reg .b16 x, y;\n mov.b32 {x, y}, %1;\n cvt.rn.f16x2.e4m3x2 %0, x;\n}\n" : "=r"(h2) : "r"(two[i][e]));
          const uint32_t scale[2] = {__byte_perm(h2, 0, 0x1010), __byte_perm(h2, 0, 0x3232)};
          const uint32_t dst = ring + (s * HALVES + e) * kHalf + (row + 16 * i) * 128;
          uint32_t y[4][4];
#pragma unroll
          for (int q = 0; q < 4; ++q)
            asm("{\n .reg .b8 a, b, c, d;\n .reg .b32 e, f, g, h;\n mov.b32 {a, b, c, d}, %4;\n cvt.rn.f16x2.e2m1x2 e, a;\n"
                " cvt.rn.f16x2.e2m1x2 f, b;\n cvt.rn.f16x2.e2m1x2 g, c;\n cvt.rn.f16x2.e2m1x2 h, d;\n mul.rn.f16x2 %0, e, %5;\n"
                " mul.rn.f16x2 %1, f, %5;\n mul.rn.f16x2 %2, g, %5;\n mul.rn.f16x2 %3, h, %5;\n}\n"
                : "=r"(y[q][0]), "=r"(y[q][1]), "=r"(y[q][2]), "=r"(y[q][3]) : "r"(word[i][e][q]), "r"(scale[q >> 1]));
          if (2 * e + odd < pieces) {
#pragma unroll
            for (int q = 0; q < 4; ++q)
              asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};\n" ::"r"(dst + (((4 * odd + q) ^ (row & 7)) << 4)),
                           "r"(y[q][0]), "r"(y[q][1]), "r"(y[q][2]), "r"(y[q][3]) : "memory");
          }
        }
      }
      asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
      __syncwarp();
      if (lane == 0) {
        mbar_arrive(&sh->staged_empty[from]);
        mbar_arrive(&b.full[s]);
      }
      if (kQueries) {
        while (queries > 0) {
          uint64_t* const raw = &sh->q_raw[nq & 1];
          if (place < min(S, 2 * n) - 1 && !__any_sync(kFull, mbar_test(raw, nq / 2 & 1))) break;
          mbar_wait(raw, nq / 2 & 1, sh, a.status);
          convert_row<HALVES>(sh, nq, q_smem, threadIdx.x & 127);
          asm volatile("fence.proxy.async.shared::cta;\n" ::: "memory");
          __syncwarp();
          if (lane == 0) mbar_arrive(&b.q_full[nq & 1]);
          ++nq, --queries;
        }
      }
    }
    if (stopped(sh)) break;
  }
}

// The query tiles of every item, in order.
template <int HALVES, bool kQueries>
__device__ __forceinline__ void copy_all_queries(const AttentionArgs& a, SharedFour* sh, Walk w, uint32_t q_smem) {
  uint32_t nq = 0;
  Item it;
  while (w.next(a, it)) {
    for (int t = 0; t < (it.pair ? 2 : 1); ++t, ++nq)
      copy_queries<HALVES>(a, sh, it, t, nq, q_smem, (kQueries ? sh->q_raw : sh->bar.q_full) + (nq & 1));
    if (stopped(sh)) break;
  }
}

// Issues the products, a step's (weights with values, then the half's next
// scores) by one elected lane in one go: this warp is close to the limit, a wait
// that is ready costs it 60 to 160 cycles. The two halves take turns.
template <typename T, int HALVES, bool kFour>
__device__ __forceinline__ void multiply(const AttentionArgs& a, Shared* sh, Walk w, uint32_t q_smem, uint32_t ring) {
  constexpr int S = stages(HALVES, kFour);
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
      if (kFour) return;  // (they are zeros already)
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

// A tile's first token in its unit, and its rows.
__device__ __forceinline__ int tile_token(const AttentionArgs& a, const Item& it, int tile) {
  return it.pair ? tile * a.tile_tokens : 0;
}
__device__ __forceinline__ int tile_rows(const AttentionArgs& a, const Item& it, int tile) {
  return min(a.tile_tokens, it.unit.tokens - tile_token(a, it, tile)) * a.group;
}

// The lowest n bits, none or all where n is outside 0..32.
__device__ __forceinline__ uint32_t below(int32_t n) { return n <= 0 ? 0 : n >= 32 ? kFull : (1u << n) - 1; }

// An item's output (a query tile's of two): O / l, or its sums and statistics where
// other CTAs have pieces of it. The four warps of a tile call, for the even and the odd
// key tiles together where an item has one query tile. no: ends of products so far.
template <typename T, bool kFour>
__device__ __forceinline__ void write_tile(const AttentionArgs& a, Shared* sh, const Item& it, int tile, uint32_t items,
                                           uint32_t (&no)[2]) {
  Barriers& b = sh->bar;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5 & 3, row = threadIdx.x & 127;
  const uint32_t o_all = sh->tmem + 2 * kTile + ((uint32_t)warp << 21);
  const int row_token = row / a.group, row_head = row - row_token * a.group;
  const bool two = !it.pair && it.te - it.tb > 1;  // sums of even and of odd key tiles
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
    float inv = it.whole ? (st.y > 0.f ? 1.f / st.y : st.y) : 1.f;  // (NaN stays)
    if (kFour && it.whole) inv *= a.v_scale;
    w1 *= inv, w2 *= inv;
    const uint32_t o_at = o_all + tile * kTile;
    T* out = static_cast<T*>(a.out.d_data) + token * a.out.token_stride + head * a.out.head_stride;
    const auto store = [&](int d, const float (&f)[16]) {
      if (!mine) return;
      if (it.whole) {
        uint32_t y[8];
#pragma unroll
        for (int i = 0; i < 8; ++i) y[i] = Type<T>::pack(f[2 * i], f[2 * i + 1]);
        store16(a.wide, out + d, y);
      } else {
        float4* p = reinterpret_cast<float4*>(a.part) + part_at(a.D, it.slot, tile, d / 4) + row;
#pragma unroll
        for (int i = 0; i < 4; ++i) p[i * kTile] = make_float4(f[4 * i], f[4 * i + 1], f[4 * i + 2], f[4 * i + 3]);
      }
    };
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
      store(d, f);
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

template <typename T>
__device__ __forceinline__ void write_out(const AttentionArgs& a, Shared* sh, Walk w) {
  uint32_t items = 0, no[2] = {0, 0};
  Item it;
  for (; w.next(a, it); ++items)
    for (int tile = 0; tile < (it.pair ? 2 : 1); ++tile) write_tile<T, false>(a, sh, it, tile, items, no);
}

// (One code for both tiles: two copies miss the instruction cache.)
// With caches in 4 bits the scores may be of rows divided by a power of two
// (kPowers), and these warps write the output, as the ones that do else convert.
template <typename T, typename Out, bool kFour>
__device__ __forceinline__ void softmax(const AttentionArgs& a, Shared* sh, Walk w, const int tile) {
  Barriers& b = sh->bar;
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5 & 3, row = threadIdx.x & 127;
  const uint32_t lanes = (uint32_t)warp << 21;  // the warp's TMEM lanes
  const uint32_t s_at = sh->tmem + tile * kTile + lanes, o_at = sh->tmem + 2 * kTile + tile * kTile + lanes;
  const int row_token = row / a.group;
  float c = a.scale * 1.4426950408889634f;
  constexpr bool kPowers = !std::is_same<T, Out>::value;
  uint32_t ns = 0, items = 0, nq = 0, no[2] = {0, 0};
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
      if (kPowers && j <= tile)
        c = score_factor(
            a.scale * 1.4426950408889634f *
            __uint_as_float((uint32_t) * (volatile uint8_t*)&static_cast<SharedFour*>(sh)->power[(nq + (it.pair ? tile : 0)) & 3][row] << 23));
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
          const float next = reference(most, c, Type<T>::kLift);
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
    if (mine && too_far(ref, Type<T>::kLift)) latch_error(a.status, SMETRIC_ERR_OVERFLOW);
    nq += it.pair ? 2 : 1;
    if (items) mbar_wait(&b.o_free[tile], (items - 1) & 1, sh, a.status);
    // (scores that are all NaN leave top where it was, but not l: the row is not
    // one without keys, and what joins its pieces must not pass over it)
    sh->stat[tile][row] = make_float2(top == -INFINITY && l == 0.f ? -INFINITY : ref, l);
    __syncwarp();
    if (lane == 0) mbar_arrive(&b.stat_full[tile]);
    if (kFour) {
      if (it.pair || tile == 0) write_tile<Out, true>(a, sh, it, tile, items, no);
      // (ends of the other tile's products)
      if (tile == 0 ? it.pair : !it.pair && n > 1) ++no[1];
    }
  }
}

template <typename T, int HALVES, bool kFour>
__global__ void __launch_bounds__(kThreads, 1) k_paged_attention(const __grid_constant__ AttentionArgs a) {
  constexpr int S = stages(HALVES, kFour);
  using M = std::conditional_t<kFour, __half, T>;  // what the matrix products take
  constexpr bool kQueries = !std::is_same<M, T>::value;  // queries are converted
  extern __shared__ __align__(1024) unsigned char smem_raw[];
  using Sh = std::conditional_t<kFour, SharedFour, Shared>;
  Sh* sh = reinterpret_cast<Sh*>(smem_raw + (2 + S) * HALVES * kHalf + staging_bytes(HALVES, kFour));
  if (smem_u32(smem_raw) & 1023) {  // (the swizzle's groups of 8 rows)
    latch_error(a.status, SMETRIC_ERR_CUDA);
    return;
  }
  const uint32_t q_smem = smem_u32(smem_raw), ring = q_smem + 2 * HALVES * kHalf, staging = ring + S * HALVES * kHalf;
  const int warp = threadIdx.x >> 5;
  if constexpr (kFour) {  // (steps of single tokens have no chunks)
    pdl_enter();
    if (a.shares[blockIdx.x].u0 < 0 && !a.clears) return;
  }
  if (threadIdx.x == 0) {
    Barriers& b = sh->bar;
    for (int i = 0; i < S; ++i) mbar_init(&b.full[i], kFour ? 4 : 1), mbar_init(&b.empty[i], 1);
    for (int t = 0; t < 2; ++t) {
      mbar_init(&b.q_full[t], kQueries ? 4 : 1);
      mbar_init(&b.q_empty[t], 1);
      mbar_init(&b.s_full[t], 1);
      mbar_init(&b.p_full[t], 4);  // (a lane of each warp)
      mbar_init(&b.o_full[t], 1);
      mbar_init(&b.o_free[t], 4);
      mbar_init(&b.stat_full[t], 4);
    }
    if constexpr (kFour) {
      // (the codes' copy and 32 lanes' of scales; four warps)
      for (int i = 0; i < kStaged; ++i) mbar_init(&sh->staged_full[i], 33), mbar_init(&sh->staged_empty[i], 4);
      mbar_init(&sh->q_raw[0], 1), mbar_init(&sh->q_raw[1], 1);
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
    if (warp == 1) {
      multiply<M, HALVES, kFour>(a, sh, w, q_smem, ring);
    } else if (warp != 3) {
      if constexpr (kFour) {
        if (warp == 0)
          copy_codes<HALVES>(a, sh, w, staging);
        else
          copy_scales<HALVES>(a, sh, w, staging);
      } else {
        copy_tiles<HALVES>(a, sh, w, q_smem, ring, warp == 2);
      }
    } else {
      if (!kFour || a.clears) {
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
        __syncwarp();
      }
      if constexpr (kFour) copy_all_queries<HALVES, kQueries>(a, sh, w, q_smem);
    }
  } else if (warp < 12) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 176;\n");
    softmax<M, T, kFour>(a, sh, w, (warp >> 2) - 1);
  } else {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 80;\n");
    if constexpr (kFour)
      convert_tiles<HALVES, kQueries>(a, sh, w, q_smem, ring, staging);
    else
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

constexpr int kJoinBlocks = 16;  // an SM
// Bound by the latency of its reads: 10 us for 150 units of 252 rows in two pieces (49
// MB), 6 for 4 units of 8 rows in 38, 3.5 for none.
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
  join_unit<T>(a, s, c1, block, blocks, threadIdx.x);
}

constexpr size_t smem_bytes(int halves, bool four) {
  return (size_t)(2 + stages(halves, four)) * halves * kHalf + staging_bytes(halves, four) +
         (four ? sizeof(SharedFour) : sizeof(Shared));
}
static_assert(smem_bytes(1, false) <= 232448 && smem_bytes(2, false) <= 232448 && smem_bytes(1, true) <= 232448 &&
                  smem_bytes(2, true) <= 232448, "227 KB");

bool encode(CUtensorMap* m, int32_t dtype, int rank, const void* base, const cuuint64_t* dims, const cuuint64_t* strides,
            const cuuint32_t* box) {
  EncodeTiledFn enc = tensor_map_encoder();
  const cuuint32_t one[5] = {1, 1, 1, 1, 1};
  return enc && enc(m, dtype == SMETRIC_BF16 ? CU_TENSOR_MAP_DATA_TYPE_BFLOAT16 : CU_TENSOR_MAP_DATA_TYPE_FLOAT16, rank,
                    const_cast<void*>(base), dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    CU_TENSOR_MAP_SWIZZLE_128B, CU_TENSOR_MAP_L2_PROMOTION_L2_256B,
                    CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// A page's rows of a head's codes, up to 128.
bool encode_codes(CUtensorMap* m, const smetric_kv_config& c, const smetric_kvq_cache& cache) {
  EncodeTiledFn enc = tensor_map_encoder();
  const cuuint32_t one[4] = {1, 1, 1, 1}, box[4] = {(cuuint32_t)c.head_dim / 2, (cuuint32_t)std::min(c.page_size, kTile), 1, 1};
  const cuuint64_t dims[4] = {(cuuint64_t)c.head_dim / 2, (cuuint64_t)c.page_size, (cuuint64_t)c.num_kv_heads,
                              (cuuint64_t)c.num_pages};
  // (a dimension of one entry may have any stride)
  const cuuint64_t strides[3] = {(cuuint64_t)cache.token_stride, c.num_kv_heads > 1 ? (cuuint64_t)cache.head_stride : 256,
                                 c.num_pages > 1 ? (cuuint64_t)cache.page_stride : 256};
  return enc && enc(m, CU_TENSOR_MAP_DATA_TYPE_UINT8, 4, cache.d_codes, dims, strides, box, one, CU_TENSOR_MAP_INTERLEAVE_NONE,
                    c.head_dim == 128  ? CU_TENSOR_MAP_SWIZZLE_64B
                    : c.head_dim == 64 ? CU_TENSOR_MAP_SWIZZLE_32B
                                       : CU_TENSOR_MAP_SWIZZLE_NONE,
                    CU_TENSOR_MAP_L2_PROMOTION_L2_64B, CU_TENSOR_MAP_FLOAT_OOB_FILL_NONE) == CUDA_SUCCESS;
}

// Bytes of a stride; a dimension of one entry may have any.
cuuint64_t stride_of(int64_t elements, int64_t entries) { return entries > 1 ? (cuuint64_t)elements * 2 : 256; }

}  // namespace

namespace {
template <typename T, bool kFour>
bool limits() {
  const auto set = [](const void* f, int halves) {
    return cudaFuncSetAttribute(f, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)smem_bytes(halves, kFour)) == cudaSuccess;
  };
  return set((const void*)k_paged_attention<T, 1, kFour>, 1) && set((const void*)k_paged_attention<T, 2, kFour>, 2);
}

// The attention and, with `joins`, its join; `a` has the caches, the rest is set here.
template <bool kFour>
int launch_attention(smetric_kv* kv, AttentionArgs& a, const smetric_heads& q, float scale, const smetric_heads& out,
                     float* d_lse, bool joins, smetric_stream_t stream) {
  const smetric_kv_config& c = kv->cfg;
  {
    const cuuint64_t dims[3] = {(cuuint64_t)c.head_dim, (cuuint64_t)c.num_q_heads, (cuuint64_t)kv->n_tokens};
    const cuuint64_t strides[2] = {stride_of(q.head_stride, c.num_q_heads), stride_of(q.token_stride, kv->n_tokens)};
    const cuuint32_t box[3] = {64, (cuuint32_t)kv->group, (cuuint32_t)kv->tile_tokens};
    if (!encode(&a.q, c.dtype, 3, q.d_data, dims, strides, box)) return SMETRIC_ERR_INVALID_ARG;
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
                  ? (halves == 2 ? k_paged_attention<__nv_bfloat16, 2, kFour> : k_paged_attention<__nv_bfloat16, 1, kFour>)
                  : (halves == 2 ? k_paged_attention<__half, 2, kFour> : k_paged_attention<__half, 1, kFour>);
  kv->launches += 1 + joins;
  const int rc = launch_k(kern, dim3((unsigned)kv->num_sms), dim3(kThreads), smem_bytes(halves, kFour),
                          reinterpret_cast<cudaStream_t>(stream), true, a);
  if (rc || !joins) return rc;
  auto join = c.dtype == SMETRIC_BF16 ? k_paged_join<__nv_bfloat16> : k_paged_join<__half>;
  return launch_k(join, dim3((unsigned)kv->num_sms * kJoinBlocks), dim3(kJoinThreads), 0,
                  reinterpret_cast<cudaStream_t>(stream), true, a);
}
}  // namespace

bool smetric::attention_limits(bool four) {
  return four ? limits<__nv_bfloat16, true>() && limits<__half, true>()
              : limits<__nv_bfloat16, false>() && limits<__half, false>();
}

int smetric::attention_many_rows(smetric_kv* kv, const smetric_kvq_cache& k_cache, const smetric_kvq_cache& v_cache,
                                 const smetric_heads& q, float scale, const smetric_heads& out, float* d_lse,
                                 smetric_stream_t stream) {
  static thread_local AttentionArgs a;
  if (!encode_codes(&a.k, kv->cfg, k_cache) || !encode_codes(&a.v, kv->cfg, v_cache)) return SMETRIC_ERR_INVALID_ARG;
  a.k4 = k_cache;
  a.v4 = v_cache;
  a.v_scale = std::ldexp(1.f, v_cache.exp);
  a.clears = !kv->few.rows;
  return launch_attention<true>(kv, a, q, std::ldexp(scale, k_cache.exp), out, d_lse, !kv->one_join, stream);
}

extern "C" {

int smetric_paged_attention(smetric_kv* kv, smetric_kv_cache cache, smetric_heads q, float scale, smetric_heads out,
                            float* d_lse, smetric_stream_t stream) {
  CallRange range("smetric_paged_attention");
  int rc = check_device(kv);
  if (rc) return rc;
  if (four_bits(kv) || !kv->planned || !scale_ok(scale) || !cache_ok(cache) || !heads_ok(q, kv->n_tokens) ||
      !heads_ok(out, kv->n_tokens) || (reinterpret_cast<uintptr_t>(d_lse) & 3))
    return SMETRIC_ERR_INVALID_ARG;
  if (kv->n_tokens == 0) return SMETRIC_OK;
  const smetric_kv_config& c = kv->cfg;
  static thread_local AttentionArgs a;
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
  a.v_scale = 1.f;
  a.clears = true;
  return launch_attention<false>(kv, a, q, scale, out, d_lse, true, stream);
}

}  // extern "C"
