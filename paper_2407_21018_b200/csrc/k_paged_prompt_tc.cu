// Attention of many new tokens of each sequence over its pages (causal) on the 5th-generation tensor cores, bf16 queries.
//
// An item is 256 rows of queries that share a key head (256 / G new tokens times the G heads), as two halves of 128 rows
// that take turns on the tensor cores: while one half's logits pass through the softmax, the other's products run.
//   S = Q K^T       tcgen05.mma from shared memory into tensor memory, a tile of 64 tokens; two tiles' S a half, so that the
//                   next one is there when a softmax ends; thread t of a half's four warps owns row t
//   P = 2^(x - m)   read from tensor memory, written back over S as bf16: the A operand of
//   O += P V        tcgen05.mma, V as stored ([token][channel]) is the MN-major B operand
// Roles: warps 0-3 and 4-7 the softmax of a half each; a warp for the products of each half; a warp for keys and one for values
// bring them into a ring of shared-memory slots (bf16 pages by TMA; others as bytes by bulk copies, which four or eight warps
// unpack from stages into the ring); four warps load the next item's queries and store the last item's outputs, so that the others
// go from item to item without a pause.  One of the loading warps walks along the items and hands out their description.  m stands
// 2^8 above the largest logit and only moves when one passes it (O is then rescaled in tensor memory), so the softmax seldom waits
// for the products.
// 4-bit values n * s have 11 bits: they enter as the sum of two bf16, which is exact, at twice the products.  Queries (on e4m3 pages keys)
// are taken times the power of two in the softmax scale, so that S passes fp32 no sooner than the logits.
// P is rounded to bf16 (2^-9 of a weight on average, what the products take); l sums the unrounded weights, with what its
// additions lose carried along, in fp32.
//
// What bounds it (a prompt of 8192 tokens, 32 heads of 128 over 8 key heads, 482 us replayed: 0.55 TFLOP at 1140 TFLOP/s, 0.70 of the
// measured GEMM rate; 564 among other calls, where the clock falls): no unit.  Tensor pipe and exponentials are each busy for 47 % of
// the cycles (a tile of both halves: 1280 cycles of products, S at 48 a product because Q and K both come from shared memory, and
// 1024 of exponentials, against 2160).  It waits for the chain of a softmax warp: tensor memory read, maximum, vote, exponentials, packing,
// write, arrival, with one warp of each half a scheduler.  Heads of 64 have half the products and take no fewer cycles a tile (2 x 4096
// tokens, 12 heads: 122 to 135 us).  e4m3 adds the unpacking (8192 tokens 610 to 740 us), 4 bits twice the products (780 to 830 us).  Few rows:
// DRAM (8 rows over 131072 tokens, twice, 1.07 GB in 173 us).  Short calls: code that is fetched for the first time (100 tokens: 22 us,
// the join among them).  Loops stay rolled for that, and because the roles' code together misses the instruction cache.
// Tiles of 128 tokens, whose S has one place a half, took 563 us for the same prompt; P in places of its own and S read ahead of
// the weights of the tile before 515; exponentials in part by a polynomial, or of the halves strictly in turn, were slower too.
// Every wait is bounded (about a second, those for whole items by the others): on a time-out the CTA raises the error word, frees its tensor memory and leaves.
#include <math.h>
#include <string.h>

#include <cuda.h>

#include "paged_prompt_walk.cuh"

namespace think {
namespace {

constexpr int kHalf = 128, kItemRows = 2 * kHalf;
// See PromptCut: starting and ending an item costs as much as six tiles (a prompt of 8192 bf16 tokens, a ragged e4m3 batch of 48 in us with
// 128: 534, 315, 256: 496, 297, 384: 489, 291, 640: 498, 319).
constexpr int kExtra = 384;
// A row's reference m stands so far (in base 2) above the largest logit there was when it last moved, and moves when a logit passes
// it: seldom, and no weight is above 1, so that a weight times a value passes fp32 only where the value does.
constexpr float kAbove = 8.f;

// ---- PTX
__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
__device__ __forceinline__ void cp_async16(uint32_t dst, const void* src, int bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(bytes) : "memory");
}
__device__ __forceinline__ void cp_async_wait_all() { asm volatile("cp.async.wait_all;" ::: "memory"); }
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
__device__ __forceinline__ float max3(float a, float b, float c) {
  float y;
  asm("max.f32 %0, %1, %2, %3;" : "=f"(y) : "f"(a), "f"(b), "f"(c));
  return y;
}
// Shared-memory matrix descriptors, 128-byte swizzle, 8-row groups of 1024 bytes: the low word has the address and the leading
// byte offset in 16-byte units, the high word is the same for all.
__device__ __forceinline__ uint32_t desc_lo(uint32_t saddr, uint32_t lbo_bytes) { return (saddr >> 4) | (lbo_bytes >> 4) << 16; }
constexpr uint32_t kDescHi = (1024u >> 4) | 1u << 14 | 2u << 29;
// instruction descriptor: fp32 accumulate, bf16 x bf16, M = 128; B K-major or MN-major
__host__ __device__ constexpr uint32_t idesc(int n, bool b_mn) {
  return (1u << 4) | (1u << 7) | (1u << 10) | ((b_mn ? 1u : 0u) << 16) | ((uint32_t)(n >> 3) << 17) | ((128u >> 4) << 24);
}
// The products' warp runs as one, so that operands stay in uniform registers; its leading lane issues.
__device__ __forceinline__ uint32_t elect_lane() {
  uint32_t x;
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "elect.sync _|p, 0xffffffff;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "}\n"
      : "=r"(x));
  return x;
}
// a, b: low words of descriptors
__device__ __forceinline__ void mma_ss(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t id, uint32_t accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p, l;\n\t"
      ".reg .b64 da, db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 l, %7, 0;\n\t"
      "mov.b64 da, {%1, %6};\n\t"
      "mov.b64 db, {%2, %6};\n\t"
      "@l tcgen05.mma.cta_group::1.kind::f16 [%0], da, db, %3, {%5, %5, %5, %5}, p;\n\t"
      "}\n"
      :: "r"(d), "r"(a), "r"(b), "r"(id), "r"(accumulate), "r"(0u), "r"(kDescHi), "r"(lead) : "memory");
}
// a: in tensor memory
__device__ __forceinline__ void mma_ts(uint32_t lead, uint32_t d, uint32_t a, uint32_t b, uint32_t id, uint32_t accumulate) {
  asm volatile(
      "{\n\t"
      ".reg .pred p, l;\n\t"
      ".reg .b64 db;\n\t"
      "setp.ne.b32 p, %4, 0;\n\t"
      "setp.ne.b32 l, %7, 0;\n\t"
      "mov.b64 db, {%2, %6};\n\t"
      "@l tcgen05.mma.cta_group::1.kind::f16 [%0], [%1], db, %3, {%5, %5, %5, %5}, p;\n\t"
      "}\n"
      :: "r"(d), "r"(a), "r"(b), "r"(id), "r"(accumulate), "r"(0u), "r"(kDescHi), "r"(lead) : "memory");
}
__device__ __forceinline__ void mma_commit(uint32_t lead, uint32_t bar) {
  asm volatile(
      "{\n\t"
      ".reg .pred l;\n\t"
      "setp.ne.b32 l, %1, 0;\n\t"
      "@l tcgen05.commit.cta_group::1.mbarrier::arrive::one.shared::cluster.b64 [%0];\n\t"
      "}\n"
      :: "r"(bar), "r"(lead) : "memory");
}
__device__ __forceinline__ void fence_before() { asm volatile("tcgen05.fence::before_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_after() { asm volatile("tcgen05.fence::after_thread_sync;" ::: "memory"); }
__device__ __forceinline__ void fence_proxy_async() { asm volatile("fence.proxy.async.shared::cta;" ::: "memory"); }
__device__ __forceinline__ void bar_init(uint32_t bar, uint32_t count) {
  asm volatile("mbarrier.init.shared::cta.b64 [%0], %1;" :: "r"(bar), "r"(count) : "memory");
}
__device__ __forceinline__ void bar_arrive(uint32_t bar) {
  asm volatile("mbarrier.arrive.shared::cta.b64 _, [%0];" :: "r"(bar) : "memory");
}
__device__ __forceinline__ void bar_arrive_tx(uint32_t lead, uint32_t bar, uint32_t bytes) {
  asm volatile(
      "{\n\t"
      ".reg .pred l;\n\t"
      "setp.ne.b32 l, %2, 0;\n\t"
      "@l mbarrier.arrive.expect_tx.shared::cta.b64 _, [%0], %1;\n\t"
      "}\n"
      :: "r"(bar), "r"(bytes), "r"(lead) : "memory");
}
__device__ __forceinline__ bool bar_try(uint32_t bar, uint32_t parity) {
  uint32_t ok;
  asm volatile(
      "{\n\t"
      ".reg .pred p;\n\t"
      "mbarrier.try_wait.parity.shared::cta.b64 p, [%1], %2;\n\t"
      "selp.u32 %0, 1, 0, p;\n\t"
      "}\n"
      : "=r"(ok) : "r"(bar), "r"(parity) : "memory");
  return ok != 0;
}
// bounded wait (about a second): false on time-out
__device__ __forceinline__ bool bar_wait(uint32_t bar, uint32_t parity) {
  if (bar_try(bar, parity)) return true;
  const long long t0 = clock64();
  while (!bar_try(bar, parity))
    if (clock64() - t0 > 2000000000LL) return false;
  return true;
}
// the same for a whole warp, whose lanes agree on the answer
__device__ __forceinline__ bool warp_wait(uint32_t bar, uint32_t parity) { return __all_sync(0xffffffffu, bar_wait(bar, parity)); }
// A warp's wait that spans items: the warps that load queries and store outputs wait for all of an item, softmax warps of a half
// without rows for the next one, and with tables of 2^31 tokens an item is 2^25 tiles (half a minute).  It ends when a wait of
// another warp, for a tile, ran out, and by itself after minutes.
__device__ __forceinline__ bool warp_wait_long(const uint32_t& failed, uint32_t bar, uint32_t parity) {
  bool ok = bar_try(bar, parity);
  if (!ok) {
    const long long t0 = clock64();
    while (!(ok = bar_try(bar, parity)))
      if (*(const volatile uint32_t*)&failed || clock64() - t0 > (1LL << 39)) break;
  }
  return __all_sync(0xffffffffu, ok);
}
__device__ __forceinline__ void tma_load(uint32_t lead, uint32_t dst, const CUtensorMap* map, int x, int y, uint32_t bar) {
  asm volatile(
      "{\n\t"
      ".reg .pred l;\n\t"
      "setp.ne.b32 l, %5, 0;\n\t"
      "@l cp.async.bulk.tensor.2d.shared::cta.global.tile.mbarrier::complete_tx::bytes [%0], [%1, {%2, %3}], [%4];\n\t"
      "}\n"
      :: "r"(dst), "l"(map), "r"(x), "r"(y), "r"(bar), "r"(lead) : "memory");
}
// contiguous bytes (a multiple of 16, both addresses too)
__device__ __forceinline__ void bulk_load(uint32_t lead, uint32_t dst, const void* src, uint32_t bytes, uint32_t bar) {
  asm volatile(
      "{\n\t"
      ".reg .pred l;\n\t"
      "setp.ne.b32 l, %4, 0;\n\t"
      "@l cp.async.bulk.shared::cluster.global.mbarrier::complete_tx::bytes [%0], [%1], %2, [%3];\n\t"
      "}\n"
      :: "r"(dst), "l"(src), "r"(bytes), "r"(bar), "r"(lead) : "memory");
}
__device__ __forceinline__ void tmem_ld32(uint32_t taddr, uint32_t* r) {
  asm volatile(
      "tcgen05.ld.sync.aligned.32x32b.x32.b32 "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31}, [%32];\n"
      : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]), "=r"(r[4]), "=r"(r[5]), "=r"(r[6]), "=r"(r[7]),
        "=r"(r[8]), "=r"(r[9]), "=r"(r[10]), "=r"(r[11]), "=r"(r[12]), "=r"(r[13]), "=r"(r[14]), "=r"(r[15]),
        "=r"(r[16]), "=r"(r[17]), "=r"(r[18]), "=r"(r[19]), "=r"(r[20]), "=r"(r[21]), "=r"(r[22]), "=r"(r[23]),
        "=r"(r[24]), "=r"(r[25]), "=r"(r[26]), "=r"(r[27]), "=r"(r[28]), "=r"(r[29]), "=r"(r[30]), "=r"(r[31])
      : "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_st32(uint32_t taddr, const uint32_t* r) {
  asm volatile(
      "tcgen05.st.sync.aligned.32x32b.x32.b32 [%32], "
      "{%0, %1, %2, %3, %4, %5, %6, %7, %8, %9, %10, %11, %12, %13, %14, %15, "
      "%16, %17, %18, %19, %20, %21, %22, %23, %24, %25, %26, %27, %28, %29, %30, %31};\n"
      :: "r"(r[0]), "r"(r[1]), "r"(r[2]), "r"(r[3]), "r"(r[4]), "r"(r[5]), "r"(r[6]), "r"(r[7]),
         "r"(r[8]), "r"(r[9]), "r"(r[10]), "r"(r[11]), "r"(r[12]), "r"(r[13]), "r"(r[14]), "r"(r[15]),
         "r"(r[16]), "r"(r[17]), "r"(r[18]), "r"(r[19]), "r"(r[20]), "r"(r[21]), "r"(r[22]), "r"(r[23]),
         "r"(r[24]), "r"(r[25]), "r"(r[26]), "r"(r[27]), "r"(r[28]), "r"(r[29]), "r"(r[30]), "r"(r[31]),
         "r"(taddr) : "memory");
}
__device__ __forceinline__ void tmem_wait_ld() { asm volatile("tcgen05.wait::ld.sync.aligned;" ::: "memory"); }
__device__ __forceinline__ void tmem_wait_st() { asm volatile("tcgen05.wait::st.sync.aligned;" ::: "memory"); }

__device__ __forceinline__ uint32_t pack_bf16(float a, float b) {
  const __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *(const uint32_t*)&v;
}

constexpr int kMaxSmem = 227 * 1024;

// What of an item belongs to this CTA, worked out once, by the warp that is ahead of all others (the roles' own arithmetic
// would be most of the kernel's instructions, and all of it is fetched for a single item).
struct Item {
  int last;                              // there is none: the roles leave
  int layer, h, b;
  int pos0;                              // position of the item's first new token
  int n, see[2];                         // tokens that the last row sees, and the first row of each half
  int t0, tiles, end[2];                 // first tile, tiles, and how many of them each half has
  int rows[2];                           // of queries, of each half
  int whole, first;                      // all of the item's tiles; its first tile
  int64_t q_at, out_at, lse_at;          // of the first token and query head, in elements
};
constexpr int kItems = 2;                // handed out and not yet taken by all

template <int SLOTS, int STAGES>
struct Shared {
  // full, empty: a slot holds an operand, may be overwritten.  s_full, p_full: S of a half is there, P is (two tiles each).
  // o_done: the item's last product has been added to O; o_full: the last but one; o_empty: O has been read.  q_full, q_empty: the
  // same of the queries.  stats_full: m and l.  left: all products are done.
  uint64_t full[SLOTS], empty[SLOTS], s_full[2][2], p_full[2][2], o_full[2], o_done[2], o_empty[2], q_full[2], q_empty[2], stats_full[2], raw, left[2];
  uint64_t st_full[STAGES], st_empty[STAGES], item_full[kItems], item_empty[kItems];
  uint32_t tmem, failed;
  // The loads are at most 8 tiles ahead of what is in use, and kItems + 1 items ahead of the outputs.
  uint8_t pages[16];                     // of the tiles under way: the tile's page is there
  uint8_t bad[4 * kItems];               // of the items under way: a value that some rows do not see is a NaN or an infinity
  Item items[kItems];
  uint8_t stage_there[STAGES];           // the stage holds a page's rows
  float stats[2][2][kHalf];              // of a half's rows: m, l as in a record
};

// ---- what depends on the format and the head dimension
constexpr int KT = kPageTokens;          // tokens of a tile

template <int D, int FMT>
struct Shape {
  static constexpr bool kInt4 = FMT == THINK_PAGE_INT4, kPlain = FMT == THINK_PAGE_PLAIN;
  static constexpr int PARTS = kInt4 ? 2 : 1;                 // bf16 operands that a key or value is the sum of
  static constexpr int kPart = KT * D * 2, kSlot = PARTS * kPart, kQBytes = 2 * kHalf * D * 2;
  static constexpr int RB = kPlain ? D * 2 : kInt4 ? D / 2 : D;       // bytes of a stored row
  static constexpr int SB = kPlain ? 0 : kInt4 ? D / 16 : 1;          // bytes of its scales
  // quantised pages: 64 stored rows and their scales a stage
  static constexpr int kBlock = 2 * kPageTokens * (RB + SB), kStage = kPlain ? 0 : kBlock / 2;
  static constexpr int kStages = kPlain ? 2 : 4;              // (of no bytes with bf16 pages)
  static constexpr int kSlots = (D == 64 ? 16 : kPlain ? 10 : 8) / PARTS;
  using Sh = Shared<kSlots, kStages>;
  static constexpr int kStageAt = kQBytes + kSlots * kSlot, kSharedAt = kStageAt + kStages * kStage, kSmem = kSharedAt + (int)sizeof(Sh);
  static_assert(kSharedAt % 16 == 0 && kSmem <= kMaxSmem, "shared memory");
  // Warps: two halves' softmax; bf16 pages: loads and products, else unpacking, products and fetching; rows.  Eight warps unpack e4m3
  // (8 rows over 131072 tokens, twice: 270 us with four, 254 with eight; long and ragged calls the same), four 4 bits (287 and 293 us).
  static constexpr int kUnpackWarps = kPlain ? 0 : kInt4 ? 4 : 8;
  static constexpr int kMmaWarp = kPlain ? 10 : 8 + kUnpackWarps, kFetchWarp = kMmaWarp + 2, kRowsWarp = 12 + kUnpackWarps;
  static constexpr int kThreads = 32 * (kRowsWarp + 4);
  // registers a thread: at launch, and as the roles have them
  static constexpr int kRegs = kPlain ? 128 : kInt4 ? 96 : 80;
  static constexpr int kSoftmaxRegs = kPlain ? 152 : kInt4 ? 128 : 120, kLoadRegs = kPlain ? 96 : kInt4 ? 80 : 56;
  static constexpr int kMmaRegs = kPlain ? 96 : kInt4 ? 64 : 56, kRowsRegs = kPlain ? 112 : kInt4 ? 80 : 72;
  static_assert(8 * kSoftmaxRegs + kUnpackWarps * kLoadRegs + 4 * kMmaRegs + 4 * kRowsRegs <= kRegs * kThreads / 32, "more registers than the block has: a wait without end");
  // tensor memory: S of each half, twice, O of each half
  static constexpr int kColO = 4 * KT;
  static __host__ __device__ constexpr PromptCut cut() { return PromptCut{kExtra}; }
};

// byte offset of 16-byte chunk ck of row r in an operand of `rows` rows: 64-channel blocks of 128-byte rows, swizzled
__device__ __forceinline__ uint32_t swz(int rows, int r, int ck) {
  return (uint32_t)((ck >> 3) * rows * 128 + r * 128 + (((ck & 7) ^ (r & 7)) << 4));
}
__device__ __forceinline__ void st_shared(uint32_t at, const uint4& w) {
  asm volatile("st.shared.v4.b32 [%0], {%1, %2, %3, %4};" :: "r"(at), "r"(w.x), "r"(w.y), "r"(w.z), "r"(w.w) : "memory");
}
__device__ __forceinline__ uint4 ld_shared(uint32_t at) {
  uint4 w;
  asm volatile("ld.shared.v4.b32 {%0, %1, %2, %3}, [%4];" : "=r"(w.x), "=r"(w.y), "=r"(w.z), "=r"(w.w) : "r"(at) : "memory");
  return w;
}
__device__ __forceinline__ uint32_t ld_shared16(uint32_t at) {
  uint16_t x;
  asm volatile("ld.shared.u16 %0, [%1];" : "=h"(x) : "r"(at) : "memory");
  return x;
}
__device__ __forceinline__ uint32_t ld_shared8(uint32_t at) {
  uint32_t x;
  asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(at) : "memory");
  return x;
}
// Sets the NaN and infinite ones of 8 bf16 to 0; whether there were any.
__device__ __forceinline__ bool drop_non_finite(uint4& w) {
  bool any = false;
  uint32_t* const u = &w.x;
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    const bool lo = (u[i] & 0x7f80u) == 0x7f80u, hi = (u[i] & 0x7f800000u) == 0x7f800000u;
    any |= lo | hi;
    u[i] &= (lo ? 0u : 0xffffu) | (hi ? 0u : 0xffff0000u);
  }
  return any;
}

// 4 e4m3 codes times a power of two as bf16 (exact)
__device__ __forceinline__ uint2 e4m3_to_bf16(uint32_t w, float s) {
  const __half2_raw a = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w & 0xffffu), __NV_E4M3);
  const __half2_raw b = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(w >> 16), __NV_E4M3);
  float2 x = __half22float2(*(const __half2*)&a), y = __half22float2(*(const __half2*)&b);
  split(mul2(two(x.x, x.y), two(s, s)), x.x, x.y);
  split(mul2(two(y.x, y.y), two(s, s)), y.x, y.y);
  return make_uint2(pack_bf16(x.x, x.y), pack_bf16(y.x, y.y));
}
// 8 4-bit codes times their scale (bf16, twice) as the sum of two bf16: the product rounded, and what the rounding took away
// (n s has 11 bits, so the rest fits).  Channels come out in the order 0 4 1 5 2 6 3 7, which saves sorting them: queries are
// permuted alike, and outputs back.  7 s may round past the largest bf16 number (a group whose largest magnitude is that number):
// the first part ends there, and the second has what is missing, exactly as long as it fits (|n s| < 2^129 - 2^121).  BOUND:
// what does not fit, which no written row holds, ends at that number too, for a value that some rows must not meet as infinite.
constexpr uint32_t kMostBf16 = 0x7f7f7f7fu;
template <bool BOUND>
__device__ __forceinline__ void int4_to_bf16(uint32_t w, uint32_t s2, uint4& hi, uint4& lo) {
  uint32_t h[4], l[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    uint32_t n;
    asm("add.rn.bf16x2 %0, %1, %2;" : "=r"(n) : "r"(((w >> (4 * i)) & 0x000f000fu) | 0x43004300u), "r"(0xc308c308u));      // (128 + c) - 136
    asm("mul.rn.bf16x2 %0, %1, %2;" : "=r"(h[i]) : "r"(n), "r"(s2));
    asm("min.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(h[i]) : "r"(kMostBf16));      // (a NaN scale: the second part is NaN)
    asm("fma.rn.bf16x2 %0, %1, %2, %3;" : "=r"(l[i]) : "r"(n), "r"(s2), "r"(h[i] ^ 0x80008000u));
    if (BOUND) asm("min.NaN.xorsign.abs.bf16x2 %0, %0, %1;" : "+r"(l[i]) : "r"(kMostBf16));
  }
  hi = make_uint4(h[0], h[1], h[2], h[3]);
  lo = make_uint4(l[0], l[1], l[2], l[3]);
}
__device__ __forceinline__ constexpr int int4_channel(int j) { return (j & ~7) | ((j & 1) << 2) | ((j >> 1) & 3); }
__device__ __forceinline__ uint4 int4_order(const uint4& v) {          // 8 channels of a query
  return make_uint4(__byte_perm(v.x, v.z, 0x5410), __byte_perm(v.x, v.z, 0x7632), __byte_perm(v.y, v.w, 0x5410), __byte_perm(v.y, v.w, 0x7632));
}

// A value of the pool that is a NaN or an infinity, as fp32, or 0: for the few that are looked at one by one.  (A 4-bit one of a
// finite scale is finite.)
template <int D, int FMT>
__device__ float non_finite_value(const uint8_t* block, int slot, int c) {
  using T = Shape<D, FMT>;
  const uint8_t* const row = block + (kPageTokens + slot) * T::RB;
  const uint8_t* const sc = block + 2 * kPageTokens * T::RB + (kPageTokens + slot) * T::SB;
  float v, by = 1.f;
  if constexpr (T::kPlain) {
    v = __uint_as_float((uint32_t)((const uint16_t*)row)[c] << 16);
  } else if constexpr (FMT == THINK_PAGE_E4M3) {
    const __half_raw h = __nv_cvt_fp8_to_halfraw(row[c], __NV_E4M3);
    v = __half2float(*(const __half*)&h) * e8m0(*sc);
  } else {
    v = __uint_as_float((uint32_t)((const uint16_t*)sc)[c / kGroupChannels] << 16);
    by = (float)((row[c / 2] >> (4 * (c & 1)) & 15) - 8);
  }
  return fabsf(v) <= 3.402823466e38f ? 0.f : v * by;
}

template <typename T>
__device__ __forceinline__ void describe(const PagedPromptParams& p, const PromptWalk& w, const PromptPiece& x, Item& o) {
  const int ll = p.by_heads.div(w.lh), h = w.lh - ll * p.g.N_kv, rows = x.tokens * p.G;
  o.last = 0;
  o.layer = p.layer0 + ll;
  o.h = h;
  o.b = w.b;
  o.pos0 = w.s.pos + x.s0;
  o.n = x.n;
  o.t0 = x.t0;
  o.tiles = x.t1 - x.t0;
#pragma unroll
  for (int i = 0; i < 2; ++i) {
    const int r = max(0, min(kHalf, rows - i * kHalf));
    const int first = o.pos0 + (int)p.by_group.div(i * kHalf), last = o.pos0 + (int)p.by_group.div(i * kHalf + max(r, 1) - 1);
    const int n = max(0, min(x.n, last + 1));          // tokens that the half sees
    o.rows[i] = r;
    o.see[i] = first + 1;
    o.end[i] = r == 0 ? 0 : max(0, min(x.t1, max(1, (n + KT - 1) / KT)) - x.t0);
  }
  o.whole = x.t0 == 0 && x.t1 == x.tiles;
  o.first = x.t0 == 0;
  o.q_at = prompt_row(p, p.q, w.b, w.s, x.s0) + ll * p.q.sl + h * p.G * p.q.sn;
  o.out_at = prompt_row(p, p.out, w.b, w.s, x.s0) + ll * p.out.sl + h * p.G * p.out.sn;
  o.lse_at = (prompt_lse_row(p, w.b, w.s, x.s0) * p.nlayers + ll) * p.N_q + h * p.G;
}

// Items as the warp that walks along them hands them out, and as the others take them.
struct Items {
  int no;
  __device__ __forceinline__ uint32_t phase() const { return no / kItems & 1; }
  // The next item; false on a time-out.  Every lane has its own copy of what it uses before the place is given back.
  template <bool LONG = false, typename Sh, typename F>
  __device__ __forceinline__ bool take(Sh& sh, F copy) {
    const int slot = no & (kItems - 1);
    if (!(LONG ? warp_wait_long(sh.failed, smem_u32(&sh.item_full[slot]), phase()) : warp_wait(smem_u32(&sh.item_full[slot]), phase()))) return false;
    copy(*(const Item*)&sh.items[slot]);
    __syncwarp();
    if ((threadIdx.x & 31) == 0) bar_arrive(smem_u32(&sh.item_empty[slot]));
    return true;
  }
};
// The warp that walks.
struct Walker {
  PromptWalk w;
  PromptDesc desc;
  int64_t cost;
  int state;                  // 0: at a new item, 1: on to the next one, 2: at the end
  __device__ __forceinline__ void begin(const PagedPromptParams& p, const PromptCut& cut) {
    desc = PromptDesc{0, 0, 0, 0, 0};
    state = prompt_walk_begin(p, cut, w) ? 0 : 2;
  }
  // hands out the next item that has tiles here, or says that there is none
  template <typename T>
  __device__ __forceinline__ bool hand_out(const PagedPromptParams& p, typename T::Sh& sh, int no) {
    constexpr PromptCut cut = T::cut();
    PromptPiece x;
#pragma unroll 1
    while (state < 2) {
      if (state == 1 && !prompt_walk_next(p, cut, w, cost)) {
        state = 2;
        break;
      }
      state = 1;
      x = prompt_piece(p, cut, w);
      cost = x.cost;
      if (x.t0 != x.t1) break;
    }
    const int slot = no & (kItems - 1);
    if (!warp_wait(smem_u32(&sh.item_empty[slot]), (no / kItems & 1) ^ 1)) return false;
    if ((threadIdx.x & 31) == 0) {
      if (state < 2) {
        describe<T>(p, w, x, sh.items[slot]);
        if (x.t0 > 0) desc.carries = x.t1 == x.tiles ? 1 : 2;
        else if (x.t1 != x.tiles) desc = PromptDesc{w.lh, w.b, w.i, 1, desc.carries};
      } else {
        sh.items[slot].last = 1;
        p.desc[blockIdx.x] = desc;
      }
      bar_arrive(smem_u32(&sh.item_full[slot]));
    }
    __syncwarp();
    return true;
  }
};

struct Ring {                 // position in the ring of slots
  int slot;
  uint32_t phase;
  template <typename T>
  __device__ __forceinline__ void next() {
    if (++slot == T::kSlots) {
      slot = 0;
      phase ^= 1;
    }
  }
};

// The pool's blocks (of a layer and key head) that hold a sequence's pages, 32 at a time in the lanes of a warp, the next ones
// on their way.
struct PageWindow {
  int32_t now, next;          // block; -1: no page of the pool
  int first;                  // page of the sequence that lane 0 holds
  __device__ __forceinline__ int32_t fetch(const PagedPromptParams& p, int b, int layer, int h, int at, int pages) const {
    const int i = at + (threadIdx.x & 31);
    if (i >= pages) return -1;
    const int32_t page = load_now(p.table.table + b * p.table.stride + i);
    if ((uint32_t)page >= (uint32_t)p.g.num_pages) {
      atomicOr(p.error, kErrPage);
      return -1;
    }
    return (layer * p.g.num_pages + page) * p.g.N_kv + h;          // fits 32 bits: a block has 4608 bytes at least
  }
  __device__ __forceinline__ void begin(const PagedPromptParams& p, int b, int layer, int h, int page, int pages) {
    first = page;
    now = fetch(p, b, layer, h, first, pages);
    next = fetch(p, b, layer, h, first + 32, pages);
  }
  // of page i of the sequence (i grows)
  __device__ __forceinline__ int at(const PagedPromptParams& p, int b, int layer, int h, int i, int pages) {
    if (i - first >= 32) {
      first += 32;
      now = next;
      next = fetch(p, b, layer, h, first + 32, pages);
    }
    return __shfl_sync(0xffffffffu, now, i - first);
  }
};

// The order of an item's operands, in which they are loaded, unpacked and used: keys two tiles ahead of values.
//   for j = 0 .. tiles + 1:   values of tile j - 2 if there is one, keys of tile j if there is one

// ---- bf16 pages: a warp brings keys, one values, by TMA
template <int D, int FMT>
__device__ __forceinline__ bool load_role(const PagedPromptParams& p, const CUtensorMap* map, typename Shape<D, FMT>::Sh& sh, uint32_t ring0, int part) {
  using T = Shape<D, FMT>;
  const int lane = threadIdx.x & 31;
  const uint32_t lead = elect_lane(), raw = smem_u32(&sh.raw);
  Ring r{0, 0};
  PageWindow win;
  uint32_t raw_phase = 0;
  int tile_no = 0;
  Items items{0};
  Walker walk;
  if (part == 0) walk.begin(p, T::cut());
  for (;; ++items.no) {
    if (part == 0 && !walk.template hand_out<T>(p, sh, items.no)) return false;
    int last, layer, h, b, n, see, t0, tiles;
    if (!items.take(sh, [&](const Item& i) { last = i.last; layer = i.layer; h = i.h; b = i.b; n = i.n; see = i.see[0]; t0 = i.t0; tiles = i.tiles; })) return false;
    if (last) return true;
    const int pages = (n + 63) >> 6;
    win.begin(p, b, layer, h, t0, pages);
#pragma unroll 1
    for (int j = 0; j < tiles + 2; ++j) {
      if (part == 0 && j >= 2) r.template next<T>();
      const int i = part ? j - 2 : j;
      if (i >= 0 && i < tiles) {
        const int block = win.at(p, b, layer, h, t0 + i, pages), tok0 = (t0 + i) * KT;
        const bool edge = part == 1 && (tok0 + KT > see || block < 0);          // some values must not be met
        const uint32_t to = ring0 + r.slot * T::kSlot, full = smem_u32(&sh.full[r.slot]), bar = edge ? raw : full;
        if (!warp_wait(smem_u32(&sh.empty[r.slot]), r.phase ^ 1)) return false;
        if (part == 0 && lane == 0) {
          sh.pages[tile_no & 15] = block >= 0;
          if (i == 0) sh.bad[(items.no + 2 * kItems) & (4 * kItems - 1)] = 0;
        }
        ++tile_no;
        __syncwarp();
        bar_arrive_tx(lead, bar, block >= 0 ? T::kSlot : 0);
        if (block >= 0) {
#pragma unroll
          for (int c = 0; c < D / 64; ++c) tma_load(lead, to + c * KT * 128, map, c * 64, block * 128 + part * 64, bar);
        }
        if (edge) {
          if (!warp_wait(raw, raw_phase)) return false;
          raw_phase ^= 1;
          // what is behind the last token or on no page becomes 0, what only some rows see finite
#pragma unroll 1
          for (int k = lane; k < KT; k += 32) {
            const bool off = tok0 + k >= n || block < 0;
            if (!off && tok0 + k < see) continue;
            bool any = false;
#pragma unroll 4
            for (int ck = 0; ck < D / 8; ++ck) {
              uint4 v = make_uint4(0u, 0u, 0u, 0u);
              if (!off) {
                v = ld_shared(to + swz(KT, k, ck));
                any |= drop_non_finite(v);
              }
              st_shared(to + swz(KT, k, ck), v);
            }
            if (any) sh.bad[items.no & (4 * kItems - 1)] = 1;
          }
          fence_proxy_async();
          __syncwarp();
          if (lane == 0) bar_arrive(full);
        }
        r.template next<T>();
      }
      if (part == 1 && j < tiles) r.template next<T>();
    }
  }
}

// ---- quantised pages: a warp has the bytes of keys copied to the stages, one those of values: 64 rows and their scales each
template <int D, int FMT>
__device__ __forceinline__ bool fetch_role(const PagedPromptParams& p, typename Shape<D, FMT>::Sh& sh, uint32_t stage0, int part) {
  using T = Shape<D, FMT>;
  const int lane = threadIdx.x & 31;
  const uint32_t lead = elect_lane();
  int stage = 0;
  uint32_t phase = 0;
  auto next = [&]() {
    if (++stage == T::kStages) {
      stage = 0;
      phase ^= 1;
    }
  };
  PageWindow win;
  Items items{0};
  Walker walk;
  if (part == 0) walk.begin(p, T::cut());
  for (;; ++items.no) {
    if (part == 0 && !walk.template hand_out<T>(p, sh, items.no)) return false;
    int last, layer, h, b, n, t0, tiles;
    if (!items.take(sh, [&](const Item& i) { last = i.last; layer = i.layer; h = i.h; b = i.b; n = i.n; t0 = i.t0; tiles = i.tiles; })) return false;
    if (last) return true;
    const int pages = (n + 63) >> 6;
    win.begin(p, b, layer, h, t0, pages);
#pragma unroll 1
    for (int j = 0; j < tiles + 2; ++j) {
      if (part == 0 && j >= 2) next();
      const int i = part ? j - 2 : j;
      if (i >= 0 && i < tiles) {
        const int block = win.at(p, b, layer, h, t0 + i, pages);
        const uint8_t* const src = p.pages + (int64_t)max(block, 0) * T::kBlock;
        if (!warp_wait(smem_u32(&sh.st_empty[stage]), phase ^ 1)) return false;
        const uint32_t bar = smem_u32(&sh.st_full[stage]), dst = stage0 + stage * T::kStage;
        if (lane == 0) sh.stage_there[stage] = block >= 0;
        __syncwarp();
        bar_arrive_tx(lead, bar, block >= 0 ? T::kStage : 0);
        if (block >= 0) {
          bulk_load(lead, dst, src + part * kPageTokens * T::RB, kPageTokens * T::RB, bar);
          bulk_load(lead, dst + kPageTokens * T::RB, src + kPageTokens * (2 * T::RB + part * T::SB), kPageTokens * T::SB, bar);
        }
        next();
      }
      if (part == 1 && j < tiles) next();
    }
  }
}

// ---- four or eight warps unpack the stages into the ring
// 64 stored rows at `from` to rows of the operand at `to` (of 64-channel blocks of KT rows).  A unit is 16 stored bytes: 16
// channels of e4m3, 32 of 4 bits.  by: a power of two that e4m3 rows are taken times.  EDGE: rows from `n` on become 0, those from `see` on finite; whether any was not.  (In a rolled
// loop: it comes too seldom to stay in the instruction cache; unrolled it took a ragged batch of 48 sequences 325 instead of 297 us.)
template <int D, int FMT, bool EDGE>
__device__ __forceinline__ bool unpack_rows(uint32_t from, uint32_t to, int n, int see, float by) {
  using T = Shape<D, FMT>;
  constexpr int CH = T::kInt4 ? 32 : 16, PER_ROW = D / CH, PASS = 32 * T::kUnpackWarps / PER_ROW, UNITS = (kPageTokens + PASS - 1) / PASS;
  constexpr int kUnroll = EDGE ? 1 : UNITS, kLoad = EDGE ? 1 : UNITS;
  static_assert(PASS % 8 == 0 && PASS <= kPageTokens, "the swizzle of a lane's rows is the same");
  const int tid = threadIdx.x & (32 * T::kUnpackWarps - 1), c = tid % PER_ROW, r0 = tid / PER_ROW;
  uint32_t src = from + r0 * T::RB + c * 16, ssrc = from + kPageTokens * T::RB + r0 * T::SB + (T::kInt4 ? 2 * c : 0);
  // neighbouring lanes store to different banks
  const int turn = T::kInt4 ? (c >> 1) ^ ((r0 & 1) << 1) : c >> 2 & 1;
  to += r0 * 128;
  bool any = false;
  uint4 w16[kLoad];
  uint32_t s16[kLoad];
#pragma unroll
  for (int u = 0; u < kLoad; ++u) {
    w16[u] = ld_shared(src + u * PASS * T::RB);
    s16[u] = T::kInt4 ? ld_shared16(ssrc + u * PASS * T::SB) : ld_shared8(ssrc + u * PASS * T::SB);
  }
#pragma unroll kUnroll
  for (int u = 0; u < UNITS; ++u) {
    const int row = r0 + u * PASS;
    uint4 w = w16[EDGE ? 0 : u];
    uint32_t sb = s16[EDGE ? 0 : u];
    if (EDGE && u + 1 < UNITS) {
      src += PASS * T::RB;
      ssrc += PASS * T::SB;
      w16[0] = ld_shared(src);
      s16[0] = T::kInt4 ? ld_shared16(ssrc) : ld_shared8(ssrc);
    }
    const uint32_t* const q = &w.x;
    if (EDGE && row >= n) {
      w = T::kInt4 ? make_uint4(0x88888888u, 0x88888888u, 0x88888888u, 0x88888888u) : make_uint4(0u, 0u, 0u, 0u);
      sb = 0;
    }
    if constexpr (T::kInt4) {
      const uint32_t s2 = sb | sb << 16;
      const bool drop = EDGE && row >= see && (sb & 0x7f80u) == 0x7f80u;
      any |= drop;
#pragma unroll
      for (int k = 0; k < 4; ++k) {
        const int kk = k ^ turn;
        const uint32_t word = kk & 2 ? (kk & 1 ? q[3] : q[2]) : (kk & 1 ? q[1] : q[0]);
        uint4 hi, lo;
        int4_to_bf16<EDGE>(word, s2, hi, lo);
        if (drop) hi = lo = make_uint4(0u, 0u, 0u, 0u);
        const uint32_t at = to + swz(KT, 0, (4 * c + kk) ^ (r0 & 7));
        st_shared(at, hi);
        st_shared(at + T::kPart, lo);
      }
    } else {
      const float sc = e8m0(sb) * by;
      uint4 v[2];
#pragma unroll
      for (int k = 0; k < 2; ++k) {
        const uint2 a = e4m3_to_bf16(q[2 * k], sc), b = e4m3_to_bf16(q[2 * k + 1], sc);
        v[k] = make_uint4(a.x, a.y, b.x, b.y);
      }
      if (EDGE && row >= see) {
        uint32_t sum = 0;                 // of products with 0: a NaN where one is not finite
#pragma unroll
        for (int k = 0; k < 8; ++k) {
          const uint32_t u = (&v[0].x)[k];
          asm("fma.rn.bf16x2 %0, %1, %2, %0;" : "+r"(sum) : "r"(u), "r"(0u));
        }
        if (sum & 0x7fff7fffu) any |= drop_non_finite(v[0]) | drop_non_finite(v[1]);
      }
      st_shared(to + swz(KT, 0, (2 * c + turn) ^ (r0 & 7)), turn ? v[1] : v[0]);
      st_shared(to + swz(KT, 0, (2 * c + !turn) ^ (r0 & 7)), turn ? v[0] : v[1]);
    }
    to += PASS * 128;
  }
  return any;
}

template <int D, int FMT>
__device__ __forceinline__ bool unpack_role(typename Shape<D, FMT>::Sh& sh, uint32_t ring0, uint32_t stage0, float by) {
  using T = Shape<D, FMT>;
  const int tid = threadIdx.x & (32 * T::kUnpackWarps - 1), lane = threadIdx.x & 31;
  Ring r{0, 0};
  int stage = 0, tile_no = 0;
  uint32_t phase = 0;
  Items items{0};
  for (;; ++items.no) {
    int last, n, see, t0, tiles;
    if (!items.take(sh, [&](const Item& i) { last = i.last; n = i.n; see = i.see[0]; t0 = i.t0; tiles = i.tiles; })) return false;
    if (last) return true;
#pragma unroll 1
    for (int k = 0; k < 2 * tiles + 4; ++k) {
      const int part = ~k & 1, i = part ? (k >> 1) - 2 : k >> 1;
      if (i < 0 || i >= tiles) continue;
      const int slot0 = r.slot, tok0 = (t0 + i) * KT;
      if (!warp_wait(smem_u32(&sh.empty[slot0]), r.phase ^ 1)) return false;
      r.template next<T>();
      if (!warp_wait(smem_u32(&sh.st_full[stage]), phase)) return false;
      const bool here = sh.stage_there[stage] != 0;
      const uint32_t from = stage0 + stage * T::kStage, to = ring0 + slot0 * T::kSlot;
      // rows that no row of queries sees become 0, values that only some see finite
      bool any = false;
      if (!here || tok0 + KT > (part ? see : n)) any = unpack_rows<D, FMT, true>(from, to, here ? n - tok0 : 0, part ? see - tok0 : KT, part ? 1.f : by);
      else unpack_rows<D, FMT, false>(from, to, KT, KT, part ? 1.f : by);
      if (part == 0) {
        if (tid == 0) {
          sh.pages[tile_no & 15] = here;
          if (i == 0) sh.bad[(items.no + 2 * kItems) & (4 * kItems - 1)] = 0;
        }
        ++tile_no;
      }
      if (any) sh.bad[items.no & (4 * kItems - 1)] = 1;
      fence_proxy_async();
      __syncwarp();
      if (lane == 0) {
        bar_arrive(smem_u32(&sh.st_empty[stage]));
        bar_arrive(smem_u32(&sh.full[slot0]));
      }
      if (++stage == T::kStages) {
        stage = 0;
        phase ^= 1;
      }
    }
  }
}

// ---- two warps: the products of a half each
// The tensor cores' queue is short and a wait costs 140 cycles even where there is nothing to wait for: two warps fill each
// other's gaps.
template <int D, int FMT>
__device__ __forceinline__ bool mma_role(typename Shape<D, FMT>::Sh& sh, uint32_t q0, uint32_t ring0, uint32_t tmem, int half) {
  using T = Shape<D, FMT>;
  constexpr uint32_t kIdQK = idesc(KT, false), kIdPV = idesc(D, true);
  const uint32_t lead = elect_lane();
  auto uniform = [](int v) { return __shfl_sync(0xffffffffu, v, 0); };
  half = uniform(half);
  ring0 = uniform(ring0);
  tmem = uniform(tmem);
  q0 = uniform(q0) + half * (kHalf * D * 2);
  const uint32_t full = uniform(smem_u32(sh.full)), empty = uniform(smem_u32(sh.empty));
  const uint32_t s_full = uniform(smem_u32(&sh.s_full[half][0])), p_full = uniform(smem_u32(&sh.p_full[half][0]));
  const uint32_t o_full = uniform(smem_u32(&sh.o_full[half])), o_done = uniform(smem_u32(&sh.o_done[half]));
  const uint32_t o_empty = uniform(smem_u32(&sh.o_empty[half])), q_full = uniform(smem_u32(&sh.q_full[half])), q_empty = uniform(smem_u32(&sh.q_empty[half]));
  const uint32_t tS = tmem + half * 2 * KT, tO = tmem + T::kColO + half * D;
  uint32_t p_phase = 0, q_phase = 0, e_phase = 1;      // p_phase: a bit for each of the two tiles
  Ring r{0, 0};                         // of the next operand
  // this half is through with the operand: behind its products, or where it has none, now
  auto release = [&](bool used) {
    if (used) mma_commit(lead, empty + r.slot * 8);
    else if (lead) bar_arrive(empty + r.slot * 8);
    r.template next<T>();
  };
  auto qk = [&](int buf) {
#pragma unroll
    for (int part = 0; part < T::PARTS; ++part) {
      const uint32_t k = desc_lo(ring0 + r.slot * T::kSlot + part * T::kPart, 16), q = desc_lo(q0, 16);
#pragma unroll
      for (int ks = 0; ks < D / 16; ++ks)
        mma_ss(lead, tS + buf * KT, q + (ks >> 2) * (kHalf * 8) + (ks & 3) * 2, k + (ks >> 2) * (KT * 8) + (ks & 3) * 2, kIdQK, part > 0 || ks > 0);
    }
    mma_commit(lead, s_full + buf * 8);
  };
  auto pv = [&](int buf, uint32_t accumulate) {
#pragma unroll
    for (int part = 0; part < T::PARTS; ++part) {
      const uint32_t v = desc_lo(ring0 + r.slot * T::kSlot + part * T::kPart, KT * 128);
#pragma unroll
      for (int ks = 0; ks < 4; ++ks) mma_ts(lead, tO, tS + buf * KT + ks * 8, v + ks * 128, kIdPV, part > 0 || ks > 0 ? 1u : accumulate);
    }
  };
  Items items{0};
  for (;; ++items.no) {
    int last, tiles, n;                 // n: tiles of this half
    if (!items.take(sh, [&](const Item& i) { last = i.last; tiles = i.tiles; n = i.end[half]; })) return false;
    if (uniform(last)) break;
    tiles = uniform(tiles);
    n = uniform(n);
#pragma unroll 1
    for (int j = 0; j < tiles + 2; ++j) {
      const int buf = j & 1;
      if (j >= 2) {                     // values of tile j - 2
        if (!warp_wait(full + r.slot * 8, r.phase)) return false;
        if (j - 2 < n) {
          if (j == 2) {
            if (!warp_wait(o_empty, e_phase)) return false;
            e_phase ^= 1;
          }
          if (!warp_wait(p_full + buf * 8, p_phase >> buf & 1)) return false;
          p_phase ^= 1u << buf;
          fence_after();
          pv(buf, j - 2);
          if (j == n) mma_commit(lead, o_full);         // of the last tile but one: see the softmax
          if (j - 1 == n) mma_commit(lead, o_done);
        }
        release(j - 2 < n);
      }
      if (j < tiles) {                  // keys of tile j: S takes the place of P of tile j - 2
        if (!warp_wait(full + r.slot * 8, r.phase)) return false;
        if (j < n) {
          if (j == 0) {
            if (!warp_wait(q_full, q_phase)) return false;
            q_phase ^= 1;
            fence_after();
          }
          qk(buf);
          if (j + 1 == n) mma_commit(lead, q_empty);
        }
        release(j < n);
      }
    }
  }
  // all that was committed has arrived before the block leaves, and its barriers with it
  const uint32_t left = uniform(smem_u32(&sh.left[half]));
  mma_commit(lead, left);
  return warp_wait(left, 0);
}

// ---- warps 0-3, 4-7: the softmax of a half
template <int D, int FMT>
__device__ __forceinline__ bool softmax_role(const PagedPromptParams& p, typename Shape<D, FMT>::Sh& sh, uint32_t tmem) {
  using T = Shape<D, FMT>;
  const int half = threadIdx.x >> 7, row = threadIdx.x & 127, lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) & 3;
  const uint32_t lanes = (uint32_t)(warp * 32) << 16;
  const uint32_t tS = tmem + lanes + half * 2 * KT, tO = tmem + lanes + T::kColO + half * D;
  const uint32_t s_full = smem_u32(&sh.s_full[half][0]), p_full = smem_u32(&sh.p_full[half][0]), o_full = smem_u32(&sh.o_full[half]);
  const int s = p.by_group.div(half * kHalf + row);    // token of the row in its item
  uint32_t s_phase = 0, o_phase = 0, e_phase = 1;
  int tile_no = 0;
  Items items{0};
  for (;; ++items.no) {
    int last, rows, see, n, pos0, t0, tiles, end;
    if (!items.take<true>(sh, [&](const Item& i) {
          last = i.last; rows = i.rows[half]; see = i.see[half]; n = i.n; pos0 = i.pos0; t0 = i.t0; tiles = i.tiles; end = i.end[half];
        })) return false;
    if (last) return true;
    const int limit = row < rows ? min(n, pos0 + s + 1) : 0;       // tokens that the row sees
    int i = 0;
    if (warp * 32 >= rows) {            // no row: P stays what it is, and what becomes of it is not looked at
#pragma unroll 1
      for (; i < end; ++i) {
        if (!warp_wait(s_full + (i & 1) * 8, s_phase >> (i & 1) & 1)) return false;
        s_phase ^= 1u << (i & 1);
        if (lane == 0) bar_arrive(p_full + (i & 1) * 8);
      }
    }
    float m = -INFINITY, l = 0.f, lc = 0.f;            // lc: what the additions to l have lost
    float ref = 0.f, scale = p.scale_log2;             // weights: 2^(scale S + ref)
    bool seen = false;
#pragma unroll 1
    for (; i < end; ++i) {
      const int buf = i & 1, tok0 = (t0 + i) * KT;
      if (!warp_wait(s_full + buf * 8, s_phase >> buf & 1)) return false;
      s_phase ^= 1u << buf;
      fence_after();
      const uint32_t tP = tS + buf * KT;
      uint32_t sr[KT];
#pragma unroll
      for (int j = 0; j < KT; j += 32) tmem_ld32(tP + j, sr + j);
      const bool here = sh.pages[(tile_no + i) & 15];
      tmem_wait_ld();
      if (tok0 + KT > see || !here) {                   // some tokens are not seen
        const int stop = here ? limit - tok0 : 0;
        seen |= stop > 0;
#pragma unroll
        for (int j = 0; j < KT; ++j)
          if (j >= stop) sr[j] = 0xff800000u;
      } else {
        seen = true;
      }
      float mx[4] = {-INFINITY, -INFINITY, -INFINITY, -INFINITY};
#pragma unroll
      for (int j = 0; j < KT; j += 8)
#pragma unroll
        for (int i = 0; i < 4; ++i) mx[i] = max3(mx[i], __uint_as_float(sr[j + 2 * i]), __uint_as_float(sr[j + 2 * i + 1]));
      const float top = max3(fmaxf(mx[0], mx[1]), mx[2], mx[3]) * p.scale_log2;
      if (__any_sync(0xffffffffu, top > m)) {           // see kAbove
        const float m_new = fmaxf(m, top + kAbove);
        const float f = m == m_new ? 1.f : ex2(m - m_new);
        if (i > 0) {
          // the product before this tile's is done when the logits of the next tile are, which are computed behind it; in the
          // last tile it has a barrier of its own
          if (!(i + 1 < end ? warp_wait(s_full + (buf ^ 1) * 8, s_phase >> (buf ^ 1) & 1) : warp_wait(o_full, o_phase))) return false;
          fence_after();
#pragma unroll 1
          for (int k = 0; k < D; k += 32) {
            uint32_t o[32];
            tmem_ld32(tO + k, o);
            tmem_wait_ld();
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = __float_as_uint(__uint_as_float(o[j]) * f);
            tmem_st32(tO + k, o);
          }
        }
        l *= f;
        lc *= f;
        m = m_new;
        // A logit minus m is exact up to one rounding, but m itself is rounded: from 2^27 on (where logits that differ are 16 and
        // more apart) both are taken so many times smaller that the rounding stays below 2^4.
        const int e = (int)(__float_as_uint(m) >> 23 & 255);
        const float less = __uint_as_float((uint32_t)(127 - (e < 255 ? max(0, e - (127 + 27)) : 0)) << 23);
        scale = p.scale_log2 * less;
        ref = m == -INFINITY ? 0.f : -m * less;
      }
      const f32x2 ref2 = two(ref, ref), scale2 = two(scale, scale);
      f32x2 ls[2] = {0ull, 0ull};
      uint32_t pk[KT / 2];
#pragma unroll
      for (int j = 0; j < KT / 2; ++j) {
        float a, b;
        split(fma2(two(__uint_as_float(sr[2 * j]), __uint_as_float(sr[2 * j + 1])), scale2, ref2), a, b);
        a = ex2(a);
        b = ex2(b);
        ls[j & 1] = add2(ls[j & 1], two(a, b));
        pk[j] = pack_bf16(a, b);
      }
      tmem_st32(tP, pk);
      tmem_wait_st();
      fence_before();
      __syncwarp();
      if (lane == 0) bar_arrive(p_full + buf * 8);
      float a0, a1;
      split(add2(ls[0], ls[1]), a0, a1);
      const float add = (a0 + a1) - lc, sum = l + add;
      lc = (sum - l) - add;
      l = sum;
    }
    tile_no += tiles;
    if (end > 1) o_phase ^= 1;
    if (end > 0) {
      if (!warp_wait(smem_u32(&sh.o_empty[half]), e_phase)) return false;     // the last item's have been read
      e_phase ^= 1;
      sh.stats[half][0][row] = m;
      sh.stats[half][1][row] = m == -INFINITY && l == 0.f ? (seen ? 1.f : 0.f) : l;
      __syncwarp();
      if (lane == 0) bar_arrive(smem_u32(&sh.stats_full[half]));
    }
  }
}

// ---- four warps: the next item's queries, the last item's outputs
template <int D, int FMT>
__device__ __forceinline__ bool rows_role(const PagedPromptParams& p, typename Shape<D, FMT>::Sh& sh, uint32_t q0, uint32_t tmem) {
  using T = Shape<D, FMT>;
  const int row = threadIdx.x & 127, lane = threadIdx.x & 31, warp = (threadIdx.x >> 5) & 3;
  const uint32_t lanes = tmem + ((uint32_t)(warp * 32) << 16);
  uint32_t phases = 0;                  // bit h: q_empty, 2 + h: stats_full, 4 + h: o_done
  Items items{0};
  Item it;
  it.last = 1;
  for (;; ++items.no) {
    Item next;
    if (!items.take<true>(sh, [&](const Item& i) { next = i; })) return false;
    if (!next.last) {
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        if ((half ? next.end[1] : next.end[0]) == 0) continue;
        if (!warp_wait_long(sh.failed, smem_u32(&sh.q_empty[half]), (phases >> half & 1) ^ 1)) return false;
        phases ^= 1u << half;
        fence_after();
        const int rows = half ? next.rows[1] : next.rows[0], ri = half * kHalf;
        const uint16_t* const q = (const uint16_t*)p.q.ptr + next.q_at;
        {
          // 16-byte pieces of a row in neighbouring lanes
          constexpr int P = D / 8;
          const uint32_t dst = q0 + half * kHalf * D * 2;
          const int c = row % P;
#pragma unroll 4
          for (int r = row / P; r < kHalf; r += 128 / P) {
            const int s = p.by_group.div(ri + r);
            const bool on = r < rows;
            const uint16_t* const src = on ? q + s * p.q.ss + (ri + r - s * p.G) * p.q.sn + c * 8 : (const uint16_t*)p.q.ptr;
            cp_async16(dst + swz(kHalf, r, c), src, on ? 16 : 0);
          }
          cp_async_wait_all();
          // Every lane its own pieces in place: times the power of two, 4-bit ones in their order.  (Through registers on the way a
          // prompt of 8192 tokens over 4-bit pages took 1105 us, not 805.)  On e4m3 pages the keys take the power, with their scales:
          // a ragged batch of short items 297 instead of 302 us.
          if constexpr (FMT != THINK_PAGE_E4M3) {
#pragma unroll 4
            for (int r = row / P; r < kHalf; r += 128 / P) {
              const uint32_t at = dst + swz(kHalf, r, c);
              uint4 v = ld_shared(at);
              if (T::kInt4) v = int4_order(v);
#pragma unroll
              for (int k = 0; k < 4; ++k) asm("mul.rn.bf16x2 %0, %0, %1;" : "+r"((&v.x)[k]) : "r"(p.q_scale2));
              st_shared(at, v);
            }
          }
          fence_proxy_async();
        }
        __syncwarp();
        if (lane == 0) bar_arrive(smem_u32(&sh.q_full[half]));
      }
    }
    if (!it.last) {
      float* const rec = (float*)p.records + (2 * blockIdx.x + it.first) * prompt_record_floats(kItemRows, D);
#pragma unroll 1
      for (int half = 0; half < 2; ++half) {
        const int end = half ? it.end[1] : it.end[0];
        const bool some = end > 0, on = row < (half ? it.rows[1] : it.rows[0]);
        float m = -INFINITY, l = 0.f;
        if (some) {
          if (!warp_wait_long(sh.failed, smem_u32(&sh.stats_full[half]), phases >> (2 + half) & 1)) return false;
          m = sh.stats[half][0][row];
          l = sh.stats[half][1][row];
          if (!warp_wait_long(sh.failed, smem_u32(&sh.o_done[half]), phases >> (4 + half) & 1)) return false;
          phases ^= 20u << half;
          fence_after();
        }
        const bool mend = *(volatile uint8_t*)&sh.bad[(items.no - 1) & (4 * kItems - 1)] != 0;      // (behind the waits)
        const int ri = half * kHalf + row, s = p.by_group.div(ri), g = ri - s * p.G;
        const bool none = m == -INFINITY && l == 0.f;
        const float f = none ? 0.f : m == -INFINITY ? __int_as_float(0x7fffffff) : 1.f / l;
        uint16_t* const dst = (uint16_t*)p.out.ptr + it.out_at + s * p.out.ss + g * p.out.sn;
#pragma unroll 1
        for (int c = 0; c < D; c += 32) {
          uint32_t o[32];
          if (some) {
            tmem_ld32(lanes + T::kColO + half * D + c, o);
            tmem_wait_ld();
            if (c + 32 == D) {          // the half's next product may overwrite it
              fence_before();
              __syncwarp();
              if (lane == 0) bar_arrive(smem_u32(&sh.o_empty[half]));
            }
          }
          if (!some || none) {
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = 0u;
          }
          if constexpr (T::kInt4) {     // back in the order of channels
            uint32_t u[32];
#pragma unroll
            for (int j = 0; j < 32; ++j) u[int4_channel(j)] = o[j];
#pragma unroll
            for (int j = 0; j < 32; ++j) o[j] = u[j];
          }
          if (on && it.whole) {
#pragma unroll
            for (int j = 0; j < 32; j += 8) {
              uint32_t u[4];
#pragma unroll
              for (int k = 0; k < 4; ++k) u[k] = none ? 0u : pack_bf16(__uint_as_float(o[j + 2 * k]) * f, __uint_as_float(o[j + 2 * k + 1]) * f);
              *(uint4*)(dst + c + j) = make_uint4(u[0], u[1], u[2], u[3]);
            }
          } else if (on) {
#pragma unroll
            for (int j = 0; j < 32; j += 4) *(uint4*)(rec + (size_t)ri * D + c + j) = make_uint4(o[j], o[j + 1], o[j + 2], o[j + 3]);
          }
          __syncwarp();
        }
        if (mend && on) {               // values that were left out because some rows do not see them
          const int stop = min(min(it.n, it.pos0 + s + 1), (it.t0 + end) * KT);
#pragma unroll 1
          for (int tok = max(max(it.pos0 + 1, it.t0 * KT), 0); tok < stop; ++tok) {
            const int page = page_of(p.table, p.g, it.b, tok, p.error);
            if (page < 0) continue;
            const uint8_t* const block = p.pages + page_block_offset(p.g, it.layer, page, it.h);
#pragma unroll 1
            for (int c = 0; c < D; ++c) {
              const float v = non_finite_value<D, FMT>(block, tok & 63, c);
              if (v == 0.f) continue;
              if (it.whole) dst[c] = (uint16_t)(pack_bf16(__uint_as_float((uint32_t)dst[c] << 16) + v, 0.f) & 0xffffu);
              else rec[(size_t)ri * D + c] += v;
            }
          }
        }
        __syncwarp();
        if (on) {
          if (!it.whole) {
            rec[kItemRows * D + ri] = m;
            rec[kItemRows * (D + 1) + ri] = l;
          } else if (p.lse) {
            p.lse[it.lse_at + (int64_t)s * p.nlayers * p.N_q + g] = prompt_log_sum(m, l);
          }
        }
      }
    }
    if (next.last) return true;
    it = next;
  }
}

template <int D, int FMT>
__global__ void __launch_bounds__(Shape<D, FMT>::kThreads, 1) k_paged_prompt_tc(const __grid_constant__ PagedPromptParams p, const __grid_constant__ CUtensorMap map) {
  using T = Shape<D, FMT>;
  extern __shared__ __align__(1024) unsigned char smem[];       // nothing else is in shared memory: it starts on such a border
  typename T::Sh& sh = *(typename T::Sh*)(smem + T::kSharedAt);
  begin_dependent();
  const int tid = threadIdx.x, warp = tid >> 5;
  const uint32_t q0 = smem_u32(smem), ring0 = q0 + T::kQBytes, stage0 = q0 + T::kStageAt;
  if (q0 & 1023) {
    if (tid == 0) {
      atomicOr(p.error, kErrSmemAlign);
      p.desc[blockIdx.x] = PromptDesc{0, 0, 0, 0, 0};
    }
    return;
  }
  if (warp == T::kMmaWarp) {
    asm volatile("tcgen05.alloc.cta_group::1.sync.aligned.shared::cta.b32 [%0], %1;" :: "r"(smem_u32(&sh.tmem)), "r"(512) : "memory");
    asm volatile("tcgen05.relinquish_alloc_permit.cta_group::1.sync.aligned;" ::: "memory");
  }
  if (T::kPlain && tid == 32) asm volatile("prefetch.tensormap [%0];" :: "l"(&map) : "memory");
  if (tid == 0) {
    for (int i = 0; i < T::kSlots; ++i) {
      bar_init(smem_u32(&sh.full[i]), T::kPlain ? 1 : T::kUnpackWarps);
      bar_init(smem_u32(&sh.empty[i]), 2);
    }
    for (int i = 0; i < 2; ++i) {
      for (int k = 0; k < 2; ++k) {
        bar_init(smem_u32(&sh.s_full[i][k]), 1);
        bar_init(smem_u32(&sh.p_full[i][k]), 4);
      }
      bar_init(smem_u32(&sh.o_full[i]), 1);
      bar_init(smem_u32(&sh.o_done[i]), 1);
      bar_init(smem_u32(&sh.o_empty[i]), 4);
      bar_init(smem_u32(&sh.q_full[i]), 4);
      bar_init(smem_u32(&sh.q_empty[i]), 1);
      bar_init(smem_u32(&sh.stats_full[i]), 4);
      bar_init(smem_u32(&sh.left[i]), 1);
    }
    for (int i = 0; i < kItems; ++i) {
      bar_init(smem_u32(&sh.item_full[i]), 1);
      bar_init(smem_u32(&sh.item_empty[i]), 8 + 2 + 2 + 4 + T::kUnpackWarps);       // softmax, products, loads, rows, unpacking
    }
    bar_init(smem_u32(&sh.raw), 1);
    for (int i = 0; i < T::kStages; ++i) {
      bar_init(smem_u32(&sh.st_full[i]), 1);
      bar_init(smem_u32(&sh.st_empty[i]), T::kPlain ? 1 : T::kUnpackWarps);
    }
    asm volatile("fence.mbarrier_init.release.cluster;" ::: "memory");
    sh.failed = 0;
    for (int i = 0; i < 4 * kItems; ++i) sh.bad[i] = 0;
  }
  fence_before();
  __syncthreads();
  fence_after();
  const uint32_t tmem = sh.tmem;
  bool ok = true;
  if (warp < 8) {
    asm volatile("setmaxnreg.inc.sync.aligned.u32 %0;" :: "n"(T::kSoftmaxRegs));
    ok = softmax_role<D, FMT>(p, sh, tmem);
  } else if (warp >= T::kRowsWarp) {
    asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(T::kRowsRegs));
    ok = rows_role<D, FMT>(p, sh, q0, tmem);
  } else {
    if (warp < 8 + T::kUnpackWarps) asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(T::kLoadRegs));
    else asm volatile("setmaxnreg.dec.sync.aligned.u32 %0;" :: "n"(T::kMmaRegs));
    if (warp < (T::kPlain ? 10 : T::kMmaWarp)) {
      if constexpr (T::kPlain) ok = load_role<D, FMT>(p, &map, sh, ring0, warp - 8);
      else ok = unpack_role<D, FMT>(sh, ring0, stage0, __uint_as_float(p.q_scale2 << 16));
    } else if (!T::kPlain && warp >= T::kFetchWarp && warp < T::kFetchWarp + 2) {
      ok = fetch_role<D, FMT>(p, sh, stage0, warp - T::kFetchWarp);
    } else {
      ok = mma_role<D, FMT>(sh, q0, ring0, tmem, warp - T::kMmaWarp);
    }
  }
  if (!ok) {
    atomicOr(p.error, kErrWaitTimeout);
    sh.failed = 1;
  }
  fence_before();
  __syncthreads();
  if (sh.failed) {                       // copies and products under way end before their memory is given up
    if (tid == 0) p.desc[blockIdx.x] = PromptDesc{0, 0, 0, 0, 0};      // (the walk may not have come to its end: nothing to join)
    const long long t0 = clock64();
    while (clock64() - t0 < 4000000LL) {}
  }
  if (warp == T::kMmaWarp) asm volatile("tcgen05.dealloc.cta_group::1.sync.aligned.b32 %0, %1;" :: "r"(tmem), "r"(512) : "memory");
}

template <int D, int FMT>
cudaError_t setup() {
  cudaError_t e = cudaFuncSetAttribute(k_paged_prompt_tc<D, FMT>, cudaFuncAttributeMaxDynamicSharedMemorySize, Shape<D, FMT>::kSmem);
  cudaFuncAttributes a;
  if (e == cudaSuccess) e = cudaFuncGetAttributes(&a, k_paged_prompt_tc<D, FMT>);
  // the roles' shares of the registers add up to these: fewer would be a wait without an end
  if (e == cudaSuccess && a.numRegs < Shape<D, FMT>::kRegs) e = cudaErrorLaunchOutOfResources;
  return e;
}
template <int D, int FMT>
cudaError_t launch(const PagedPromptParams& p, const CUtensorMap& map, cudaStream_t s) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(p.grid);
  cfg.blockDim = dim3(Shape<D, FMT>::kThreads);
  cfg.dynamicSmemBytes = Shape<D, FMT>::kSmem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, k_paged_prompt_tc<D, FMT>, p, map);
  if (e != cudaSuccess) (void)cudaGetLastError();
  return e;
}

}  // namespace

PromptCut paged_prompt_tc_cut() { return PromptCut{kExtra}; }
int paged_prompt_tc_rows() { return kItemRows; }

cudaError_t paged_prompt_tc_setup(int format, int D) {
  switch (format * 256 + D) {
    case THINK_PAGE_PLAIN * 256 + 64: return setup<64, THINK_PAGE_PLAIN>();
    case THINK_PAGE_PLAIN * 256 + 128: return setup<128, THINK_PAGE_PLAIN>();
    case THINK_PAGE_E4M3 * 256 + 64: return setup<64, THINK_PAGE_E4M3>();
    case THINK_PAGE_E4M3 * 256 + 128: return setup<128, THINK_PAGE_E4M3>();
    case THINK_PAGE_INT4 * 256 + 64: return setup<64, THINK_PAGE_INT4>();
    case THINK_PAGE_INT4 * 256 + 128: return setup<128, THINK_PAGE_INT4>();
  }
  return cudaErrorInvalidValue;
}
cudaError_t launch_paged_prompt_tc(const PagedPromptParams& p, int format, const void* map, cudaStream_t s) {
  CUtensorMap m;
  memcpy(&m, map, sizeof(m));
  switch (format * 256 + p.g.D) {
    case THINK_PAGE_PLAIN * 256 + 64: return launch<64, THINK_PAGE_PLAIN>(p, m, s);
    case THINK_PAGE_PLAIN * 256 + 128: return launch<128, THINK_PAGE_PLAIN>(p, m, s);
    case THINK_PAGE_E4M3 * 256 + 64: return launch<64, THINK_PAGE_E4M3>(p, m, s);
    case THINK_PAGE_E4M3 * 256 + 128: return launch<128, THINK_PAGE_E4M3>(p, m, s);
    case THINK_PAGE_INT4 * 256 + 64: return launch<64, THINK_PAGE_INT4>(p, m, s);
    case THINK_PAGE_INT4 * 256 + 128: return launch<128, THINK_PAGE_INT4>(p, m, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace think
