// Attention of one new token per sequence over the paged cache: out = softmax(scale q K^T) V, and its log sum.
//
// Every byte of the pages is read once and used for at most 8 query heads, so the stream of pages is the floor.  Pages of
// bf16 and fp32 come near it (0.94 to 0.98 of the copy rate).  Quantised pages are held by latency: a scheduler has two
// (e4m3) or three (4 bits) warps, each one chain of dependent steps (ldmatrix, unpack, mma, vote, ex2, transpose, mma), and
// issues in 46 and 56 % of its cycles, with no unit above 44 % busy.  The kernel is built around the stream:
//  * The tiles (64-token pages) of all (entry, layer, key head) units stand on one line, with some room for starting and
//    ending a unit; it is cut evenly over the CTAs of one wave and inside a CTA over its warps, whatever the lengths:
//    one long sequence uses the whole card and a ragged batch leaves no SM idle.  Lengths and page table are device
//    memory; each CTA scans the lengths itself.  (Cut by tiles alone, 192 sequences of 1 to 2000 tokens took 95 us
//    instead of 71 when that was tried: the CTAs with the short ones came last.)
//  * A warp is the worker.  It owns a ring of stages in shared memory that it fills with cp.async, crossing page and
//    unit borders, and waits for nobody until its range is done.
//  * Rows are stored token-major.  16-byte chunks are XOR-swizzled on the way into shared memory so that ldmatrix
//    reads without bank conflicts.  Products run on mma.sync m16n8k16 with keys and values as A (16 tokens or channels)
//    and the group's queries or weights as B: a group has at most 8 query rows, which is N here, and 8 of the 128 rows
//    that a tcgen05 tile would have.
//      logits  bf16 and 4-bit pages: bf16 products, exact (a masked 4-bit code is the subnormal c * 2^-133 or c * 2^-129,
//              one multiply-add makes it (c - 8) / 64).  e4m3 codes become f16 by byte conversion; the query is f16
//              times a power of two, exact unless its channels are more than 2^28 apart.  (The fp8 form of the
//              instruction takes codes as they are, but here it is a sequence of conversions and two f16
//              instructions: 22 cycles against 8.3, measured.)
//      values  through ldmatrix.trans, as bf16 (4-bit codes as above, e4m3 through f16 and fp32); the weights, which
//              come out token by token, are transposed in registers.  A weight, times its value's scale, is a bf16 pair
//              high + low (two instructions), 2^-16: it has the range of fp32, so that no channel's or token's share
//              is lost to larger ones.  (f16 weights relative to the largest weight * scale so far took one instruction
//              - e4m3, 4 x 32768 tokens: 51 us against 53; 4-bit ragged: 68 against 73 - but left 21 binary orders
//              below that largest one, over all channels and tokens.)
//      scales  of keys multiply logits, those of values the weights.
//      fp32    CUDA cores: fp32 products summed over lanes pairwise.
//  * The softmax is online in base 2 with fp32 maximum, sum and accumulators.  Units that several warps share leave
//    partial states; the warps' states are joined by their CTA, the CTAs' states by the CTA that arrives last at
//    the unit's ticket, always in token order, so results do not depend on timing.
//
// Measured (one call among others, buffers that change from call to call; the share is of the copy rate, 6.54 TB/s):
//   bf16  32 heads of 128, 16 sequences of 2048 to 4096      139 us   0.94
//   bf16  32 / 8 heads, 131072 tokens, two layers            168 us   0.98
//   fp32  32 / 8 heads, 4 x 32768 tokens (replayed)          171 us   0.96
//   e4m3  32 / 8 heads, 4 x 32768 tokens                      55 us   0.76
//   int4  32 / 8 heads, 192 sequences of 1 to 2000            73 us   0.52
//   int4  32 / 8 heads, 8192 tokens                           13 us   launch, three dependent loads and two joins
#include <cuda_fp16.h>
#include <cuda_fp8.h>
#include <float.h>
#include <math.h>

#include "paged_internal.h"
#include "paged_split.h"

namespace think {
namespace {

constexpr int kMaxWarps = 12;
// reference of a unit whose tokens had no logit above -infinity so far; without any token it is -infinity
constexpr float kLowest = -FLT_MAX;
constexpr float kAhead = 8.f;                 // how far above the largest logit weights' reference is put when it moves
// While all value scales of a unit are below 2^-80 the reference is put 48 below the largest logit, and moves when that
// is 8 more: weights from 2^48 on keep products with scales down to 2^-133 away from the ends of bf16 and fp32.
constexpr float kSmallBehind = 48.f, kSmallLead = 56.f;
constexpr uint32_t kSmallScale = 127 - 80;    // exponent field
constexpr int kMaxG = kMaxPagedGroup;

// GP: query heads that the fp32 kernel computes at a time
template <int D, int E, int FMT, int GP = 1>
struct Shape {
  static constexpr bool F32 = E == 4;
  // Eight warps keep 130 KB of copies in flight with up to 255 registers each (e4m3 takes 245).  4-bit pages have twelve:
  // against eight, 192 ragged sequences take the same 72.7 us, one of 8192 tokens 13.1 instead of 13.9, heads of 64
  // 43.5 instead of 46.8, and 4 x 32768 tokens 46.4 instead of 45.3 (heads of 128 spill 72 bytes at 168 registers).
  static constexpr int WARPS = FMT == THINK_PAGE_INT4 ? 12 : 8;
  static constexpr int THREADS = WARPS * 32;
  static constexpr int RB = FMT == THINK_PAGE_PLAIN ? D * E : FMT == THINK_PAGE_E4M3 ? D : D / 2;   // bytes of a row
  static constexpr int SB = FMT == THINK_PAGE_PLAIN ? 0 : FMT == THINK_PAGE_E4M3 ? 1 : D / 16;      // bytes of its scales
  // tokens of a step: at most 8 KB of keys and values, at most 32; fp32: at most 64 products with queries a lane
  static constexpr int ST = F32 && GP * (4096 / RB) > 64 ? 64 / GP : 4096 / RB < 32 ? 4096 / RB : 32;
  // starting and ending a unit takes about as long as a tile of quantised pages or a quarter of a tile of others
  // (measured: 1.4 to 1.7 us beside 1.8 to 2.4, 0.8 beside 3.5; half as much weight: 95 us instead of 84 for 192 ragged
  // sequences of e4m3).  Two places a tile cut a little more evenly than one (4 x 32768 tokens 50.8 against 52.9 us).
  static __device__ __forceinline__ Weights weights() { return FMT == THINK_PAGE_PLAIN ? Weights{4, 1} : Weights{2, 2}; }
  static constexpr int HALF = ST * RB;                       // key (or value) bytes of a stage
  static constexpr int STAGE = (2 * (HALF + ST * SB) + 127) / 128 * 128;
  static constexpr int SPACE = 200 * 1024 / WARPS;           // shared memory of a warp
  static constexpr int STAGES = SPACE / STAGE < 8 ? SPACE / STAGE : 8;
  static constexpr int RING = STAGES * STAGE;
  static_assert(STAGES >= 2 && WARPS <= kMaxWarps && WARPS >= kMaxG && WARPS % 4 == 0, "ring");
  // a warp's ring takes its partial state and the weights of a join afterwards, or a join's statistics
  static_assert(RING >= (2 * kMaxG + kMaxG * (D + 4) + kMaxWarps * kMaxG) * 4 && RING >= kSMs * 2 * 8 + 512, "ring");
};

// Partial state of one (worker, unit).  m: the logit (base 2) that weights are relative to, near the largest one; l: sum
// of the weights exp2(logit - m).
// Rows are 4 floats longer than D: the lanes of a fragment, two rows apart, then store to different banks.
template <int D>
struct Record {
  float2 s[kMaxG];           // m, l
  float o[kMaxG][D + 4];
};

__device__ __forceinline__ uint32_t smem_u32(const void* p) { return (uint32_t)__cvta_generic_to_shared(p); }
// copies src_bytes (0..16) and zero-fills the rest of the 16 bytes
__device__ __forceinline__ void cp16(uint32_t dst, const void* src, int src_bytes) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16, %2;" ::"r"(dst), "l"(src), "r"(src_bytes) : "memory");
}
__device__ __forceinline__ void cp16(uint32_t dst, const void* src) {
  asm volatile("cp.async.cg.shared.global [%0], [%1], 16;" ::"r"(dst), "l"(src) : "memory");
}
__device__ __forceinline__ void cp_commit() { asm volatile("cp.async.commit_group;" ::: "memory"); }
template <int N>
__device__ __forceinline__ void cp_wait() { asm volatile("cp.async.wait_group %0;" ::"n"(N) : "memory"); }

__device__ __forceinline__ void ldsm4(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
__device__ __forceinline__ void ldsm4t(uint32_t addr, uint32_t (&r)[4]) {
  asm volatile("ldmatrix.sync.aligned.m8n8.x4.trans.shared.b16 {%0,%1,%2,%3}, [%4];"
               : "=r"(r[0]), "=r"(r[1]), "=r"(r[2]), "=r"(r[3]) : "r"(addr) : "memory");
}
template <bool BF16>
__device__ __forceinline__ void mma(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%0,%1,%2,%3};"
        : "+f"(d[0]), "+f"(d[1]), "+f"(d[2]), "+f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1));
}
// the same without an accumulator yet
template <bool BF16>
__device__ __forceinline__ void mma_first(float (&d)[4], uint32_t a0, uint32_t a1, uint32_t a2, uint32_t a3, uint32_t b0, uint32_t b1) {
  if (BF16)
    asm("mma.sync.aligned.m16n8k16.row.col.f32.bf16.bf16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
  else
    asm("mma.sync.aligned.m16n8k16.row.col.f32.f16.f16.f32 {%0,%1,%2,%3}, {%4,%5,%6,%7}, {%8,%9}, {%10,%10,%10,%10};"
        : "=f"(d[0]), "=f"(d[1]), "=f"(d[2]), "=f"(d[3]) : "r"(a0), "r"(a1), "r"(a2), "r"(a3), "r"(b0), "r"(b1), "f"(0.f));
}
// 8 x 8 matrix of 16-bit elements, rows over lanes / 4: its transpose
__device__ __forceinline__ uint32_t transpose8(uint32_t x) {
  uint32_t y;
  asm("movmatrix.sync.aligned.m8n8.trans.b16 %0, %1;" : "=r"(y) : "r"(x));
  return y;
}
__device__ __forceinline__ float ex2(float x) {
  float y;
  asm("ex2.approx.ftz.f32 %0, %1;" : "=f"(y) : "f"(x));
  return y;
}
// larger of two pairs of bf16
__device__ __forceinline__ uint32_t max_bf16x2(uint32_t a, uint32_t b) {
  uint32_t r;
  asm("max.bf16x2 %0, %1, %2;" : "=r"(r) : "r"(a), "r"(b));
  return r;
}
__device__ __forceinline__ uint32_t pack_bf16(float lo, float hi) {
  __nv_bfloat162 v = __floats2bfloat162_rn(lo, hi);
  return *(uint32_t*)&v;
}
__device__ __forceinline__ uint32_t pack_f16(float lo, float hi) {
  __half2 v = __floats2half2_rn(lo, hi);
  return *(uint32_t*)&v;
}
// Two weights w >= 0 as sums of two bf16: the first 8 bits, cut off, and the rest, rounded: within 2^-16.  Both parts
// multiply a value, so neither may be zero or negative beside a weight: an infinite value would become a NaN.  Cutting
// keeps the rest from being negative, w * 2^-23 on top of it (fused, one rounding) from being zero.
__device__ __forceinline__ void pair_bf16(float w0, float w1, uint32_t& hi, uint32_t& lo) {
  const uint32_t u0 = __float_as_uint(w0), u1 = __float_as_uint(w1);
  hi = __byte_perm(u0, u1, 0x7632);
  float a, b;
  split(fma2(two(w0, w1), two(1.f + 0x1p-23f, 1.f + 0x1p-23f),
             two(__uint_as_float((u0 & 0xffff0000u) ^ 0x80000000u), __uint_as_float((u1 & 0xffff0000u) ^ 0x80000000u))), a, b);
  lo = pack_bf16(a, b);
}
// Two such pairs (here the first part is rounded to the nearest) times two bf16 scales, as pairs again: the product's
// first 8 bits, and what they leave of it (exact, it has 8 more) plus the second part's product.  Within 2^-17.
__device__ __forceinline__ void scale_pair(uint32_t wh, uint32_t wl, uint32_t f, uint32_t& hi, uint32_t& lo) {
  const __nv_bfloat162 a = *(const __nv_bfloat162*)&wh, b = *(const __nv_bfloat162*)&wl, s = *(const __nv_bfloat162*)&f;
  const __nv_bfloat162 h = __hmul2_rn(a, s);
  const __nv_bfloat162 r = __hfma2(b, s, __hfma2(a, s, __hneg2(h)));
  hi = *(const uint32_t*)&h;
  lo = *(const uint32_t*)&r;
}
// two e4m3 bytes as f16: the lower and the upper half of a word
__device__ __forceinline__ uint32_t e4m3_lo_to_f16x2(uint32_t w) {
  uint32_t d;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, lo;\n\t}" : "=r"(d) : "r"(w));
  return d;
}
__device__ __forceinline__ uint32_t e4m3_hi_to_f16x2(uint32_t w) {
  uint32_t d;
  asm("{\n\t.reg .b16 lo, hi;\n\tmov.b32 {lo, hi}, %1;\n\tcvt.rn.f16x2.e4m3x2 %0, hi;\n\t}" : "=r"(d) : "r"(w));
  return d;
}
__device__ __forceinline__ uint32_t f16x2_to_bf16x2(uint32_t w) {
  const float2 f = __half22float2(*(const __half2*)&w);
  return pack_bf16(f.x, f.y);
}
// the codes at bits 0..3 and 16..19 of w as bf16 numbers n / 64: the masked word holds subnormals c * 2^-133
__device__ __forceinline__ uint32_t int4_lo_to_bf16x2(uint32_t w) {
  const uint32_t t = w & 0x000f000fu, k = 0x7f007f00u, o = 0xbe00be00u;       // 2^127, -8 / 64
  const __nv_bfloat162 r = __hfma2(*(const __nv_bfloat162*)&t, *(const __nv_bfloat162*)&k, *(const __nv_bfloat162*)&o);
  return *(const uint32_t*)&r;
}
// the same at bits 4..7 and 20..23: c * 2^-129 (from c = 8 on the exponent field is 1, which goes on in the same steps)
__device__ __forceinline__ uint32_t int4_hi_to_bf16x2(uint32_t w) {
  const uint32_t t = w & 0x00f000f0u, k = 0x7d007d00u, o = 0xbe00be00u;       // 2^123
  const __nv_bfloat162 r = __hfma2(*(const __nv_bfloat162*)&t, *(const __nv_bfloat162*)&k, *(const __nv_bfloat162*)&o);
  return *(const uint32_t*)&r;
}
constexpr float kInt4Unit = 64.f;
// 2^k for -126 <= k <= 127
__device__ __forceinline__ float pow2i(int k) { return __uint_as_float((uint32_t)(k + 127) << 23); }

// where chunk ck (16 bytes) of row r lands: a permutation within the row under which 8 rows' equal chunks fall into
// different banks
template <int RB>
__device__ __forceinline__ int swz(int r, int ck) {
  if (RB >= 128) return r * RB + ((ck ^ (r & 7)) << 4);
  if (RB == 64) return r * RB + ((ck ^ ((r >> 1) & 3)) << 4);
  return r * RB + ((ck ^ ((r >> 2) & 1)) << 4);
}

// Tables of a launch in shared memory: cumulative places (per layer and head) and the tokens of each sequence's last
// tile.
struct Tables {
  const int* cum;            // [B + 1]
  const uint8_t* last;       // tokens in the last tile, minus 1
  Weights w;
  int B, nlayers, N_kv;
};
struct Cursor {              // a tile of the line
  int b, ll, h;              // entry, layer of the call, key head
  int j, nt;                 // tile and tiles of the unit
  int len;
  int64_t us;                // place of the unit's first tile
};
__device__ __forceinline__ void seq_of(const Tables& t, Cursor& c) {
  c.nt = t.w.tiles(t.cum[c.b + 1] - t.cum[c.b]);
  c.len = (c.nt - 1) * kPageTokens + t.last[c.b] + 1;
}
// to the first tile of the next unit, if there is one
__device__ __forceinline__ void next_unit(const Tables& t, Cursor& c) {
  c.us += t.w.cost(c.nt);
  c.j = 0;
  if (++c.h < t.N_kv) return;
  c.h = 0;
  if (++c.ll < t.nlayers) return;
  c.ll = 0;
  do ++c.b; while (c.b < t.B && t.cum[c.b + 1] == t.cum[c.b]);
  if (c.b < t.B) seq_of(t, c);
}
// the first tile at place f or behind, f below the line's end; none if the result's place is the line's end
__device__ __forceinline__ Cursor locate(const Tables& t, int64_t f) {
  const int LH = t.nlayers * t.N_kv;
  int lo = 0, hi = t.B - 1;                    // last entry that begins at f or before: it has tiles
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if ((int64_t)t.cum[mid] * LH <= f) lo = mid; else hi = mid - 1;
  }
  Cursor c;
  c.b = lo;
  seq_of(t, c);
  const int cost = t.w.cost(c.nt);
  const int64_t rem = f - (int64_t)t.cum[lo] * LH;
  const int u = (int)div_wide(rem, cost);
  c.us = f - rem + (int64_t)u * cost;
  c.ll = (int)((unsigned)u / (unsigned)t.N_kv);
  c.h = u - c.ll * t.N_kv;
  c.j = t.w.first_tile(f - c.us);
  if (c.j >= c.nt) next_unit(t, c);
  return c;
}

// brings `bytes` (a multiple of 128, at most 4096) towards the SM; the values are not waited for
__device__ __forceinline__ void touch(const uint8_t* p, int bytes, int lane) {
  uint32_t x;
  if (lane * 128 < bytes) asm volatile("ld.global.ca.u32 %0, [%1];" : "=r"(x) : "l"(p + lane * 128));
}

__device__ __forceinline__ uint32_t ticket_add(uint32_t* p) {
  uint32_t x;
  asm volatile("atom.add.acq_rel.gpu.global.u32 %0, [%1], 1;" : "=r"(x) : "l"(p) : "memory");
  return x;
}

// What a warp tells its CTA: its first and its last unit, with the places of their first and last tiles.
struct WarpInfo {
  int64_t first_us, first_ul, last_us, last_ul;
  int first_unit, last_unit; // index of the unit in the call
  int busy;                  // has tiles
};

// ---------------------------------------------------------------------------------------------------------
// Tensor-core formats: fragments of a warp.  Lane (r = lane / 4, qd = lane % 4).  Logits and accumulators have the
// lane's queries 2 qd, 2 qd + 1 in register pairs: logits of tokens 8 n + r of the step, accumulators of channels by r.
template <int FMT>
__device__ __forceinline__ float finish(float m, float l);

template <int D, int FMT>
struct MmaState {
  using S = Shape<D, 2, FMT>;
  static constexpr bool PLAIN = FMT == THINK_PAGE_PLAIN;
  static constexpr bool INT4 = FMT == THINK_PAGE_INT4;
  static constexpr int NT = S::ST / 8;          // groups of 8 tokens of a step
  static constexpr int NG = D / 32;             // blocks of 32 channels, the scale groups of 4-bit rows
  static constexpr int OT = D / 16;
  static constexpr int WIDTH = PLAIN ? 1 : INT4 ? 4 : 2;     // consecutive channels that a lane holds

  uint32_t q[NG][4];         // B fragments of the two k16 instructions of a block: query r
  f32x2 rs;                  // base-2 logit per unit of the q k product
  float m[2];                // what weights are relative to
  float lead;                // how far a logit may exceed that: 0, or kSmallLead (value scales all small so far)
  f32x2 l;                   // of this lane's tokens until end()
  float o[OT][4];

  // the unit's queries in the order of the fragments, as they lie in memory; qg: its first query row
  struct Raw { uint32_t w[NG][4]; };
  static __device__ __forceinline__ void fetch(const void* qg, int G, int lane, Raw& raw) {
    const __nv_bfloat16* qr = (const __nv_bfloat16*)qg + (lane >> 2) * D;
    const int qd = lane & 3;
    const bool on = (lane >> 2) < G;
#pragma unroll
    for (int g = 0; g < NG; ++g) {
      uint32_t (&w)[4] = raw.w[g];
      if constexpr (PLAIN) {
#pragma unroll
        for (int i = 0; i < 4; ++i) w[i] = on ? *(const uint32_t*)(qr + 32 * g + 8 * i + 2 * qd) : 0u;
      } else if constexpr (INT4) {              // channels 32 g + 8 qd .. + 7
        const uint4 x = on ? *(const uint4*)(qr + 32 * g + 8 * qd) : make_uint4(0u, 0u, 0u, 0u);
        w[0] = x.x; w[1] = x.y; w[2] = x.z; w[3] = x.w;
      } else {                                  // 32 g + 4 qd .. + 3 and 16 behind
        const uint2 x = on ? *(const uint2*)(qr + 32 * g + 4 * qd) : make_uint2(0u, 0u);
        const uint2 y = on ? *(const uint2*)(qr + 32 * g + 16 + 4 * qd) : make_uint2(0u, 0u);
        w[0] = x.x; w[1] = x.y; w[2] = y.x; w[3] = y.y;
      }
    }
  }
  // starts a unit: its queries as B fragments, no tokens yet
  __device__ __forceinline__ void begin(const Raw& raw, float scale_log2, int lane) {
    const uint32_t (&w)[NG][4] = raw.w;
    if constexpr (PLAIN) {
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[g][i] = w[g][i];
      rs = two(scale_log2, scale_log2);
    } else if constexpr (INT4) {                // the codes of a word pair up as channels (0,4) (1,5) | (2,6) (3,7)
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          q[g][2 * j] = __byte_perm(w[g][j], w[g][2 + j], 0x5410);
          q[g][2 * j + 1] = __byte_perm(w[g][j], w[g][2 + j], 0x7632);
        }
      rs = two(scale_log2 * kInt4Unit, scale_log2 * kInt4Unit);
    } else {
      const int qd = lane & 3;
      uint32_t t = 0;                           // largest magnitude's bits (as numbers: NaN counts as none)
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) t = max_bf16x2(t, w[g][i] & 0x7fff7fffu);
      t = max(t & 0xffffu, t >> 16);
      t = max(t, __shfl_xor_sync(0xffffffffu, t, 1));
      t = max(t, __shfl_xor_sync(0xffffffffu, t, 2));
      // the row's largest channel goes to [2^14, 2^15), as far as the power and the factor that takes it back are
      // ordinary numbers
      const int k = min(141 - (int)(t >> 7), min(126, (int)(__float_as_uint(scale_log2) >> 23) - 1));
      const float up = pow2i(k), down = scale_log2 * pow2i(-k);
      rs = two(__shfl_sync(0xffffffffu, down, 8 * qd), __shfl_sync(0xffffffffu, down, 8 * qd + 4));
#pragma unroll
      for (int g = 0; g < NG; ++g)
#pragma unroll
        for (int i = 0; i < 4; ++i) q[g][i] = pack_f16(bf16lo(w[g][i]) * up, bf16hi(w[g][i]) * up);
    }
    m[0] = m[1] = -INFINITY;
    lead = PLAIN ? 0.f : kSmallLead;
    l = 0;
#pragma unroll
    for (int t = 0; t < OT; ++t) o[t][0] = o[t][1] = o[t][2] = o[t][3] = 0.f;
  }

  // bf16 scales of a token: NG / 2 words
  static __device__ __forceinline__ void load_scales(uint32_t a, uint32_t (&sc)[NG / 2]) {
    if constexpr (NG == 4)
      asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(sc[0]), "=r"(sc[1]) : "r"(a));
    else
      asm volatile("ld.shared.u32 %0, [%1];" : "=r"(sc[0]) : "r"(a));
  }
  // those of two neighbouring tokens, the first one even
  static __device__ __forceinline__ void load_scales2(uint32_t a, uint32_t (&sc)[NG]) {
    if constexpr (NG == 4)
      asm volatile("ld.shared.v4.u32 {%0,%1,%2,%3}, [%4];" : "=r"(sc[0]), "=r"(sc[1]), "=r"(sc[2]), "=r"(sc[3]) : "r"(a));
    else
      asm volatile("ld.shared.v2.u32 {%0,%1}, [%2];" : "=r"(sc[0]), "=r"(sc[1]) : "r"(a));
  }
  static __device__ __forceinline__ float scale_of(const uint32_t (&sc)[NG / 2], int g) {
    return (g & 1) ? bf16hi(sc[g >> 1]) : bf16lo(sc[g >> 1]);
  }
  static __device__ __forceinline__ uint32_t load_byte(uint32_t a) {
    uint32_t x;
    asm volatile("ld.shared.u8 %0, [%1];" : "=r"(x) : "r"(a));
    return x;
  }

  // one step: keys at sb, values at sb + HALF, scales behind; ntok of its tokens count
  __device__ __forceinline__ void step(uint32_t sb, int ntok, int lane) {
    const int r = lane >> 2, mi = lane >> 3, tr = lane & 7;
    const uint32_t ks = sb + 2 * S::HALF + r * S::SB, vs = ks + S::ST * S::SB;     // scales of token r
    const uint32_t vs2 = sb + 2 * S::HALF + (S::ST + 2 * (lane & 3)) * S::SB;      // values' scales of token 2qd
    f32x2 x[NT];
    // ---- logits, 16 tokens at a time
#pragma unroll
    for (int n = 0; n < NT; n += 2) {
      if constexpr (PLAIN) {
        const int off = (tr + 8 * (mi >> 1)) * S::RB + (((mi & 1) ^ tr) << 4);
        float c[2][4];                          // two chains
#pragma unroll
        for (int s = 0; s < D / 16; ++s) {
          const uint32_t b0 = q[s >> 1][2 * (s & 1)], b1 = q[s >> 1][2 * (s & 1) + 1];
          uint32_t k[4];
          ldsm4(sb + n * 8 * S::RB + (off ^ (s << 5)), k);
          if (s < 2) mma_first<true>(c[s], k[0], k[2], k[1], k[3], b0, b1);
          else mma<true>(c[s & 1], k[0], k[2], k[1], k[3], b0, b1);
        }
        x[n] = mul2(add2(two(c[0][0], c[0][1]), two(c[1][0], c[1][1])), rs);
        x[n + 1] = mul2(add2(two(c[0][2], c[0][3]), two(c[1][2], c[1][3])), rs);
      } else if constexpr (!INT4) {
        const int off = S::RB == 128 ? tr * 128 + ((mi ^ tr) << 4) : tr * 64 + ((mi ^ (tr >> 1)) << 4);
        float c[2][4];
#pragma unroll
        for (int i = 0; i < NG / 2; ++i) {
          uint32_t k[4], k8[4];                 // tokens r and r + 8; a word: channels 4qd .. 4qd + 3 of 16
          ldsm4(sb + n * 8 * S::RB + (off ^ (i << 6)), k);
          ldsm4(sb + (n + 1) * 8 * S::RB + (off ^ (i << 6)), k8);
#pragma unroll
          for (int j = 0; j < 4; ++j) {
            const uint32_t b0 = q[2 * i + (j >> 1)][2 * (j & 1)], b1 = q[2 * i + (j >> 1)][2 * (j & 1) + 1];
            const uint32_t a0 = e4m3_lo_to_f16x2(k[j]), a1 = e4m3_lo_to_f16x2(k8[j]), a2 = e4m3_hi_to_f16x2(k[j]), a3 = e4m3_hi_to_f16x2(k8[j]);
            if (i == 0 && j < 2) mma_first<false>(c[j], a0, a1, a2, a3, b0, b1);
            else mma<false>(c[j & 1], a0, a1, a2, a3, b0, b1);
          }
        }
        const float s0 = e8m0(load_byte(ks + 8 * n)), s1 = e8m0(load_byte(ks + 8 * n + 8));
        x[n] = mul2(add2(two(c[0][0], c[0][1]), two(c[1][0], c[1][1])), mul2(rs, two(s0, s0)));
        x[n + 1] = mul2(add2(two(c[0][2], c[0][3]), two(c[1][2], c[1][3])), mul2(rs, two(s1, s1)));
      } else {
        uint32_t k[NG], k8[NG], s0[NG / 2], s1[NG / 2];      // tokens r and r + 8; a word: channels 8qd .. 8qd + 7 of 32
        if constexpr (NG == 4) {
          const int off = tr * 64 + ((mi ^ (tr >> 1)) << 4);
          ldsm4(sb + n * 8 * S::RB + off, k);
          ldsm4(sb + (n + 1) * 8 * S::RB + off, k8);
        } else {
          uint32_t t[4];
          ldsm4(sb + n * 8 * S::RB + (tr + 8 * (mi >> 1)) * 32 + (((mi & 1) ^ (tr >> 2)) << 4), t);
          k[0] = t[0]; k[1] = t[1]; k8[0] = t[2]; k8[1] = t[3];
        }
        load_scales(ks + 8 * n * S::SB, s0);
        load_scales(ks + (8 * n + 8) * S::SB, s1);
        f32x2 y0 = 0, y1 = 0;
#pragma unroll
        for (int g = 0; g < NG; ++g) {
          const uint32_t a = k[g], b = k8[g], ah = a >> 8, bh = b >> 8;
          float c[4];
          mma_first<true>(c, int4_lo_to_bf16x2(a), int4_lo_to_bf16x2(b), int4_hi_to_bf16x2(a), int4_hi_to_bf16x2(b), q[g][0], q[g][1]);
          mma<true>(c, int4_lo_to_bf16x2(ah), int4_lo_to_bf16x2(bh), int4_hi_to_bf16x2(ah), int4_hi_to_bf16x2(bh), q[g][2], q[g][3]);
          const float f0 = scale_of(s0, g), f1 = scale_of(s1, g);
          y0 = fma2(two(c[0], c[1]), two(f0, f0), y0);
          y1 = fma2(two(c[2], c[3]), two(f1, f1), y1);
        }
        x[n] = mul2(y0, rs);
        x[n + 1] = mul2(y1, rs);
      }
    }
    if (ntok < S::ST) {
#pragma unroll
      for (int n = 0; n < NT; ++n)
        if (8 * n + r >= ntok) x[n] = two(-INFINITY, -INFINITY);
    }
    float mx[2] = {ntok > 0 ? kLowest : -INFINITY, ntok > 0 ? kLowest : -INFINITY};
#pragma unroll
    for (int n = 0; n < NT; ++n) {
      float a, b;
      split(x[n], a, b);
      mx[0] = fmaxf(mx[0], a);
      mx[1] = fmaxf(mx[1], b);
    }
    if (!PLAIN && lead > 0.f) {
      bool big = false;
#pragma unroll
      for (int n = 0; n < NT; ++n) {
        if constexpr (INT4) {                   // bit 15 of a half: its exponent field is at least kSmallScale
          uint32_t sc[NG / 2];
          load_scales(vs + 8 * n * S::SB, sc);
#pragma unroll
          for (int i = 0; i < NG / 2; ++i)
            big |= (((sc[i] & 0x7fff7fffu) + 0x00010001u * (0x8000u - (kSmallScale << 7))) & 0x80008000u) != 0;
        } else {
          big |= load_byte(vs + 8 * n) >= kSmallScale;
        }
      }
      if (__any_sync(0xffffffffu, big)) lead = 0.f;
    }
    // The reference moves when a logit exceeds it, and is then put 8 above, so that it seldom moves.  Weights are at most
    // 1, the largest at least 2^-8: weight times value keeps to the value's range.
    if (__any_sync(0xffffffffu, mx[0] > m[0] + lead || mx[1] > m[1] + lead)) {
      const float ahead = lead > 0.f ? -kSmallBehind : kAhead;
      float sm[2];
#pragma unroll
      for (int i = 0; i < 2; ++i) {
#pragma unroll
        for (int k = 4; k < 32; k <<= 1) mx[i] = fmaxf(mx[i], __shfl_xor_sync(0xffffffffu, mx[i], k));
        const float to = mx[i] > m[i] + lead ? mx[i] + ahead : m[i];
        sm[i] = m[i] == -INFINITY ? 0.f : ex2(m[i] - to);
        m[i] = to;
      }
      const f32x2 s01 = two(sm[0], sm[1]);
      l = mul2(l, s01);
#pragma unroll
      for (int t = 0; t < OT; ++t) {
        split(mul2(two(o[t][0], o[t][1]), s01), o[t][0], o[t][1]);
        split(mul2(two(o[t][2], o[t][3]), s01), o[t][2], o[t][3]);
      }
    }
    // (a query that no token had a weight for yet has nothing to subtract)
    const f32x2 mr = two(m[0] == -INFINITY ? 0.f : -m[0], m[1] == -INFINITY ? 0.f : -m[1]);
    // ---- weights and V p, 16 tokens at a time
#pragma unroll
    for (int kk = 0; kk < NT / 2; ++kk) {
      const uint32_t vb = sb + S::HALF + kk * 16 * S::RB;
      const int vr = ((mi & 1) << 3) + tr;
      float w[2][2];                            // of tokens r and r + 8
#pragma unroll
      for (int j = 0; j < 2; ++j) {
        split(add2(x[2 * kk + j], mr), w[j][0], w[j][1]);
        w[j][0] = ex2(w[j][0]);
        w[j][1] = ex2(w[j][1]);
        l = add2(l, two(w[j][0], w[j][1]));
      }
      if constexpr (!INT4) {
        uint32_t hi[2], lo[2];
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          if constexpr (!PLAIN) {               // the row's scale
            const float f = e8m0(load_byte(vs + 16 * kk + 8 * j));
            split(mul2(two(w[j][0], w[j][1]), two(f, f)), w[j][0], w[j][1]);
          }
          pair_bf16(w[j][0], w[j][1], hi[j], lo[j]);
          hi[j] = transpose8(hi[j]);
          lo[j] = transpose8(lo[j]);
        }
        if constexpr (PLAIN) {
          const int off = vr * S::RB + (((mi >> 1) ^ tr) << 4);
#pragma unroll
          for (int t = 0; t < OT; ++t) {
            uint32_t v[4];
            ldsm4t(vb + (off ^ (t << 5)), v);
            mma<true>(o[t], v[0], v[2], v[1], v[3], hi[0], hi[1]);
            mma<true>(o[t], v[0], v[2], v[1], v[3], lo[0], lo[1]);
          }
        } else {
          const int off = S::RB == 128 ? vr * 128 + (((mi >> 1) ^ tr) << 4) : vr * 64 + (((mi >> 1) ^ (tr >> 1)) << 4);
#pragma unroll
          for (int i = 0; i < OT / 2; ++i) {
            uint32_t v[4];
            ldsm4t(vb + (off ^ (i << 5)), v);
#pragma unroll
            for (int j = 0; j < 2; ++j) {       // a word: channels 2r, 2r + 1 of token 2qd, the same of token 2qd + 1
              const uint32_t a = __byte_perm(v[2 * j], 0u, 0x3120), b = __byte_perm(v[2 * j + 1], 0u, 0x3120);
              const uint32_t a0 = f16x2_to_bf16x2(e4m3_lo_to_f16x2(a)), a1 = f16x2_to_bf16x2(e4m3_hi_to_f16x2(a));
              const uint32_t a2 = f16x2_to_bf16x2(e4m3_lo_to_f16x2(b)), a3 = f16x2_to_bf16x2(e4m3_hi_to_f16x2(b));
              mma<true>(o[2 * i + j], a0, a1, a2, a3, hi[0], hi[1]);
              mma<true>(o[2 * i + j], a0, a1, a2, a3, lo[0], lo[1]);
            }
          }
        }
      } else {
        // weights are transposed as pairs, once, and meet the scales of their tokens behind that
        uint32_t wh[2], wl[2];                  // query r, tokens 2qd, 2qd + 1 and the same + 8
        uint32_t sc[2][NG];                     // their scales: NG / 2 words a token
#pragma unroll
        for (int j = 0; j < 2; ++j) {
          wh[j] = pack_bf16(w[j][0], w[j][1]);
          wl[j] = transpose8(pack_bf16(w[j][0] - bf16lo(wh[j]), w[j][1] - bf16hi(wh[j])));
          wh[j] = transpose8(wh[j]);
          load_scales2(vs2 + (16 * kk + 8 * j) * S::SB, sc[j]);
        }
        const int off = S::RB == 64 ? vr * 64 + (((mi >> 1) ^ (tr >> 1)) << 4) : vr * 32 + (((mi >> 1) ^ (tr >> 2)) << 4);
#pragma unroll
        for (int g2 = 0; g2 < NG / 2; ++g2) {
          uint32_t v[4];
          ldsm4t(vb + (off ^ (g2 << 5)), v);
#pragma unroll
          for (int j = 0; j < 2; ++j) {         // a word: channels 4r .. 4r + 3 of token 2qd, the same of token 2qd + 1
            const int g = 2 * g2 + j;
            uint32_t hi[2], lo[2];
#pragma unroll
            for (int t = 0; t < 2; ++t) {
              const uint32_t f = __byte_perm(sc[t][g2], sc[t][NG / 2 + g2], j ? 0x7632 : 0x5410);
              scale_pair(wh[t], wl[t], f, hi[t], lo[t]);
            }
            const uint32_t a = v[2 * j], b = v[2 * j + 1], a8 = a >> 8, b8 = b >> 8;
            uint32_t a0 = int4_lo_to_bf16x2(a), a1 = int4_hi_to_bf16x2(a), a2 = int4_lo_to_bf16x2(b), a3 = int4_hi_to_bf16x2(b);
            mma<true>(o[2 * g], a0, a1, a2, a3, hi[0], hi[1]);
            mma<true>(o[2 * g], a0, a1, a2, a3, lo[0], lo[1]);
            a0 = int4_lo_to_bf16x2(a8), a1 = int4_hi_to_bf16x2(a8), a2 = int4_lo_to_bf16x2(b8), a3 = int4_hi_to_bf16x2(b8);
            mma<true>(o[2 * g + 1], a0, a1, a2, a3, hi[0], hi[1]);
            mma<true>(o[2 * g + 1], a0, a1, a2, a3, lo[0], lo[1]);
          }
        }
      }
    }
  }

  // the lane's accumulators: f(first channel, values[WIDTH] of query 2qd, of query 2qd + 1)
  template <typename F>
  __device__ __forceinline__ void each(int lane, F f) const {
    const int r = lane >> 2;
#pragma unroll
    for (int i = 0; i < D / (8 * WIDTH); ++i) {
      float a[WIDTH], b[WIDTH];
      if constexpr (PLAIN) {
        a[0] = o[i >> 1][2 * (i & 1)];
        b[0] = o[i >> 1][2 * (i & 1) + 1];
      } else {
#pragma unroll
        for (int h = 0; h < WIDTH / 2; ++h) {
          a[2 * h] = o[i * (WIDTH / 2) + h][0];
          a[2 * h + 1] = o[i * (WIDTH / 2) + h][2];
          b[2 * h] = o[i * (WIDTH / 2) + h][1];
          b[2 * h + 1] = o[i * (WIDTH / 2) + h][3];
        }
      }
      f(8 * WIDTH * i + WIDTH * r, a, b);
    }
  }
  __device__ __forceinline__ void end() {
    float a, b;
    split(l, a, b);
#pragma unroll
    for (int k = 4; k < 32; k <<= 1) {
      a += __shfl_xor_sync(0xffffffffu, a, k);
      b += __shfl_xor_sync(0xffffffffu, b, k);
    }
    l = two(a, b);
  }
  static __device__ __forceinline__ void put(float* to, const float (&v)[WIDTH]) {
    if constexpr (WIDTH == 1) *to = v[0];
    else if constexpr (WIDTH == 2) *(float2*)to = make_float2(v[0], v[1]);
    else *(float4*)to = make_float4(v[0], v[1], v[2], v[3]);
  }
  __device__ __forceinline__ void store_record(Record<D>* rec, int G, int lane) const {
    const int q0 = 2 * (lane & 3);
    float ls[2];
    split(l, ls[0], ls[1]);
    if (lane < 4) {
#pragma unroll
      for (int i = 0; i < 2; ++i)
        if (q0 + i < G) rec->s[q0 + i] = make_float2(m[i], ls[i]);
    }
    each(lane, [&](int c, const float (&a)[WIDTH], const float (&b)[WIDTH]) {
      if (q0 < G) put(&rec->o[q0][c], a);
      if (q0 + 1 < G) put(&rec->o[q0 + 1][c], b);
    });
  }
  __device__ __forceinline__ void store_out(void* out, float* lse, int G, int lane) const;
};

// Factor that turns joined accumulators into outputs: 0 where no token counted.  Tokens whose logits are all -infinity
// have no softmax: 1 / 0 times accumulators of 0, a NaN.  (A NaN logit leaves m alone, not l.)
template <int FMT>
__device__ __forceinline__ float finish(float m, float l) {
  return m == -INFINITY && l == 0.f ? 0.f : (FMT == THINK_PAGE_INT4 ? kInt4Unit : 1.f) / l;
}
// four joined accumulators to four outputs of EO bytes
template <int EO>
__device__ __forceinline__ void put4(void* to, const float4& a, float f) {
  const float4 x = f == 0.f ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(a.x * f, a.y * f, a.z * f, a.w * f);
  if (EO == 4) *(float4*)to = x;
  else *(uint2*)to = make_uint2(pack_bf16(x.x, x.y), pack_bf16(x.z, x.w));
}
// m + log2(l) in natural logarithms; l's exponent meets m first, of which it takes back what weights' reference is off
__device__ __forceinline__ float log_sum(float m, float l) {
  if (l == 0.f) return -INFINITY;
  if (!(l <= FLT_MAX)) return l;                 // NaN
  const uint32_t u = __float_as_uint(l);
  const int e = (int)(u >> 23) - 127;            // (l is no subnormal: the largest weight is at least 2^-8)
  return (m + (float)e + log2f(__uint_as_float((u & 0x007fffffu) | 0x3f800000u))) * 0.693147180559945309f;
}

template <int D, int FMT>
__device__ __forceinline__ void MmaState<D, FMT>::store_out(void* out, float* lse, int G, int lane) const {
  const int q0 = 2 * (lane & 3);
  float ls[2];
  split(l, ls[0], ls[1]);
  const float f0 = finish<FMT>(m[0], ls[0]), f1 = finish<FMT>(m[1], ls[1]);
  __nv_bfloat16* const po = (__nv_bfloat16*)out + q0 * D;
  auto write = [&](__nv_bfloat16* to, const float (&v)[WIDTH], float f) {
    if constexpr (WIDTH == 1) {
      *to = __float2bfloat16_rn(f == 0.f ? 0.f : v[0] * f);
    } else {
      uint32_t w[(WIDTH + 1) / 2];
#pragma unroll
      for (int i = 0; i < WIDTH / 2; ++i) w[i] = f == 0.f ? 0u : pack_bf16(v[2 * i] * f, v[2 * i + 1] * f);
      if constexpr (WIDTH == 2) *(uint32_t*)to = w[0];
      else *(uint2*)to = make_uint2(w[0], w[1]);
    }
  };
  each(lane, [&](int c, const float (&a)[WIDTH], const float (&b)[WIDTH]) {
    if (q0 < G) write(po + c, a, f0);
    if (q0 + 1 < G) write(po + D + c, b, f1);
  });
  if (lse && lane < 4) {
#pragma unroll
    for (int i = 0; i < 2; ++i)
      if (q0 + i < G) lse[q0 + i] = log_sum(m[i], ls[i]);
  }
}

// ---------------------------------------------------------------------------------------------------------
// fp32: a lane owns D / 32 channels.  The products of a step's tokens with the group's queries are NV partial sums a
// lane, reduced over the lanes by halving exchanges (each exchange adds two lanes' halves and keeps one half), after
// which the lane owns the logits idx = owner(lane) .. of (query g = idx / ST, token t = idx % ST).
template <int D, int GP>
struct F32State {
  using S = Shape<D, 4, THINK_PAGE_PLAIN, GP>;
  static constexpr int N = D / 32, ST = S::ST, NV = GP * ST;
  static __host__ __device__ constexpr int log2c(int x) { return x <= 1 ? 0 : 1 + log2c(x / 2); }
  static constexpr int NB = log2c(NV), LB = NB < 5 ? NB : 5, R = NV >> LB;   // idx bits, of which in the lane, values a lane
  static constexpr int TB = log2c(ST);

  float q[GP][N], o[GP][N];
  float m, l;                // of query owner(lane) / ST; l: this lane's tokens only
  float* sp;                 // the warp's NV weights in shared memory

  static __device__ __forceinline__ int owner(int lane) { return (lane >> (5 - LB)) * R; }

  struct Raw { float q[GP][N]; };
  static __device__ __forceinline__ void fetch(const void* qg, int G, int lane, Raw& raw) {
#pragma unroll
    for (int g = 0; g < GP; ++g)
#pragma unroll
      for (int i = 0; i < N; ++i) raw.q[g][i] = g < G ? ((const float*)qg)[g * D + lane * N + i] : 0.f;
  }
  __device__ __forceinline__ void begin(const Raw& raw, float scale_log2, int lane) {
#pragma unroll
    for (int g = 0; g < GP; ++g)
#pragma unroll
      for (int i = 0; i < N; ++i) {
        q[g][i] = raw.q[g][i] * scale_log2;
        o[g][i] = 0.f;
      }
    m = -INFINITY;
    l = 0.f;
  }
  static __device__ __forceinline__ void load(uint32_t a, float (&v)[N]) {
    if constexpr (N == 4)
      asm volatile("ld.shared.v4.f32 {%0,%1,%2,%3}, [%4];" : "=f"(v[0]), "=f"(v[1]), "=f"(v[2]), "=f"(v[3]) : "r"(a));
    else
      asm volatile("ld.shared.v2.f32 {%0,%1}, [%2];" : "=f"(v[0]), "=f"(v[1]) : "r"(a));
  }
  __device__ __forceinline__ void step(uint32_t sb, int ntok, int lane) {
    float x[NV];
#pragma unroll
    for (int t = 0; t < ST; ++t) {
      float k[N];
      load(sb + t * S::RB + lane * N * 4, k);
#pragma unroll
      for (int g = 0; g < GP; ++g) {
        float a = q[g][0] * k[0];
#pragma unroll
        for (int i = 1; i < N; ++i) a = fmaf(q[g][i], k[i], a);
        x[g * ST + t] = a;
      }
    }
#pragma unroll
    for (int b = 0; b < LB; ++b) {
      const bool up = lane & (16 >> b);
#pragma unroll
      for (int i = 0; i < (NV >> (b + 1)); ++i) {
        const float lo = x[i], hi = x[i + (NV >> (b + 1))];
        x[i] = (up ? hi : lo) + __shfl_xor_sync(0xffffffffu, up ? lo : hi, 16 >> b);
      }
    }
#pragma unroll
    for (int b = LB; b < 5; ++b)
#pragma unroll
      for (int i = 0; i < R; ++i) x[i] += __shfl_xor_sync(0xffffffffu, x[i], 16 >> b);
    const int idx = owner(lane);
    float mx = ntok > 0 ? kLowest : -INFINITY;
#pragma unroll
    for (int i = 0; i < R; ++i) {
      if (((idx + i) & (ST - 1)) >= ntok) x[i] = -INFINITY;
      mx = fmaxf(mx, x[i]);
    }
    // over the other lanes of the same query: idx bits log2(R) .. TB - 1
    constexpr int RB_ = log2c(R);
#pragma unroll
    for (int b = RB_; b < TB; ++b) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, 1 << (b - RB_ + 5 - LB)));
    if (__any_sync(0xffffffffu, mx > m)) {
      const float mn = fmaxf(m, mx), sc = m == -INFINITY ? 0.f : exp2f(m - mn);
      m = mn;
      l *= sc;
#pragma unroll
      for (int g = 0; g < GP; ++g) {
        const float s = __shfl_sync(0xffffffffu, sc, (g * ST / R) << (5 - LB));
#pragma unroll
        for (int i = 0; i < N; ++i) o[g][i] *= s;
      }
    }
    const float mr = m == -INFINITY ? 0.f : m;
    const bool first = (lane & ((1 << (5 - LB)) - 1)) == 0;     // lanes that share logits: one of them counts
#pragma unroll
    for (int i = 0; i < R; ++i) {
      const float p = exp2f(x[i] - mr);
      if (first) {
        l += p;
        sp[idx + i] = p;
      }
    }
    __syncwarp();
#pragma unroll
    for (int t0 = 0; t0 < ST; t0 += 4) {
      float v[4][N];
#pragma unroll
      for (int t = 0; t < 4; ++t) load(sb + S::HALF + (t0 + t) * S::RB + lane * N * 4, v[t]);
#pragma unroll
      for (int g = 0; g < GP; ++g) {
        const float4 p = *(const float4*)(sp + g * ST + t0);
#pragma unroll
        for (int i = 0; i < N; ++i)
          o[g][i] = fmaf(p.w, v[3][i], fmaf(p.z, v[2][i], fmaf(p.y, v[1][i], fmaf(p.x, v[0][i], o[g][i]))));
      }
    }
    __syncwarp();
  }
  __device__ __forceinline__ void end() {
    constexpr int RB_ = log2c(R);
#pragma unroll
    for (int b = RB_; b < TB; ++b) l += __shfl_xor_sync(0xffffffffu, l, 1 << (b - RB_ + 5 - LB));
    l = __shfl_sync(0xffffffffu, l, threadIdx.x & 31 & ~((1 << (5 - LB)) - 1));
  }
  __device__ __forceinline__ void store_record(Record<D>* r, int G, int lane) const {
#pragma unroll
    for (int g = 0; g < GP; ++g) {
      if (g >= G) break;
      if (lane == (g * ST / R) << (5 - LB)) r->s[g] = make_float2(m, l);
#pragma unroll
      for (int i = 0; i < N; i += 2) *(float2*)&r->o[g][lane * N + i] = make_float2(o[g][i], o[g][i + 1]);
    }
  }
  __device__ __forceinline__ void store_out(void* out, float* lse, int G, int lane) const {
#pragma unroll
    for (int g = 0; g < GP; ++g) {
      const int src = (g * ST / R) << (5 - LB);
      const float mg = __shfl_sync(0xffffffffu, m, src), lg = __shfl_sync(0xffffffffu, l, src);
      if (g < G) {
        const float f = finish<THINK_PAGE_PLAIN>(mg, lg);
#pragma unroll
        for (int i = 0; i < N; ++i) ((float*)out)[g * D + lane * N + i] = f == 0.f ? 0.f : o[g][i] * f;
        if (lse && lane == 0) lse[g] = log_sum(mg, lg);
      }
    }
  }
};

template <int D, int E, int FMT, int GP>
struct StateOf { using type = MmaState<D, FMT>; };
template <int D, int GP>
struct StateOf<D, 4, THINK_PAGE_PLAIN, GP> { using type = F32State<D, GP>; };

constexpr int kSpBytes = 256;        // fp32: a warp's weights of a step, read 16 bytes at a time

// shared memory behind the rings
struct alignas(16) Shared {
  WarpInfo info[kMaxWarps];
  int2 warp_sum[kMaxWarps];
  int valid[kMaxWarps][8];   // tokens that count in the stage
  int join[2];               // contributors to the units that this CTA joins
};

template <int D, int E, int FMT, int GP>
__global__ void __launch_bounds__((Shape<D, E, FMT, GP>::THREADS), 1) k_paged_decode(PagedDecodeParams p) {
  using S = Shape<D, E, FMT, GP>;
  constexpr int kWarps = S::WARPS, kThreads = S::THREADS;
  using State = typename StateOf<D, E, FMT, GP>::type;
  constexpr int EO = E;                         // bytes of an output element
  extern __shared__ __align__(128) unsigned char smem[];
  Shared& sh = *(Shared*)(smem + kWarps * (S::RING + (E == 4 ? kSpBytes : 0)));
  int* const cum = (int*)(&sh + 1);
  uint8_t* const last = (uint8_t*)(cum + p.table.B + 1);
  const int tid = threadIdx.x, lane = tid & 31;
  // Which part of the CTA's tiles this warp takes.  Parts that are a tile larger come at regular distances; neighbours
  // share a scheduler (the hardware's warps w, w + 4, ...), so that whatever the distance each gets its share of them.
  const int warp = (tid >> 5 & 3) * (kWarps / 4) + (tid >> 7);
  const int B = p.table.B, LH = p.nlayers * p.g.N_kv, grid = gridDim.x, cta = blockIdx.x;

  begin_dependent();
  // ---- tiles of every sequence, cumulated
  bool empty = false;
  Weights wt;
  {
    const int per = (B + kThreads - 1) / kThreads, b0 = min(B, tid * per), b1 = min(B, b0 + per);
    const int cap = p.table.max_pages * kPageTokens;
    int mine = 0, some = 0;                     // tiles, sequences that have any
    for (int b = b0; b < b1; ++b) {
      int n = load_now(p.seq_len + b);
      if (n > cap) {
        n = cap;
        if (cta == 0) atomicOr(p.error, kErrPage);
      }
      const int nt = n > 0 ? (n + kPageTokens - 1) / kPageTokens : 0;
      empty |= nt == 0;
      some += nt > 0;
      last[b] = (uint8_t)((n + kPageTokens - 1) & (kPageTokens - 1));
      cum[b + 1] = nt;
      mine += nt;
    }
    int x = mine, y = some;
#pragma unroll
    for (int o = 1; o < 32; o <<= 1) {
      const int xo = __shfl_up_sync(0xffffffffu, x, o), yo = __shfl_up_sync(0xffffffffu, y, o);
      if (lane >= o) {
        x += xo;
        y += yo;
      }
    }
    if (lane == 31) sh.warp_sum[tid >> 5] = make_int2(x, y);
    empty = __syncthreads_or(empty);
    int tiles = x - mine, seqs = y - some, all_tiles = 0, all_seqs = 0;
    for (int w = 0; w < kWarps; ++w) {
      const int2 t = sh.warp_sum[w];
      if (w < tid >> 5) {
        tiles += t.x;
        seqs += t.y;
      }
      all_tiles += t.x;
      all_seqs += t.y;
    }
    wt = weights_for(S::weights(), (int64_t)all_tiles * LH, (int64_t)all_seqs * LH, grid);
    for (int b = b0; b < b1; ++b) {
      const int nt = cum[b + 1];
      tiles += nt;
      seqs += nt > 0;
      cum[b + 1] = wt.tile * tiles + wt.unit * seqs;
    }
    if (tid == 0) cum[0] = 0;
    __syncthreads();
  }
  const Tables tab = {cum, last, wt, B, p.nlayers, p.g.N_kv};

  // ---- sequences without tokens
  if (empty) {
    for (int64_t i = (int64_t)cta * kWarps + warp; i < (int64_t)B * LH; i += (int64_t)grid * kWarps) {
      const int b = (int)div_wide(i, LH);
      if (cum[b + 1] != cum[b]) continue;
      const int64_t row = i * p.G;              // units in order are query rows in order
      uint4* const o = (uint4*)((uint8_t*)p.out + row * D * EO);
      for (int e = lane; e < p.G * D * EO / 16; e += 32) o[e] = make_uint4(0u, 0u, 0u, 0u);
      if (p.lse && lane < p.G) p.lse[row + lane] = -INFINITY;
    }
  }

  const int64_t total = (int64_t)cum[B] * LH;
  if (total == 0) return;
  const int64_t F0 = split_begin(total, grid, cta), F1 = split_begin(total, grid, cta + 1);
  const int64_t f0 = F0 + split_begin(F1 - F0, kWarps, warp), f1 = F0 + split_begin(F1 - F0, kWarps, warp + 1);
  // fewer tiles than CTAs: a CTA has one tile or none
  const bool sparse = wt.unit == 0 && total < grid;
  if (sparse && F0 == F1) return;
  Cursor c = {};
  if (f0 < f1) c = locate(tab, f0);
  const bool busy_warp = f0 < f1 && c.us + wt.slot(c.j) < f1;
  Record<D>* const records = (Record<D>*)p.records;
  Record<D>* const cta_rec = records + 2 * cta;                                         // units shared with other CTAs
  Record<D>* const head_rec = records + 2 * grid + (cta * kWarps + warp);               // the warp's first unit
  Record<D>* const tail_rec = (Record<D>*)(smem + warp * S::RING);                      // its last unit
  if (lane == 0) sh.info[warp].busy = busy_warp;

  if (busy_warp) {
    const uint32_t ring = smem_u32(smem) + warp * S::RING;
    State st;
    if constexpr (E == 4) st.sp = (float*)(smem + kWarps * S::RING + warp * kSpBytes);

    // ---- producer: fills the ring tile after tile
    const int q_bytes = p.G * D * E;            // queries of a unit, in the order of units
    const int64_t page_bytes = (int64_t)p.g.N_kv * p.g.block_bytes;
    Cursor pc = c;
    typename State::Raw raw;                    // the first unit's queries, asked for ahead of the pages
    State::fetch((const uint8_t*)p.q + (int64_t)(pc.b * LH + pc.ll * p.g.N_kv + pc.h) * q_bytes, p.G, lane, raw);
    const int32_t* p_entry = p.table.table + pc.b * p.table.stride + pc.j;       // table entry of the next tile
    int p_page = load_now(p_entry);                // looked up a tile ahead
    const uint8_t* p_base = p.pages + page_block_offset(p.g, p.layer0 + pc.ll, 0, pc.h);    // of the unit
    int p_tiles = min(pc.nt, wt.first_tile(f1 - pc.us)) - pc.j;                  // of the unit, not begun
    int p_toks = pc.len - pc.j * kPageTokens;                                    // of the unit, not begun
    uint32_t p_slot = ring;                     // next stage to fill
    int p_ntok = 0;                             // rows of the current tile that are left
    bool p_ok = false;
    const uint8_t* p_row = nullptr;             // its next key row
    const uint8_t* p_scale = nullptr;           // and scale
    int* p_valid = sh.valid[warp];
    auto open_tile = [&]() {
      p_ok = (uint32_t)p_page < (uint32_t)p.g.num_pages;
      if (!p_ok && lane == 0) atomicOr(p.error, kErrPage);
      p_row = p_base + (p_ok ? p_page : 0) * page_bytes;
      if (S::SB > 0) p_scale = p_row + 2 * kPageTokens * S::RB;
      p_ntok = min(kPageTokens, p_toks);
      p_toks -= kPageTokens;
      ++p_entry;
      if (--p_tiles == 0 && pc.us + wt.cost(pc.nt) < f1) {
        next_unit(tab, pc);
        p_entry = p.table.table + pc.b * p.table.stride;
        p_base = p.pages + page_block_offset(p.g, p.layer0 + pc.ll, 0, pc.h);
        p_tiles = min(pc.nt, wt.first_tile(f1 - pc.us));
        p_toks = pc.len;
      }
      if (p_tiles > 0) p_page = load_now(p_entry);
    };
    constexpr int CPR = S::RB / 16, RPI = 32 / CPR > 0 ? 32 / CPR : 1, IT = S::HALF / 512;
    constexpr int SC = S::SB > 0 ? S::ST * S::SB / 16 : 1;   // 16-byte pieces of a step's key scales
    static_assert(2 * SC <= 32 && S::ST * S::SB % 16 == 0, "one piece a lane");
    const int r0 = CPR < 32 ? lane / CPR : 0, ck = lane % CPR;
    const int s_part = lane / SC, s_at = 16 * (lane % SC);
    const uint32_t s_dst = 2 * S::HALF + s_part * S::ST * S::SB + s_at;
    const int s_src = s_part * kPageTokens * S::SB + s_at;
    auto issue = [&]() {
      if (p_ntok <= 0 && p_tiles > 0) open_tile();
      if (p_ntok > 0) {
        const int n = p_ok ? min(S::ST, p_ntok) : 0;
        const uint8_t* const kl = p_row + lane * 16;
        if (n == S::ST) {
#pragma unroll
          for (int it = 0; it < IT; ++it) {
            const uint32_t d = p_slot + (S::F32 ? it * 512 + lane * 16 : swz<S::RB>(it * RPI + r0, ck));
            cp16(d, kl + it * 512);
            cp16(d + S::HALF, kl + kPageTokens * S::RB + it * 512);
          }
          if (S::SB > 0 && lane < 2 * SC) cp16(p_slot + s_dst, p_scale + s_src);
        } else {                                // rows that do not count become zeros
#pragma unroll 1
          for (int it = 0; it < IT; ++it) {
            const int r = S::F32 ? (it * 512 + lane * 16) / S::RB : it * RPI + r0;
            const uint32_t d = p_slot + (S::F32 ? it * 512 + lane * 16 : swz<S::RB>(r, ck));
            const int bytes = r < n ? 16 : 0;   // (the address is in the pool in any case)
            cp16(d, kl + it * 512, bytes);
            cp16(d + S::HALF, kl + kPageTokens * S::RB + it * 512, bytes);
          }
          if (S::SB > 0 && lane < 2 * SC) cp16(p_slot + s_dst, p_scale + s_src, max(0, min(16, n * S::SB - s_at)));
        }
        if (lane == 0) *p_valid = n;
        p_ntok -= S::ST;
        p_row += S::HALF;
        if (S::SB > 0) p_scale += S::ST * S::SB;
      }
      cp_commit();                              // one group a call, possibly empty
      p_slot += S::STAGE;
      ++p_valid;
      if (p_slot == ring + S::RING) {
        p_slot = ring;
        p_valid = sh.valid[warp];
      }
    };
#pragma unroll 1
    for (int i = 0; i < S::STAGES - 1; ++i) issue();

    // ---- consumer: unit after unit
    uint32_t c_slot = ring;
    const int* c_valid = sh.valid[warp];
    bool first = true;                          // the warp's first unit
    while (true) {
      const int j1 = min(c.nt, wt.first_tile(f1 - c.us));    // its tiles c.j .. j1 - 1
      const int64_t ul = c.us + wt.slot(c.nt - 1);
      const bool is_last = c.us + wt.cost(c.nt) >= f1, whole = c.j == 0 && j1 == c.nt;
      const int ntok = min(c.len, j1 * kPageTokens) - c.j * kPageTokens;
      const int unit = c.b * LH + c.ll * p.g.N_kv + c.h;
      const int64_t row = (int64_t)unit * p.G;   // first query row
      if (!first) State::fetch((const uint8_t*)p.q + row * D * E, p.G, lane, raw);
      st.begin(raw, p.scale_log2, lane);
      // the next unit's queries come while this one is worked on (it may be one of an empty sequence)
      if (!is_last) touch((const uint8_t*)p.q + (row + p.G) * D * E, q_bytes, lane);
#pragma unroll 1
      for (int left = ntok; left > 0; left -= S::ST) {
        cp_wait<S::STAGES - 2>();
        __syncwarp();                           // the step has landed; all lanes are done with the slot before
        const int n = *c_valid;
        issue();
        st.step(c_slot, n, lane);
        c_slot += S::STAGE;
        ++c_valid;
        if (c_slot == ring + S::RING) {
          c_slot = ring;
          c_valid = sh.valid[warp];
        }
      }
      st.end();
      if (whole) {
        st.store_out((uint8_t*)p.out + row * D * EO, p.lse ? p.lse + row : nullptr, p.G, lane);
      } else if (sparse) {                      // the CTA's only tile: nothing to join here
        st.store_record(cta_rec + (c.us < F0 ? 0 : 1), p.G, lane);
      } else if (is_last) {
        cp_wait<0>();
        __syncwarp();
        st.store_record(tail_rec, p.G, lane);
      } else {                                  // the end of a unit that an earlier warp, or CTA, began
        const bool from_before = c.us < F0 && wt.first_tile(F0 - c.us) == c.j;     // an earlier CTA, no earlier warp
        st.store_record(from_before ? cta_rec : head_rec, p.G, lane);
      }
      if (lane == 0) {
        WarpInfo& wi = sh.info[warp];
        if (first) {
          wi.first_unit = unit;
          wi.first_us = c.us;
          wi.first_ul = ul;
        }
        wi.last_unit = unit;
        wi.last_us = c.us;
        wi.last_ul = ul;
      }
      first = false;
      if (is_last) break;
      next_unit(tab, c);
    }
    cp_wait<0>();
  }
  __syncthreads();

  // ---- Joins inside the CTA.  The warps whose last unit is the same share its join: each takes some of the
  // accumulators.  The states: those of these warps, and of the next one if it finished the unit and went on.  (A unit
  // that the CTA's first warp only finishes is one state, already where it belongs.)
  const uint32_t busy = __ballot_sync(0xffffffffu, lane < kWarps && sh.info[lane < kWarps ? lane : 0].busy);
  if (busy == 0) return;
  const int first_warp = __ffs(busy) - 1, last_warp = 31 - __clz(busy);
  const int64_t us = sh.info[warp].last_us, ul = sh.info[warp].last_ul;
  if (busy_warp && !sparse && !(us >= f0 && ul < f1)) {
    const int unit = sh.info[warp].last_unit;
    const uint32_t same = busy & __ballot_sync(0xffffffffu, lane < kWarps && sh.info[lane < kWarps ? lane : 0].last_unit == unit);
    const int helpers = __popc(same), me = __popc(same & ((1u << warp) - 1u));
    uint64_t list = 0;                          // these warps, 4 bits each (with few tiles, not all neighbours have any)
#pragma unroll
    for (int v = 0, k = 0; v < kWarps; ++v)
      if (same >> v & 1) {
        list |= (uint64_t)v << k;
        k += 4;
      }
    const int end_warp = 32 - __clz(same);                             // behind the last of them
    const uint32_t on = busy >> end_warp << end_warp;                  // the next one that has tiles
    const int extra = on ? __ffs(on) - 1 : -1;
    const bool more = extra >= 0 && sh.info[extra].first_unit == unit;
    const int n = helpers + more;
    auto rec = [&](int i) -> const Record<D>* {                        // state i, in token order
      return i == helpers ? records + 2 * grid + (cta * kWarps + extra) : (const Record<D>*)(smem + ((int)(list >> (4 * i)) & 15) * S::RING);
    };
    // statistics: lane = query head + 8 * (a quarter of the states)
    float* const weight = (float*)(smem + warp * S::RING + sizeof(Record<D>));        // [state][query head]
    const int g8 = lane & 7;
    constexpr int QN = kWarps / 4 + 1;          // states of a lane at most
    float2 t[QN];
    float m = -INFINITY, l = 0.f;
#pragma unroll
    for (int k = 0; k < QN; ++k) {
      const int i = (lane >> 3) + 4 * k;
      t[k] = i < n && g8 < p.G ? rec(i)->s[g8] : make_float2(-INFINITY, 0.f);
      m = fmaxf(m, t[k].x);
    }
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 8));
    m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, 16));
    const float ms = m == -INFINITY ? 0.f : m;
#pragma unroll
    for (int k = 0; k < QN; ++k) {
      const int i = (lane >> 3) + 4 * k;
      const float w = ex2(t[k].x - ms);
      l = fmaf(t[k].y, w, l);
      if (i < n) weight[i * kMaxG + g8] = w;
    }
    l += __shfl_xor_sync(0xffffffffu, l, 8);
    l += __shfl_xor_sync(0xffffffffu, l, 16);
    __syncwarp();
    const bool open = us < F0 || ul >= F1;
    Record<D>* const to = cta_rec + (us < F0 ? 0 : 1);
    const int64_t row = (int64_t)unit * p.G;
    const float f = finish<FMT>(m, l);
    if (me == 0 && lane < p.G) {
      if (open) {
        to->s[lane] = make_float2(m, l);
      } else if (p.lse) {
        p.lse[row + lane] = log_sum(m, l);
      }
    }
    // accumulators, 128 at a time, four a lane
#pragma unroll 1
    for (int e = 128 * me + 4 * lane; e - 4 * lane < p.G * D; e += 128 * helpers) {
      const int g = (e / D) & 7;
      const float fg = __shfl_sync(0xffffffffu, f, g);
      if (e < p.G * D) {
        float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
#pragma unroll 4
        for (int i = 0; i < n; ++i) {
          const float w = weight[i * kMaxG + g];
          const float4 x = *(const float4*)&rec(i)->o[g][e % D];
          a.x = fmaf(w, x.x, a.x);
          a.y = fmaf(w, x.y, a.y);
          a.z = fmaf(w, x.z, a.z);
          a.w = fmaf(w, x.w, a.w);
        }
        if (open) *(float4*)&to->o[g][e % D] = a;
        else put4<EO>((uint8_t*)p.out + (row * D + e) * EO, a, fg);
      }
    }
  }

  // ---- Units shared between CTAs, at most one with earlier and one with later CTAs: the last to arrive joins.
  const WarpInfo& wa = sh.info[first_warp];
  const WarpInfo& wb = sh.info[last_warp];
  const bool before = wa.first_us < F0, after = wb.last_us >= F0 && wb.last_ul >= F1;
  if (!before && !after) return;
  __syncthreads();
  if (tid < 2) {
    int join = 0;                               // contributors, if this CTA joins them
    if (tid == 0 ? before : after) {
      const int64_t ts = tid == 0 ? wa.first_us : wb.last_us, tl = tid == 0 ? wa.first_ul : wb.last_ul;
      uint32_t* const ticket = p.counters + (tid == 0 ? wa.first_unit : wb.last_unit);
      const int n = sparse ? (int)(tl - ts) + 1 : split_owner(total, grid, tl) - split_owner(total, grid, ts) + 1;
      // after the barrier the whole CTA's states are ordered before this thread's release
      if (ticket_add(ticket) == (unsigned)(n - 1)) {
        *ticket = 0u;                           // ready for the next call
        join = n;
      }
    }
    sh.join[tid] = join;
  }
  __syncthreads();
  // a warp takes 128 accumulators (four a lane, LPG lanes a query head) of every `slices`-th contributor: of all of them
  // if they are few.  (The order of the sums must not depend on which CTA joins, and so on what else it joins.)  Two
  // units with few take half of the warps each (one after the other, the CTAs that end last cost 1 to 2 us more)
  constexpr int LPG = D / 4;
  constexpr int AHEAD = 6;                      // states whose accumulators come while the statistics are made
  const int chunks = (p.G * D + 127) / 128, n0 = sh.join[0], n1 = sh.join[1];
  const bool halves = n0 > 0 && n0 <= AHEAD && n1 > 0 && n1 <= AHEAD && 2 * chunks <= kWarps;
  const int team = halves ? kWarps / 2 : kWarps, team0 = warp - warp % team;
  const int chunk = (warp - team0) % chunks, slice = (warp - team0) / chunks;
#pragma unroll 1
  for (int round = 0; round < (halves ? 1 : 2); ++round) {
    const int k = halves ? team0 > 0 : round;
    const int n = k == 0 ? n0 : n1;
    if (n == 0) continue;
    const int slices = n <= AHEAD ? 1 : kWarps / chunks;
    const int64_t ts = k == 0 ? wa.first_us : wb.last_us;
    const int c0 = split_owner(total, grid, ts);
    const int64_t row = (int64_t)(k == 0 ? wa.first_unit : wb.last_unit) * p.G;
    const int e = 128 * chunk + 4 * lane;
    const bool on = e < p.G * D && slice < slices;
    const int g = on ? e / D : 0;
    // the unit began in the first contributor (its record 1); for all others it is the unit that they began with
    auto record = [&](int i) -> const Record<D>* {
      return records + 2 * (sparse ? split_owner(total, grid, ts + i) : c0 + i) + (i == 0);
    };
    float4 y[AHEAD];
#pragma unroll
    for (int j = 0; j < AHEAD; ++j)
      if (on && slice + j * slices < n) y[j] = __ldcg((const float4*)&record(slice + j * slices)->o[g][e % D]);
    float2* const st = (float2*)(smem + warp * S::RING) + (lane / LPG) * kSMs;          // m, l of contributor i, then its weight
    float m = -INFINITY, l = 0.f;
#pragma unroll 1
    for (int i = lane % LPG; i < n; i += LPG) {
      const float2 x = __ldcg(&record(i)->s[g]);
      st[i] = x;
      m = fmaxf(m, x.x);
    }
#pragma unroll
    for (int o = 1; o < LPG; o <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, o));
    const float ms = m == -INFINITY ? 0.f : m;
#pragma unroll 1
    for (int i = lane % LPG; i < n; i += LPG) {
      const float2 x = st[i];
      const float w = ex2(x.x - ms);
      l = fmaf(x.y, w, l);
      st[i].x = w;
    }
#pragma unroll
    for (int o = 1; o < LPG; o <<= 1) l += __shfl_xor_sync(0xffffffffu, l, o);
    __syncwarp();
    float4 a = make_float4(0.f, 0.f, 0.f, 0.f);
    auto add = [&](float w, const float4& v) {
      a.x = fmaf(w, v.x, a.x);
      a.y = fmaf(w, v.y, a.y);
      a.z = fmaf(w, v.z, a.z);
      a.w = fmaf(w, v.w, a.w);
    };
    if (on) {
#pragma unroll
      for (int j = 0; j < AHEAD; ++j)
        if (slice + j * slices < n) add(st[slice + j * slices].x, y[j]);
#pragma unroll 4
      for (int i = slice + AHEAD * slices; i < n; i += slices) add(st[i].x, __ldcg((const float4*)&record(i)->o[g][e % D]));
    }
    // a slice leaves its sums behind its statistics
    auto part = [&](int s) { return (float4*)(smem + (team0 + s * chunks + chunk) * S::RING + kSMs * 2 * sizeof(float2)) + lane; };
    if (slice > 0 && slice < slices) *part(slice) = a;
    __syncthreads();
    if (on && slice == 0) {
#pragma unroll 1
      for (int s = 1; s < slices; ++s) add(1.f, *part(s));
      put4<EO>((uint8_t*)p.out + (row * D + e) * EO, a, finish<FMT>(m, l));
      if (p.lse && e % D == 0) p.lse[row + g] = log_sum(m, l);
    }
    __syncthreads();                            // before the other unit's join takes the same memory
  }
}

template <int D, int E, int FMT, int GP>
constexpr size_t smem_fixed() {
  using S = Shape<D, E, FMT, GP>;
  return (size_t)S::WARPS * (S::RING + (E == 4 ? kSpBytes : 0)) + sizeof(Shared);
}
inline size_t smem_tables(int B) { return ((size_t)(B + 1) * 4 + B + 15) / 16 * 16; }

template <int D, int E, int FMT, int GP>
cudaError_t launch_k(const PagedDecodeParams& p, cudaStream_t s) {
  const size_t smem = smem_fixed<D, E, FMT, GP>() + smem_tables(p.table.B);
  return launch_dependent(k_paged_decode<D, E, FMT, GP>, dim3(p.grid), Shape<D, E, FMT, GP>::THREADS, smem, s, p);
}
template <int D, int E, int FMT, int GP>
cudaError_t setup_k() {
  static_assert(smem_fixed<D, E, FMT, GP>() + kMaxPagedBatch * 5 + 32 <= 227 * 1024, "shared memory of a CTA");
  return cudaFuncSetAttribute(k_paged_decode<D, E, FMT, GP>, cudaFuncAttributeMaxDynamicSharedMemorySize,
                              (int)(smem_fixed<D, E, FMT, GP>() + smem_tables(kMaxPagedBatch)));
}

#define THINK_PAGED_DISPATCH(FN, ...)                                                          \
  do {                                                                                         \
    if (dtype == THINK_F32) switch (gp) {                                                      \
      case 1: return D == 128 ? FN<128, 4, THINK_PAGE_PLAIN, 1>(__VA_ARGS__) : FN<64, 4, THINK_PAGE_PLAIN, 1>(__VA_ARGS__); \
      case 2: return D == 128 ? FN<128, 4, THINK_PAGE_PLAIN, 2>(__VA_ARGS__) : FN<64, 4, THINK_PAGE_PLAIN, 2>(__VA_ARGS__); \
      case 4: return D == 128 ? FN<128, 4, THINK_PAGE_PLAIN, 4>(__VA_ARGS__) : FN<64, 4, THINK_PAGE_PLAIN, 4>(__VA_ARGS__); \
      default: return D == 128 ? FN<128, 4, THINK_PAGE_PLAIN, 8>(__VA_ARGS__) : FN<64, 4, THINK_PAGE_PLAIN, 8>(__VA_ARGS__); \
    }                                                                                          \
    switch (format) {                                                                          \
      case THINK_PAGE_PLAIN: return D == 128 ? FN<128, 2, THINK_PAGE_PLAIN, 8>(__VA_ARGS__) : FN<64, 2, THINK_PAGE_PLAIN, 8>(__VA_ARGS__); \
      case THINK_PAGE_E4M3: return D == 128 ? FN<128, 2, THINK_PAGE_E4M3, 8>(__VA_ARGS__) : FN<64, 2, THINK_PAGE_E4M3, 8>(__VA_ARGS__); \
      default: return D == 128 ? FN<128, 2, THINK_PAGE_INT4, 8>(__VA_ARGS__) : FN<64, 2, THINK_PAGE_INT4, 8>(__VA_ARGS__); \
    }                                                                                          \
  } while (0)

int padded_group(int G) { return G <= 1 ? 1 : G <= 2 ? 2 : G <= 4 ? 4 : 8; }

}  // namespace

cudaError_t launch_paged_decode(const PagedDecodeParams& p, int dtype, int format, cudaStream_t s) {
  const int D = p.g.D, gp = padded_group(p.G);
  THINK_PAGED_DISPATCH(launch_k, p, s);
}
cudaError_t paged_decode_setup(int dtype, int format, int D, int G) {
  const int gp = padded_group(G);
  THINK_PAGED_DISPATCH(setup_k);
}
// two records a CTA for units shared between CTAs, one a warp for units shared between warps
size_t paged_decode_record_bytes(int ctas) {
  static_assert(sizeof(Record<128>) >= sizeof(Record<64>), "the larger one");
  return (size_t)ctas * (2 + kMaxWarps) * sizeof(Record<128>);
}

}  // namespace think
