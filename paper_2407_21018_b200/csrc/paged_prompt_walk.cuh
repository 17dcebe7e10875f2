// Device side of paged_prompt.h: the sequences of a call and a CTA's way along its part of the line.
#pragma once
#include "paged_internal.h"
#include "paged_prompt.h"

namespace think {

struct PagedPromptParams {
  PageGeom g;
  const uint8_t* pages;
  View5 q, out;               // [b][s][layer - layer0][head][D] or [s][..] from start[b] on; element strides
  float* lse;                 // dense, or null
  PageTableView table;
  const int32_t *pos, *rows, *start;      // or null: 0, max_rows, padded
  int max_rows;
  int N_q, G, per;            // per: new tokens of an item
  int layer0, nlayers;
  float scale_log2;           // on logits
  uint32_t q_scale2;          // on bf16 queries or on e4m3 keys, two bf16: see PromptScale
  uint32_t* error;
  PromptDesc* desc;           // one per CTA
  uint8_t* records;           // two per CTA
  int grid;
  FastDiv by_group, by_heads;
};

// A piece's state, row by row: O [rows][D] (not divided by l), m, l [rows].  m: the logit in base 2 that the weights are relative
// to, the largest one or up to 2^8 above it.  l = 0 and m = -infinity: no token; l = 1 with that m: tokens, but all their logits are -infinity.
__host__ __device__ inline size_t prompt_record_floats(int rows, int D) { return (size_t)rows * (D + 2); }

// `map`: of a bf16 cache of plain pages, the pool as rows of D elements in boxes of 64 x 64 (a CUtensorMap)
cudaError_t launch_paged_prompt(const PagedPromptParams& p, int dtype, int format, const void* map, cudaStream_t s);
cudaError_t paged_prompt_setup(int dtype, int format, int D);       // kernel attributes on the current device
int paged_prompt_rows(int dtype);                                   // query rows of an item
PromptCut paged_prompt_cut(int dtype);

cudaError_t launch_paged_prompt_tc(const PagedPromptParams& p, int format, const void* map, cudaStream_t s);
cudaError_t paged_prompt_tc_setup(int format, int D);
int paged_prompt_tc_rows();
PromptCut paged_prompt_tc_cut();

#ifdef __CUDACC__
struct PromptSeq {
  int pos, rows, start;
};
// Sequence b of a call with its counts cut to what there is; `bad`: something was out of range.
__device__ __forceinline__ PromptSeq prompt_seq(const PagedPromptParams& p, int b, bool& bad) {
  PromptSeq s;
  const int rows = p.rows ? load_now(p.rows + b) : p.max_rows;
  const int pos = p.pos ? load_now(p.pos + b) : 0;
  s.pos = min(pos, p.table.max_pages * kPageTokens);      // (pos + rows then fits 32 bits: checked on the host)
  s.start = p.start ? load_now(p.start + b) : 0;
  s.rows = max(0, min(rows, p.max_rows));
  bad |= rows > p.max_rows;
  if (p.start && s.rows > 0) {
    const int room = s.start >= 0 && s.start < p.max_rows ? p.max_rows - s.start : 0;
    bad |= s.rows > room;
    s.rows = min(s.rows, room);
  }
  bad |= s.rows > 0 && (pos < 0 || (int64_t)pos + s.rows > (int64_t)p.table.max_pages * kPageTokens);
  return s;
}
__device__ __forceinline__ PromptLine prompt_line(const PagedPromptParams& p, const PromptSeq& s, int extra) {
  return PromptLine{(int64_t)extra + max(s.pos, 0), s.rows, p.per};
}

// Place of row s of a sequence in q or out (in elements, head and layer aside) and in lse (in rows).
__device__ __forceinline__ int64_t prompt_row(const PagedPromptParams& p, const View5& v, int b, const PromptSeq& q, int s) {
  return p.start ? (int64_t)(q.start + s) * v.ss : b * v.sb + (int64_t)s * v.ss;
}
__device__ __forceinline__ int64_t prompt_lse_row(const PagedPromptParams& p, int b, const PromptSeq& q, int s) {
  return p.start ? q.start + s : (int64_t)b * p.max_rows + s;
}

struct PromptWalk {
  int64_t at, begin, end;     // where the item begins; the CTA's part of the line
  int lh, b, i;
  PromptSeq s;
};

// A warp; its lanes share the sequences.  False: the CTA has no part.
__device__ __forceinline__ bool prompt_walk_begin(const PagedPromptParams& p, const PromptCut& cut, PromptWalk& w) {
  const int lane = threadIdx.x & 31, B = p.table.B, per = (B + 31) >> 5, b0 = min(B, lane * per), b1 = min(B, b0 + per);
  bool bad = false;
  long long upto = 0, before = 0, place = 0, items = 0, items_before = 0, largest = 0, cost = 0;
  int owner = -1, pieces = 0, number = 0;
  // first the sums, then the lane with the CTA's place (or item) looks for it
#pragma unroll 1
  for (int pass = 0; pass < 2; ++pass) {
    long long sum = before, num = items_before;
#pragma unroll 1
    for (int b = b0; b < b1 && (pass == 0 || lane == owner); ++b) {
      const PromptSeq s = prompt_seq(p, b, bad);
      const PromptLine line = prompt_line(p, s, cut.extra);
      const long long n = line.total();
      const int m = line.items();
      if (pass == 1 && (pieces ? number < num + m : place < sum + n)) {
        w.b = b;
        w.i = pieces ? number - (int)num : line.find(place - sum);
        w.s = s;
        w.at = sum + line.begin(w.i);
        cost = line.cost(w.i);
        break;
      }
      sum += n;
      num += m;
      if (m > 0) largest = max(largest, (long long)line.cost(m - 1));
    }
    if (pass == 1) break;
    upto = sum;
    items = num;
#pragma unroll 1
    for (int o = 1; o < 32; o <<= 1) {
      const long long y = __shfl_up_sync(0xffffffffu, upto, o), z = __shfl_up_sync(0xffffffffu, items, o);
      if (lane >= o) {
        upto += y;
        items += z;
      }
      largest = max(largest, __shfl_xor_sync(0xffffffffu, largest, o));
    }
    before = upto - sum;
    items_before = items - num;
    const long long W = __shfl_sync(0xffffffffu, upto, 31), total = W * p.nlayers * p.g.N_kv;
    const long long each = __shfl_sync(0xffffffffu, items, 31), all = each * p.nlayers * p.g.N_kv;
    if (bad && blockIdx.x == 0) atomicOr(p.error, kErrPage);
    if (W == 0) return false;
    pieces = cut.pieces(total, all, largest, p.grid);
    if (pieces) {
      number = (int)blockIdx.x / pieces;
      if (number >= all) return false;
      w.lh = number / (int)each;
      number -= w.lh * (int)each;
    } else {
      const PromptShare share(total, p.grid);
      w.begin = share.begin(blockIdx.x);
      w.end = share.begin(blockIdx.x + 1);
      w.lh = prompt_quotient(w.begin, W);
      place = w.begin - w.lh * W;
    }
    owner = __ffs(__ballot_sync(0xffffffffu, pieces ? number < items : place < upto)) - 1;      // the first lane whose sequences reach behind it
    w.at = W;
  }
  const long long W = __shfl_sync(0xffffffffu, upto, 31);
  w.b = __shfl_sync(0xffffffffu, w.b, owner);
  w.i = __shfl_sync(0xffffffffu, w.i, owner);
  w.s.pos = __shfl_sync(0xffffffffu, w.s.pos, owner);
  w.s.rows = __shfl_sync(0xffffffffu, w.s.rows, owner);
  w.s.start = __shfl_sync(0xffffffffu, w.s.start, owner);
  w.at = w.lh * W + __shfl_sync(0xffffffffu, w.at, owner);
  if (pieces) {
    const PromptShare share(__shfl_sync(0xffffffffu, cost, owner), pieces);
    const int j = (int)blockIdx.x % pieces;
    w.begin = w.at + share.begin(j);
    w.end = w.at + share.begin(j + 1);
  }
  return w.begin < w.end;
}

// What of the current item belongs to this CTA.
struct PromptPiece {
  int s0, tokens;             // new tokens of the item: s0 .. s0 + tokens - 1
  int n;                      // tokens that its last row sees
  int tiles, t0, t1;          // tiles of the item, and those of this piece (none if t0 == t1)
  int64_t cost;
};
__device__ __forceinline__ PromptPiece prompt_piece(const PagedPromptParams& p, const PromptCut& cut, const PromptWalk& w) {
  PromptPiece x;
  x.cost = prompt_line(p, w.s, cut.extra).cost(w.i);
  x.s0 = w.i * p.per;
  x.tokens = min(p.per, w.s.rows - x.s0);
  x.n = (int)max((int64_t)0, min((int64_t)w.s.pos + x.s0 + x.tokens, (int64_t)p.table.max_pages * kPageTokens));
  x.tiles = max(1, (x.n + cut.tile - 1) / cut.tile);
  x.t0 = (int)min((int64_t)x.tiles, cut.first_tile(w.begin - w.at));
  x.t1 = (int)min((int64_t)x.tiles, cut.first_tile(w.end - w.at));
  return x;
}
// On to the next item; false at the end of the CTA's part.
__device__ __forceinline__ bool prompt_walk_next(const PagedPromptParams& p, const PromptCut& cut, PromptWalk& w, int64_t cost) {
  w.at += cost;
  if (w.at >= w.end) return false;
  bool bad = false;
  if ((int64_t)(w.i + 1) * p.per < w.s.rows) {
    ++w.i;
    return true;
  }
  w.i = 0;
  do {
    if (++w.b == p.table.B) {
      w.b = 0;
      ++w.lh;
    }
    w.s = prompt_seq(p, w.b, bad);
  } while (w.s.rows == 0);                  // some sequence has rows: the line is not at its end
  return true;
}

// (m + log2 l) in natural logarithms; l's exponent meets m first, so that small sums keep their bits
__device__ __forceinline__ float prompt_log_sum(float m, float l) {
  if (!(l <= 3.402823466e38f)) return l;     // NaN
  if (m == -INFINITY) return -INFINITY;
  const uint32_t u = __float_as_uint(l);
  const int e = (int)(u >> 23) - 127;
  return (m + (float)e + log2f(__uint_as_float((u & 0x007fffffu) | 0x3f800000u))) * 0.693147180559945309f;
}
#endif

}  // namespace think
