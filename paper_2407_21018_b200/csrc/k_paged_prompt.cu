// Attention of many new tokens of each sequence over its pages (causal), on CUDA cores in fp32, and the kernel that joins
// the pieces of items that were cut.
//
// out_s = sum_t w_t V_t / sum_t w_t, w_t = 2^(x_t - m), x = scale log2(e) q_s K_t, over the tokens t <= pos + s, in one
// pass over tiles of 64 tokens with the running maximum m and sum of a softmax.
//
// fp32 caches keep fp32 products, which the tensor cores do not have: a block has 64 rows of queries and a tile in shared
// memory, a thread 4 x 4 logits and 4 rows of outputs in registers.  Bound: shared memory reads (two 16-byte reads feed 16
// multiply-adds).  Short calls (two sequences of up to 512 tokens, 4 heads of 64: 44 us) are one item a block, 5 tiles in a row, and
// the join.  The cut into parts (paged_prompt.h) keeps one of those from having a long item all to itself.
#include <math.h>

#include "paged_prompt_walk.cuh"

namespace think {
namespace {

constexpr int kRows = 64, kTile = 64, kThreads = 256;
constexpr int kExtra = 64;              // see PromptCut

// A thread owns 4 rows (4 ty ..) and, of the logits, the tokens tx + 16 j, of the outputs the channels 4 tx + 64 j.
template <int D>
__global__ void __launch_bounds__(kThreads) k_paged_prompt_fp32(const PagedPromptParams p) {
  constexpr int RS = D + 4, PS = kTile + 4;         // row strides that keep 16-byte reads of neighbouring rows apart
  constexpr int J = D / 64;
  const PromptCut cut{kExtra};
  extern __shared__ __align__(16) float smem[];
  float* const sq = smem;
  float* const sk = sq + kRows * RS;
  float* const sv = sk + kTile * RS;
  float* const sp = sv + kTile * RS;
  begin_dependent();
  const int tid = threadIdx.x, ty = tid >> 4, tx = tid & 15;
  PromptDesc desc = {0, 0, 0, 0, 0};
  PromptWalk w;
  if (!prompt_walk_begin(p, cut, w)) {              // (every warp for itself)
    if (tid == 0) p.desc[blockIdx.x] = desc;
    return;
  }
  PromptPiece x;
  do {
    x = prompt_piece(p, cut, w);
    if (x.t0 == x.t1) continue;
    const int ll = p.by_heads.div(w.lh), h = w.lh - ll * p.g.N_kv;
    const int rows = x.tokens * p.G;
    for (int i = tid; i < kRows * (D / 4); i += kThreads) {
      const int r = i / (D / 4), c = 4 * (i % (D / 4)), s = p.by_group.div(r), g = r - s * p.G;
      float4 f = make_float4(0.f, 0.f, 0.f, 0.f);
      if (r < rows) f = *(const float4*)((const float*)p.q.ptr + prompt_row(p, p.q, w.b, w.s, x.s0 + s) + ll * p.q.sl + (h * p.G + g) * p.q.sn + c);
      *(float4*)(sq + r * RS + c) = make_float4(f.x * p.scale_log2, f.y * p.scale_log2, f.z * p.scale_log2, f.w * p.scale_log2);
    }
    int limit[4];                                   // tokens that a row sees
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int r = 4 * ty + a;
      limit[a] = r < rows ? min(x.n, w.s.pos + x.s0 + (int)p.by_group.div(r) + 1) : 0;
    }
    const int all_see = w.s.pos + x.s0 + 1;         // tokens that every row sees
    float m[4], l[4];
    bool any[4];
    float4 o[4][J];
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      m[a] = -INFINITY;
      l[a] = 0.f;
      any[a] = false;
#pragma unroll
      for (int j = 0; j < J; ++j) o[a][j] = make_float4(0.f, 0.f, 0.f, 0.f);
    }
    for (int t = x.t0; t < x.t1; ++t) {
      const int tok0 = t * kTile;
      const int page = tok0 < x.n ? page_of(p.table, p.g, w.b, tok0, p.error) : -1;
      if (page < 0) continue;                       // (the same in every thread)
      __syncthreads();                              // the last tile, and the queries' place, are no longer read
      const float* const block = (const float*)(p.pages + page_block_offset(p.g, p.layer0 + ll, page, h));
      for (int i = tid; i < kTile * (D / 4); i += kThreads) {
        const int r = i / (D / 4), c = 4 * (i % (D / 4));
        float4 k = make_float4(0.f, 0.f, 0.f, 0.f), v = k;
        if (tok0 + r < x.n) {
          k = *(const float4*)(block + r * D + c);
          v = *(const float4*)(block + (kPageTokens + r) * D + c);
        }
        *(float4*)(sk + r * RS + c) = k;
        *(float4*)(sv + r * RS + c) = v;
      }
      __syncthreads();
      float acc[4][4] = {};
#pragma unroll 4
      for (int c = 0; c < D; c += 4) {
        float4 qa[4], kb[4];
#pragma unroll
        for (int a = 0; a < 4; ++a) qa[a] = *(const float4*)(sq + (4 * ty + a) * RS + c);
#pragma unroll
        for (int j = 0; j < 4; ++j) kb[j] = *(const float4*)(sk + (tx + 16 * j) * RS + c);
#pragma unroll
        for (int a = 0; a < 4; ++a)
#pragma unroll
          for (int j = 0; j < 4; ++j)
            acc[a][j] = fmaf(qa[a].w, kb[j].w, fmaf(qa[a].z, kb[j].z, fmaf(qa[a].y, kb[j].y, fmaf(qa[a].x, kb[j].x, acc[a][j]))));
      }
#pragma unroll
      for (int a = 0; a < 4; ++a) {
        float mx = -INFINITY;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          if (tok0 + tx + 16 * j >= limit[a]) acc[a][j] = -INFINITY;
          mx = fmaxf(mx, acc[a][j]);
        }
#pragma unroll
        for (int s = 1; s < 16; s <<= 1) mx = fmaxf(mx, __shfl_xor_sync(0xffffffffu, mx, s));
        any[a] |= tok0 < limit[a];
        const float mn = fmaxf(m[a], mx), ref = mn == -INFINITY ? 0.f : mn;
        const float f = exp2f(m[a] - ref);
        m[a] = mn;
        float sum = 0.f;
#pragma unroll
        for (int j = 0; j < 4; ++j) {
          const float e = exp2f(acc[a][j] - ref);
          sum += e;
          sp[(4 * ty + a) * PS + tx + 16 * j] = e;
        }
        l[a] = fmaf(l[a], f, sum);
#pragma unroll
        for (int j = 0; j < J; ++j) {
          o[a][j].x *= f; o[a][j].y *= f; o[a][j].z *= f; o[a][j].w *= f;
        }
      }
      __syncwarp();                                 // a row's 16 threads are lanes of one warp
      const int seen = min(kTile, x.n - tok0);
      auto add = [&](int u, int a, float e) {
#pragma unroll
        for (int j = 0; j < J; ++j) {
          const float4 v = *(const float4*)(sv + u * RS + 4 * tx + 64 * j);
          o[a][j].x = fmaf(e, v.x, o[a][j].x);
          o[a][j].y = fmaf(e, v.y, o[a][j].y);
          o[a][j].z = fmaf(e, v.z, o[a][j].z);
          o[a][j].w = fmaf(e, v.w, o[a][j].w);
        }
      };
      if (tok0 + seen <= all_see) {
#pragma unroll 4
        for (int u = 0; u < seen; ++u)
#pragma unroll
          for (int a = 0; a < 4; ++a) add(u, a, sp[(4 * ty + a) * PS + u]);
      } else {                                      // a value that a row does not see may be a NaN: no product with 0
        for (int u = 0; u < seen; ++u)
#pragma unroll
          for (int a = 0; a < 4; ++a)
            if (tok0 + u < limit[a]) add(u, a, sp[(4 * ty + a) * PS + u]);
      }
    }
    const bool whole = x.t0 == 0 && x.t1 == x.tiles;
    float* const rec = (float*)p.records + (2 * blockIdx.x + (x.t0 == 0)) * prompt_record_floats(kRows, D);
#pragma unroll
    for (int a = 0; a < 4; ++a) {
      const int r = 4 * ty + a;
#pragma unroll
      for (int s = 1; s < 16; s <<= 1) l[a] += __shfl_xor_sync(0xffffffffu, l[a], s);
      if (r >= rows) continue;
      const bool none = m[a] == -INFINITY && !any[a];
      if (whole) {
        const int s = p.by_group.div(r), head = h * p.G + r - s * p.G;
        const float f = none ? 0.f : 1.f / l[a];
        const int64_t at = prompt_row(p, p.out, w.b, w.s, x.s0 + s) + ll * p.out.sl + head * p.out.sn + 4 * tx;
#pragma unroll
        for (int j = 0; j < J; ++j)
          *(float4*)((float*)p.out.ptr + at + 64 * j) =
              none ? make_float4(0.f, 0.f, 0.f, 0.f) : make_float4(o[a][j].x * f, o[a][j].y * f, o[a][j].z * f, o[a][j].w * f);
        if (p.lse && tx == 0) p.lse[(prompt_lse_row(p, w.b, w.s, x.s0 + s) * p.nlayers + ll) * p.N_q + head] = prompt_log_sum(m[a], l[a]);
      } else {
#pragma unroll
        for (int j = 0; j < J; ++j) *(float4*)(rec + r * D + 4 * tx + 64 * j) = o[a][j];
        if (tx == 0) {
          rec[kRows * D + r] = m[a];
          rec[kRows * (D + 1) + r] = m[a] == -INFINITY && l[a] == 0.f ? (any[a] ? 1.f : 0.f) : l[a];
        }
      }
    }
    if (x.t0 > 0) desc.carries = x.t1 == x.tiles ? 1 : 2;
    else if (!whole) desc = PromptDesc{w.lh, w.b, w.i, 1, desc.carries};
    __syncthreads();                                // the next item's queries take this one's place
  } while (prompt_walk_next(p, cut, w, x.cost));
  if (tid == 0) p.desc[blockIdx.x] = desc;
}

// Joins the pieces of the items that were cut, in their order: a warp per row, the states' statistics over its lanes.  Two blocks
// an SM: with more than 32 registers there is one, and a prompt of 8192 tokens takes 8 us longer.
constexpr int kJoinWarps = 32;
template <int D, int E, int ROWS>
__global__ void __launch_bounds__(32 * kJoinWarps, 2) k_paged_prompt_join(const PagedPromptParams p) {
  constexpr int W = D / 32;                         // channels of a lane
  begin_dependent();
  const PromptDesc d = p.desc[blockIdx.x];
  if (!d.names_item(p.table.B, p.nlayers * p.g.N_kv)) return;
  bool bad = false;
  const PromptSeq seq = prompt_seq(p, d.b, bad);
  const int lane = threadIdx.x & 31;
  int pieces = 2;                                   // up to the CTA that ends it
  for (int c = blockIdx.x + 1;; c += 32) {
    const uint32_t ends = __ballot_sync(0xffffffffu, c + lane < p.grid && p.desc[min(c + lane, p.grid - 1)].carries == 1);
    if (ends || c + 32 >= p.grid) {
      pieces = c - (int)blockIdx.x + __ffs(ends);
      break;
    }
  }
  const int r = blockIdx.y * kJoinWarps + (threadIdx.x >> 5);
  const int64_t s0 = (int64_t)d.item * p.per;
  const int rows = (int)max((int64_t)0, min((int64_t)p.per, seq.rows - s0)) * p.G;
  if (r >= rows) return;                            // (nor is there an item behind the sequence's last row)
  constexpr size_t kRec = (size_t)ROWS * (D + 2);
  auto rec = [&](int i) { return (const float*)p.records + (i == 0 ? 2 * blockIdx.x + 1 : 2 * (blockIdx.x + i)) * kRec; };
  float m = -INFINITY;
  bool any = false;
  auto there = [&](int i) { return i < pieces && (i == 0 || p.desc[blockIdx.x + i].carries != 0); };      // (a CTA may have no tile)
  for (int i = lane; i < pieces; i += 32) {
    if (!there(i)) continue;
    const float x = rec(i)[ROWS * D + r], y = rec(i)[ROWS * (D + 1) + r];
    any |= !(y == 0.f);
    m = fmaxf(m, x);
  }
#pragma unroll
  for (int s = 1; s < 32; s <<= 1) m = fmaxf(m, __shfl_xor_sync(0xffffffffu, m, s));
  any = __any_sync(0xffffffffu, any);
  float o[W] = {}, l = 0.f;
  for (int i0 = 0; i0 < pieces; i0 += 32) {
    const int i = i0 + lane;
    float f = 0.f, fl = 0.f;
    bool some = false;                              // tokens: their values count however small their weights (0 times infinity is a NaN)
    if (there(i)) {
      const float x = rec(i)[ROWS * D + r], y = rec(i)[ROWS * (D + 1) + r];
      some = !(y == 0.f);
      f = x == -INFINITY ? (y == y ? 0.f : y) : exp2f(x - m);      // (a sum may be NaN under a maximum of -infinity)
      fl = f * y;
    }
    const uint32_t with = __ballot_sync(0xffffffffu, some);
#pragma unroll 4
    for (int k = 0; k < min(32, pieces - i0); ++k) {
      const float g = __shfl_sync(0xffffffffu, f, k);
      l += __shfl_sync(0xffffffffu, fl, k);
      if (!(with >> k & 1)) continue;
      const float* const src = rec(i0 + k) + (size_t)r * D + lane * W;
      float v[W];
      if constexpr (W == 4) *(float4*)v = *(const float4*)src; else *(float2*)v = *(const float2*)src;
#pragma unroll
      for (int c = 0; c < W; ++c) o[c] = fmaf(g, v[c], o[c]);
    }
  }
  const int ll = p.by_heads.div(d.lh), h = d.lh - ll * p.g.N_kv, s = p.by_group.div(r), head = h * p.G + r - s * p.G;
  const bool none = m == -INFINITY && !any;
  const float f = 1.f / l;
#pragma unroll
  for (int c = 0; c < W; ++c) o[c] = none ? 0.f : o[c] * f;
  const int64_t at = prompt_row(p, p.out, d.b, seq, s0 + s) + ll * p.out.sl + head * p.out.sn + lane * W;
  if constexpr (E == 4) {
    float* const to = (float*)p.out.ptr + at;
    if constexpr (W == 4) *(float4*)to = *(const float4*)o; else *(float2*)to = *(const float2*)o;
  } else {
    uint32_t u[W / 2];
#pragma unroll
    for (int c = 0; c < W; c += 2) {
      const __nv_bfloat162 t = __floats2bfloat162_rn(o[c], o[c + 1]);
      u[c / 2] = *(const uint32_t*)&t;
    }
    uint16_t* const to = (uint16_t*)p.out.ptr + at;
    if constexpr (W == 4) *(uint2*)to = make_uint2(u[0], u[1]); else *(uint32_t*)to = u[0];
  }
  if (p.lse && lane == 0) p.lse[(prompt_lse_row(p, d.b, seq, s0 + s) * p.nlayers + ll) * p.N_q + head] = prompt_log_sum(m, l);
}

template <int D>
constexpr size_t fp32_smem() { return sizeof(float) * (size_t)((kRows + 2 * kTile) * (D + 4) + kRows * (kTile + 4)); }

template <int D>
cudaError_t launch_fp32(const PagedPromptParams& p, cudaStream_t s) {
  const cudaError_t e = launch_dependent(k_paged_prompt_fp32<D>, dim3(p.grid), kThreads, fp32_smem<D>(), s, p);
  return e != cudaSuccess ? e : launch_dependent(k_paged_prompt_join<D, 4, kRows>, dim3(p.grid, kRows / kJoinWarps), 32 * kJoinWarps, 0, s, p);
}
template <int D>
cudaError_t launch_tc(const PagedPromptParams& p, int format, const void* map, cudaStream_t s) {
  const cudaError_t e = launch_paged_prompt_tc(p, format, map, s);
  return e != cudaSuccess ? e : launch_dependent(k_paged_prompt_join<D, 2, 256>, dim3(p.grid, 256 / kJoinWarps), 32 * kJoinWarps, 0, s, p);
}
template <int D>
cudaError_t setup_fp32() {
  return cudaFuncSetAttribute(k_paged_prompt_fp32<D>, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)fp32_smem<D>());
}

}  // namespace

cudaError_t paged_prompt_setup(int dtype, int format, int D) {
  const cudaError_t e = dtype == THINK_BF16 ? paged_prompt_tc_setup(format, D) : D == 128 ? setup_fp32<128>() : setup_fp32<64>();
  if (e != cudaSuccess) (void)cudaGetLastError();    // reported by the call that needs the kernel
  return e;
}
int paged_prompt_rows(int dtype) { return dtype == THINK_BF16 ? paged_prompt_tc_rows() : kRows; }
PromptCut paged_prompt_cut(int dtype) { return dtype == THINK_BF16 ? paged_prompt_tc_cut() : PromptCut{kExtra}; }

cudaError_t launch_paged_prompt(const PagedPromptParams& p, int dtype, int format, const void* map, cudaStream_t s) {
  if (dtype == THINK_BF16) return p.g.D == 128 ? launch_tc<128>(p, format, map, s) : launch_tc<64>(p, format, map, s);
  return p.g.D == 128 ? launch_fp32<128>(p, s) : launch_fp32<64>(p, s);
}

}  // namespace think
