// Pages, positions and slots of a step from the sequences' lengths (integers only).
//
// A sequence of n tokens owns ceil(n / 64) pages, so what it gains or loses is known from its length and the wanted
// change alone.  Two sums over the sequences, in order, decide everything:
//   the pages given back stand behind the free ones, sequence after sequence;
//   the pages wanted are taken from the end of that list, first sequence first, for as long as they and the room for
//   tokens suffice (sums over all that was asked for, so that one large request is not passed by the ones behind it;
//   a sequence that needs no page is not held up by the lack of one).
// Every CTA of the one cluster computes the sums for itself from the inputs (a few thousand integers at most).  Then
// the CTAs share the pages, meet, and share the tokens.  Lengths and the count of free pages are stored behind that
// meeting, so inputs and results may be the same arrays; the pages taken are read below the old count and the ones given
// back are stored at or above it, so that one list serves as both, too.
// Bound: latency.  A step of 64 tokens is three dependent loads behind the launch; 100,000 tokens write 0.8 MB.  A call takes the host
// 8 us, which hides the kernel (4 us; 76,800 tokens of 256 sequences 10).
#include <cooperative_groups.h>

#include "paged_internal.h"

namespace think {
namespace {

namespace cg = cooperative_groups;

constexpr int kPer = 4;              // sequences of a thread: kMaxPagedBatch / 1024
constexpr int kParts = 32;           // warps, at most
__host__ __device__ constexpr size_t plan_smem(int B) { return sizeof(long long) * kParts + sizeof(int) * (4 * (size_t)B + 3); }

__host__ __device__ constexpr int pages_of(int n) { return (int)(((int64_t)n + kPageTokens - 1) / kPageTokens); }

// inclusive sum over the block's threads; `part`: a value per warp
__device__ __forceinline__ long long block_sum(long long x, long long* part, long long& total) {
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5, warps = blockDim.x >> 5;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, x, o);
    if (lane >= o) x += y;
  }
  if (lane == 31) part[warp] = x;
  __syncthreads();
  long long w = lane < warps ? part[lane] : 0;
#pragma unroll
  for (int o = 1; o < 32; o <<= 1) {
    const long long y = __shfl_up_sync(0xffffffffu, w, o);
    if (lane >= o) w += y;
  }
  total = __shfl_sync(0xffffffffu, w, 31);
  const long long before = __shfl_sync(0xffffffffu, w, warp > 0 ? warp - 1 : 0);
  __syncthreads();                                   // `part` may be used again
  return x + (warp > 0 ? before : 0);
}

// the last index i < n with at[i] <= x, for at[0] = 0 <= x
__device__ __forceinline__ int last_at_or_below(const int* at, int n, int x) {
  int lo = 0, hi = n - 1;
  while (lo < hi) {
    const int mid = (lo + hi + 1) >> 1;
    if (at[mid] <= x) lo = mid; else hi = mid - 1;
  }
  return lo;
}

__global__ void __launch_bounds__(1024) k_paged_plan(const PagedPlanParams p) {
  extern __shared__ long long smem[];
  long long* const s_part = smem;
  begin_dependent();
  const int tid = threadIdx.x, nt = blockDim.x, B = p.table.B;
  int* const s_start = (int*)(s_part + kParts);      // [B + 1] granted tokens in front of a sequence
  int* const s_held = s_start + B + 1;               // [B]     tokens held before, less what it loses
  int* const s_take = s_held + B;                    // [B + 1] pages taken in front of a sequence
  int* const s_give = s_take + B + 1;                // [B + 1] pages given back in front of a sequence
  const int per = (B + nt - 1) / nt;                 // neighbouring sequences of a thread, at most kPer
  const int b0 = tid * per;
  const int most = p.table.max_pages * kPageTokens;  // fits: checked on the host
  const int free_raw = load_now(p.free_count);
  const int F = max(0, min(free_raw, p.num_pages));
  bool bad = free_raw != F;

  int kept[kPer], ask[kPer], give[kPer], need[kPer];
  long long gave = 0, needs = 0, asks = 0;
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const bool on = i < per && b0 + i < B;
    const int n = on ? load_now(p.seq_len + b0 + i) : 0, change = on ? load_now(p.change + b0 + i) : 0;
    const int held = max(0, min(n, most));
    ask[i] = change > 0 && (long long)held + change <= most ? change : 0;
    kept[i] = change < 0 ? (int)max(0ll, (long long)held + change) : held;
    bad |= n > most || (change > 0 && ask[i] == 0);
    give[i] = pages_of(held) - pages_of(kept[i]);
    need[i] = pages_of(held + ask[i]) - pages_of(held);
    gave += give[i];
    needs += need[i];
    asks += ask[i];
  }
  long long given, needed, asked;
  long long at_give = block_sum(gave, s_part, given) - gave, at_take = block_sum(needs, s_part, needed) - needs;
  long long at_row = block_sum(asks, s_part, asked) - asks;
  const long long have = F + given;
  long long total_rows = asked, taken = needed;
  if (needed > have || asked > p.max_tokens) {       // (the same in every thread) some are refused
    long long n = at_take, a = at_row, rows = 0, take = 0;
#pragma unroll
    for (int i = 0; i < kPer; ++i) {
      n += need[i];
      a += ask[i];
      if ((need[i] != 0 && n > have) || a > p.max_tokens) ask[i] = need[i] = 0;
      rows += ask[i];
      take += need[i];
    }
    at_row = block_sum(rows, s_part, total_rows) - rows;
    at_take = block_sum(take, s_part, taken) - take;
  }
#pragma unroll
  for (int i = 0; i < kPer; ++i) {
    const int b = b0 + i;
    if (i < per && b < B) {
      s_start[b] = (int)at_row;
      s_held[b] = kept[i];
      s_take[b] = (int)at_take;
      s_give[b] = (int)at_give;
      if (blockIdx.x == 0) {
        p.pos[b] = kept[i];
        p.rows[b] = ask[i];
        p.start[b] = (int)at_row;
      }
      at_row += ask[i];
      at_take += need[i];
      at_give += give[i];
    }
  }
  if (tid == 0) {
    s_start[B] = (int)total_rows;
    s_take[B] = (int)taken;
    s_give[B] = (int)given;
    if (blockIdx.x == 0) p.start[B] = (int)total_rows;
  }
  __syncthreads();

  // ---- pages: place x of the list [free | given back]
  const int ctas = gridDim.x, me = blockIdx.x * nt + tid, all_threads = ctas * nt;
  auto page_at = [&](long long x) {
    int page;
    if (x < F) {
      page = load_now(p.free_pages + x);
    } else {
      const int i = (int)(x - F), b = last_at_or_below(s_give, B, i);
      page = load_now(p.table.table + b * p.table.stride + pages_of(s_held[b]) + (i - s_give[b]));
    }
    bad |= (uint32_t)page >= (uint32_t)p.num_pages;
    return page;
  };
  const long long left = have - taken;
  for (int i = me; i < (int)taken; i += all_threads) {
    const int b = last_at_or_below(s_take, B, i);
    p.table_out[b * p.table.stride + pages_of(s_held[b]) + (i - s_take[b])] = page_at(have - 1 - i);
  }
  for (long long x = F + me; x < left; x += all_threads) {
    const int page = page_at(x);
    if (x < p.num_pages) p.free_pages[x] = page;     // (more than the pool has: some were given back twice)
    else bad = true;
  }
  if (ctas > 1) cg::this_cluster().sync();           // every input has been read, the table is complete
  else __syncthreads();

  // ---- tokens, four neighbours a thread; nothing behind the last
  for (int i0 = 4 * me; i0 < p.max_tokens; i0 += 4 * all_threads) {
    int4 pos = make_int4(-1, -1, -1, -1), slot = pos;
    if (i0 < (int)total_rows) {
      int b = last_at_or_below(s_start, B, i0), page = -1, page_no = -1, page_b = -1;
#pragma unroll
      for (int j = 0; j < 4; ++j) {
        const int i = i0 + j;
        if (i < (int)total_rows) {
          while (i >= s_start[b + 1]) ++b;
          const int t = s_held[b] + (i - s_start[b]);
          if ((t >> 6) != page_no || b != page_b) {
            page_b = b;
            page_no = t >> 6;
            page = load_now(p.table.table + b * p.table.stride + page_no);
            bad |= (uint32_t)page >= (uint32_t)p.num_pages;
          }
          (&pos.x)[j] = t;
          (&slot.x)[j] = (uint32_t)page < (uint32_t)p.num_pages ? page * kPageTokens + (t & (kPageTokens - 1)) : -1;
        }
      }
    }
    if (i0 + 4 <= p.max_tokens) {
      *(int4*)(p.token_pos + i0) = pos;
      *(int4*)(p.slots + i0) = slot;
    } else {
      for (int j = 0; i0 + j < p.max_tokens; ++j) {
        p.token_pos[i0 + j] = (&pos.x)[j];
        p.slots[i0 + j] = (&slot.x)[j];
      }
    }
  }
  if (blockIdx.x == 0) {
    for (int b = tid; b < B; b += nt) p.seq_len_out[b] = s_held[b] + (s_start[b + 1] - s_start[b]);
    if (tid == 0) p.free_left[0] = (int)min(left, (long long)p.num_pages);
  }
  if (bad) atomicOr(p.error, kErrPage);
}

}  // namespace

// One CTA for as many sequences and tokens as it serves in the time that a cluster needs to meet; else a cluster of eight,
// the portable most.
cudaError_t launch_paged_plan(const PagedPlanParams& p, cudaStream_t s) {
  // One CTA saves the cluster's start and meeting (256 sequences, with the copies around it in a graph: 6 instead of 8.5 us), until
  // the tokens are too many for it (2048: 6.6 against 8.1 us; 7680: 13.9 against 8.4).
  const bool small = p.table.B <= 256 * kPer && p.max_tokens <= 2048;
  const int ctas = small ? 1 : 8, threads = small ? 256 : 1024;
  const size_t smem = plan_smem(p.table.B);          // all that the kernel has
  if (smem > 48 * 1024) {
    // (the same value in every call: calls of different sizes on several threads do not take it away from one another)
    const cudaError_t e = cudaFuncSetAttribute(k_paged_plan, cudaFuncAttributeMaxDynamicSharedMemorySize, (int)plan_smem(kMaxPagedBatch));
    if (e != cudaSuccess) {
      (void)cudaGetLastError();                      // reported here, not by the caller's next check
      return e;
    }
  }
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = dim3(ctas);
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[2];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  attr[1].id = cudaLaunchAttributeClusterDimension;
  attr[1].val.clusterDim.x = ctas;
  attr[1].val.clusterDim.y = attr[1].val.clusterDim.z = 1;
  cfg.attrs = attr;
  cfg.numAttrs = small ? 1 : 2;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, k_paged_plan, p);
  if (e != cudaSuccess) (void)cudaGetLastError();
  return e;
}

}  // namespace think
