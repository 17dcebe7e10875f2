// Shared by the translation units of the paged key-value cache.
#pragma once
#include <cuda_fp8.h>

#include "think_internal.h"

namespace think {

constexpr uint32_t kErrPage = 16u;     // device error word: page-table entry, position, length or row count out of range
constexpr int kPageTokens = kTileTokens;
constexpr int kGroupChannels = 32;     // channels that share a scale in 4-bit pages
constexpr int kMaxPagedBatch = 4096;
constexpr int kMaxPagedGroup = 8;      // query heads per key head

// The pool: [L][num_pages][N_kv] blocks of 64 key rows | 64 value rows | key scales | value scales.
struct PageGeom {
  int L, N_kv, D, num_pages;
  int row_bytes;             // one row of D codes
  int scale_bytes;           // scales of one row (0, 1 or 2 * D / 32)
  int block_bytes;
};

__host__ __device__ inline int page_part_offset(const PageGeom& g, int part) {
  const int a = kPageTokens * g.row_bytes, b = kPageTokens * g.scale_bytes;
  return part < 2 ? part * a : 2 * a + (part - 2) * b;
}
__host__ __device__ inline int64_t page_block_offset(const PageGeom& g, int layer, int page, int head) {
  return (((int64_t)layer * g.num_pages + page) * g.N_kv + head) * g.block_bytes;
}

// x / d and x % d for 0 <= x < 2^31 by one 32 x 32 -> 64 bit product (round-up reciprocal; exact over that range
// because the error of the reciprocal times x stays below 1 / d)
struct FastDiv {
  uint32_t d, mul, shift;
  FastDiv() = default;
  explicit FastDiv(uint32_t d_) : d(d_), mul(0), shift(0) {
    if (d_ <= 1) return;
    uint32_t s = 0;
    while ((1ull << s) < d_) ++s;                             // ceil(log2 d)
    shift = s - 1;
    mul = (uint32_t)(((1ull << (32 + shift)) + d_ - 1) / d_);
  }
  __host__ __device__ __forceinline__ uint32_t div(uint32_t x) const {
    if (d <= 1) return x;
#ifdef __CUDA_ARCH__
    return __umulhi(x, mul) >> shift;
#else
    return (uint32_t)(((uint64_t)x * mul) >> 32) >> shift;
#endif
  }
};

struct PageTableView {
  const int32_t* table;
  int64_t stride;
  int max_pages, B;
};

struct PagedRowsParams {     // rows <-> pages
  PageGeom g;
  View5 k, v;                // [b][s][layer - layer0][head][D], element strides
  uint8_t* pages;
  PageTableView table;
  const int32_t* pos;        // or null: 0
  const int32_t* rows;       // or null: max_rows
  int max_rows;
  int layer0, nlayers;
  FastDiv by_heads, by_layers;
  uint32_t* error;
};

struct PagedDecodeParams {
  PageGeom g;
  const uint8_t* pages;
  const void* q;             // [B][nlayers][N_q][D]
  void* out;
  float* lse;                // [B][nlayers][N_q] or null
  PageTableView table;
  const int32_t* seq_len;
  int N_q, G;
  int layer0, nlayers;
  float scale_log2;          // softmax scale * log2(e)
  uint32_t* error;
  uint32_t* counters;        // one ticket per unit of the call, zero between calls
  uint8_t* records;          // partial states
  int grid;
};

cudaError_t launch_paged_rows(const PagedRowsParams& p, int dtype, int format, bool write, cudaStream_t s);
cudaError_t launch_paged_decode(const PagedDecodeParams& p, int dtype, int format, cudaStream_t s);
cudaError_t paged_decode_setup(int dtype, int format, int D, int G);   // kernel attributes on the current device
size_t paged_decode_record_bytes(int ctas);             // partial states of a launch of that many CTAs, any head dimension

// Launches a kernel that begins with begin_dependent(): it may be set up while the kernel ahead of it in the stream
// finishes.
template <typename Params>
inline cudaError_t launch_dependent(void (*kernel)(Params), dim3 grid, int threads, size_t smem, cudaStream_t s, const Params& p) {
  cudaLaunchConfig_t cfg = {};
  cfg.gridDim = grid;
  cfg.blockDim = dim3(threads);
  cfg.dynamicSmemBytes = smem;
  cfg.stream = s;
  cudaLaunchAttribute attr[1];
  attr[0].id = cudaLaunchAttributeProgrammaticStreamSerialization;
  attr[0].val.programmaticStreamSerializationAllowed = 1;
  cfg.attrs = attr;
  cfg.numAttrs = 1;
  const cudaError_t e = cudaLaunchKernelEx(&cfg, kernel, p);
  if (e != cudaSuccess) (void)cudaGetLastError();            // reported here, not by the caller's next check
  return e;
}

#ifdef __CUDACC__
// Lets the next kernel of the stream be set up, then waits until everything ahead of this one has completed and can be
// read.  Every thread of such a kernel calls it before anything else and before any return: the next kernel only waits
// for this one, so this one must not complete ahead of its own predecessors.
__device__ __forceinline__ void begin_dependent() {
  asm volatile("griddepcontrol.launch_dependents;" ::: "memory");
  asm volatile("griddepcontrol.wait;" ::: "memory");
}

// A load that stays behind begin_dependent() and does not go by the read-only path: what it reads may have been written
// by a kernel that was still running when this one was set up.
__device__ __forceinline__ int32_t load_now(const int32_t* p) {
  int32_t x;
  asm volatile("ld.global.s32 %0, [%1];" : "=r"(x) : "l"(p));
  return x;
}

// Page that holds token t of entry b, or -1 (error bit) if the table or the position is out of range.
__device__ __forceinline__ int page_of(const PageTableView& t, const PageGeom& g, int b, int64_t tok, uint32_t* error) {
  int page = -1;
  if (tok >= 0 && tok < (int64_t)t.max_pages * kPageTokens) page = load_now(t.table + b * t.stride + (tok >> 6));
  if ((uint32_t)page >= (uint32_t)g.num_pages) {
    atomicOr(error, kErrPage);
    return -1;
  }
  return page;
}

// two fp32 in a register pair: one instruction for both
using f32x2 = unsigned long long;
__device__ __forceinline__ f32x2 two(float a, float b) {
  f32x2 r;
  asm("mov.b64 %0, {%1, %2};" : "=l"(r) : "f"(a), "f"(b));
  return r;
}
__device__ __forceinline__ void split(f32x2 v, float& a, float& b) { asm("mov.b64 {%0, %1}, %2;" : "=f"(a), "=f"(b) : "l"(v)); }
__device__ __forceinline__ f32x2 fma2(f32x2 a, f32x2 b, f32x2 c) {
  f32x2 r;
  asm("fma.rn.f32x2 %0, %1, %2, %3;" : "=l"(r) : "l"(a), "l"(b), "l"(c));
  return r;
}
__device__ __forceinline__ f32x2 mul2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("mul.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}
__device__ __forceinline__ f32x2 add2(f32x2 a, f32x2 b) {
  f32x2 r;
  asm("add.rn.f32x2 %0, %1, %2;" : "=l"(r) : "l"(a), "l"(b));
  return r;
}

// value of a scale byte e of an e4m3 row: 2^(e - 127), which for byte 0 is a subnormal; byte 255 is NaN.  (One conversion;
// selecting the two ends by hand cost the attention 9 %.)
__device__ __forceinline__ float e8m0(uint32_t e) {
  return __uint_as_float((uint32_t)__nv_cvt_e8m0_to_bf16raw((__nv_fp8_storage_t)e).x << 16);
}
#endif

}  // namespace think
