// Attention of one new token per sequence over the paged cache.
//
// One CTA per (entry, layer, key head); its four warps take tokens in turn, a lane owns D / 32 channels, the softmax
// runs online with fp32 maximum, sum and accumulators, and the warps' states are joined in warp order.
#include <cuda_fp8.h>
#include <math.h>

#include "paged_internal.h"

namespace think {
namespace {

constexpr int kThreads = 128;
constexpr int kWarps = kThreads / 32;

// channels [c0, c0 + N) of a stored row as fp32
template <int E, int FMT, int N>
__device__ __forceinline__ void load_row(const uint8_t* row, const uint8_t* scales, int c0, float (&x)[N]) {
  float f = 1.f;
  if (FMT == THINK_PAGE_E4M3) f = e8m0(*scales);
  if (FMT == THINK_PAGE_INT4) f = __uint_as_float((uint32_t)((const uint16_t*)scales)[c0 / kGroupChannels] << 16);
#pragma unroll
  for (int i = 0; i < N; ++i) {
    const int c = c0 + i;
    if (FMT == THINK_PAGE_PLAIN) {
      x[i] = E == 4 ? ((const float*)row)[c] : __bfloat162float(((const __nv_bfloat16*)row)[c]);
    } else if (FMT == THINK_PAGE_E4M3) {
      const __half_raw h = __nv_cvt_fp8_to_halfraw(row[c], __NV_E4M3);
      x[i] = __half2float(*(const __half*)&h) * f;
    } else {
      x[i] = (float)((int)(row[c >> 1] >> (4 * (c & 1)) & 15) - 8) * f;
    }
  }
}

template <int D, int E, int FMT>
__global__ void __launch_bounds__(kThreads) k_paged_decode(const PagedDecodeParams p) {
  constexpr int N = D / 32;
  __shared__ float so[kWarps][kMaxPagedGroup][D];
  __shared__ float sm[kWarps][kMaxPagedGroup], sl[kWarps][kMaxPagedGroup];
  const int lane = threadIdx.x & 31, warp = threadIdx.x >> 5;
  const int h = blockIdx.x % p.g.N_kv, ll = blockIdx.x / p.g.N_kv, b = blockIdx.y;
  const int cap = p.table.max_pages * kPageTokens;
  int len = __ldg(p.seq_len + b);
  if (len > cap) {
    if (threadIdx.x == 0) atomicOr(p.error, kErrPage);
    len = cap;
  }
  const int64_t q0 = ((int64_t)(b * p.nlayers + ll) * p.N_q + h * p.G);
  float q[kMaxPagedGroup][N], o[kMaxPagedGroup][N], m[kMaxPagedGroup], l[kMaxPagedGroup];
#pragma unroll
  for (int g = 0; g < kMaxPagedGroup; ++g) {
    m[g] = -INFINITY;
    l[g] = 0.f;
#pragma unroll
    for (int i = 0; i < N; ++i) {
      o[g][i] = 0.f;
      const int64_t e = (q0 + g) * D + lane * N + i;
      q[g][i] = g >= p.G ? 0.f : E == 4 ? ((const float*)p.q)[e] : __bfloat162float(((const __nv_bfloat16*)p.q)[e]);
      q[g][i] *= p.scale_log2;
    }
  }
  for (int t = warp; t < len; t += kWarps) {
    const int page = page_of(p.table, p.g, b, t, p.error);
    if (page < 0) continue;
    const uint8_t* block = p.pages + page_block_offset(p.g, p.layer0 + ll, page, h);
    const int slot = t & (kPageTokens - 1);
    float k[N], v[N];
    load_row<E, FMT, N>(block + page_part_offset(p.g, 0) + slot * p.g.row_bytes, block + page_part_offset(p.g, 2) + slot * p.g.scale_bytes, lane * N, k);
    load_row<E, FMT, N>(block + page_part_offset(p.g, 1) + slot * p.g.row_bytes, block + page_part_offset(p.g, 3) + slot * p.g.scale_bytes, lane * N, v);
#pragma unroll
    for (int g = 0; g < kMaxPagedGroup; ++g) {
      if (g >= p.G) break;
      float x = 0.f;
#pragma unroll
      for (int i = 0; i < N; ++i) x = fmaf(q[g][i], k[i], x);
#pragma unroll
      for (int i = 1; i < 32; i <<= 1) x += __shfl_xor_sync(0xffffffffu, x, i);
      const float mn = fmaxf(m[g], x), a = exp2f(m[g] - mn), w = exp2f(x - mn);
      m[g] = mn;
      l[g] = l[g] * a + w;
#pragma unroll
      for (int i = 0; i < N; ++i) o[g][i] = fmaf(w, v[i], o[g][i] * a);
    }
  }
#pragma unroll
  for (int g = 0; g < kMaxPagedGroup; ++g) {
    if (lane == 0) {
      sm[warp][g] = m[g];
      sl[warp][g] = l[g];
    }
#pragma unroll
    for (int i = 0; i < N; ++i) so[warp][g][lane * N + i] = o[g][i];
  }
  __syncthreads();
  for (int i = threadIdx.x; i < p.G * D; i += kThreads) {
    const int g = i / D, c = i % D;
    float M = -INFINITY, L = 0.f, x = 0.f;
    for (int w = 0; w < kWarps; ++w) M = fmaxf(M, sm[w][g]);
    if (M > -INFINITY) {
      for (int w = 0; w < kWarps; ++w) {
        const float a = exp2f(sm[w][g] - M);
        L += a * sl[w][g];
        x += a * so[w][g][c];
      }
      x /= L;
    }
    if (E == 4) ((float*)p.out)[(q0 + g) * D + c] = x;
    else ((__nv_bfloat16*)p.out)[(q0 + g) * D + c] = __float2bfloat16_rn(x);
    if (c == 0 && p.lse) p.lse[q0 + g] = M > -INFINITY ? (M + log2f(L)) * 0.69314718055994530942f : -INFINITY;
  }
}

template <int D>
cudaError_t launch_d(const PagedDecodeParams& p, int dtype, int format, cudaStream_t s) {
  const dim3 grid((unsigned)(p.nlayers * p.g.N_kv), (unsigned)p.table.B);
  if (dtype == THINK_F32) k_paged_decode<D, 4, THINK_PAGE_PLAIN><<<grid, kThreads, 0, s>>>(p);
  else if (format == THINK_PAGE_PLAIN) k_paged_decode<D, 2, THINK_PAGE_PLAIN><<<grid, kThreads, 0, s>>>(p);
  else if (format == THINK_PAGE_E4M3) k_paged_decode<D, 2, THINK_PAGE_E4M3><<<grid, kThreads, 0, s>>>(p);
  else k_paged_decode<D, 2, THINK_PAGE_INT4><<<grid, kThreads, 0, s>>>(p);
  return cudaGetLastError();
}

}  // namespace

cudaError_t launch_paged_decode(const PagedDecodeParams& p, int dtype, int format, cudaStream_t s) {
  return p.g.D == 128 ? launch_d<128>(p, dtype, format, s) : launch_d<64>(p, dtype, format, s);
}
cudaError_t paged_decode_setup(int, int, int) { return cudaSuccess; }
int paged_decode_max_ctas(int num_sms) { return num_sms; }
size_t paged_decode_record_bytes(int D, int G) { return rec_size(D, G); }

}  // namespace think
