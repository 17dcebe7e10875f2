// Rows of the paged cache: quantised as they are written, dequantised as they are read back.
//
// Both directions only move bytes (512 bytes of bf16 key and value against 258 or 144 stored ones a row at
// D = 128), so the DRAM stream is the bound and the kernels are one pass: a lane owns 16 bytes of a row's elements
// (8 bf16 or 4 fp32 channels) of the key AND of the value, both loads in flight before anything waits, the row's (or
// group's) maximum goes over the lanes of the row by shuffles, and codes leave from registers.  The lanes of a warp
// hold consecutive rows with the head running fastest, which is the order of the [b, s, l, n, d] tensors: loads are
// whole 128-byte lines, and the stores of a row are one contiguous piece of its page.
#include <cuda_fp8.h>

#include "paged_internal.h"

namespace think {
namespace {

constexpr int kRowThreads = 256;

// largest |x| of 8 bf16 as the integer of its bits: orders finite < infinite < NaN
__device__ __forceinline__ uint32_t amax_bits(const uint4& w) {
  uint32_t m = __vmaxu2(__vmaxu2(w.x & 0x7fff7fffu, w.y & 0x7fff7fffu), __vmaxu2(w.z & 0x7fff7fffu, w.w & 0x7fff7fffu));
  return max(m >> 16, m & 0xffffu);
}
template <int LANES>
__device__ __forceinline__ uint32_t lane_max(uint32_t x) {
#pragma unroll
  for (int o = 1; o < LANES; o <<= 1) x = max(x, __shfl_xor_sync(0xffffffffu, x, o));
  return x;
}
constexpr uint32_t kInfBits = 0x7f80u;   // bf16 infinity: anything at or above is not finite

__device__ __forceinline__ uint32_t e4m3x4(float a, float b, float c, float d) {
  const uint32_t lo = __nv_cvt_float2_to_fp8x2(make_float2(a, b), __NV_SATFINITE, __NV_E4M3);
  const uint32_t hi = __nv_cvt_float2_to_fp8x2(make_float2(c, d), __NV_SATFINITE, __NV_E4M3);
  return lo | (hi << 16);
}

// 8 bf16 -> 8 e4m3 codes; LANES lanes hold the row.  `e` receives the scale byte.
template <int LANES>
__device__ __forceinline__ uint2 encode_e4m3(const uint4& w, uint32_t& e, bool& bad) {
  const uint32_t top = lane_max<LANES>(amax_bits(w));
  bad = top >= kInfBits;
  // top = 1.m * 2^(E - 127): 448 = 1.75 * 2^8, so the scale's exponent is E - 8, one more if 1.m > 1.75
  const int k = max((int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0), -126);
  e = (uint32_t)(k + 127);
  if (bad) {
    e = 127u;
    return make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
  }
  const float inv = __uint_as_float((uint32_t)(127 - k) << 23);    // 2^-k: the product is exact, the code rounds once
  return make_uint2(e4m3x4(bf16lo(w.x) * inv, bf16hi(w.x) * inv, bf16lo(w.y) * inv, bf16hi(w.y) * inv),
                    e4m3x4(bf16lo(w.z) * inv, bf16hi(w.z) * inv, bf16lo(w.w) * inv, bf16hi(w.w) * inv));
}

// 8 bf16 -> 8 4-bit codes; 4 lanes hold the group of 32 channels.  `sbits` receives the bf16 scale.
// The quotient is an IEEE division: x and s have 8 significant bits each, so a quotient that is no tie is at least
// 2^-12 away from one and the fp32 rounding cannot cross it.
__device__ __forceinline__ uint32_t encode_int4(const uint4& w, uint32_t& sbits, bool& bad) {
  const uint32_t top = lane_max<4>(amax_bits(w));
  bad = top >= kInfBits;
  const __nv_bfloat16 sb = __float2bfloat16_rn(__fdiv_rn(__uint_as_float(top << 16), 7.f));
  sbits = bad ? 0x7fc0u : (uint32_t)__bfloat16_as_ushort(sb);
  const float s = __bfloat162float(sb);
  if (bad || s == 0.f) return 0x88888888u;
  uint32_t out = 0;
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
  for (int i = 0; i < 8; ++i) {
    const float x = (i & 1) ? bf16hi(ws[i >> 1]) : bf16lo(ws[i >> 1]);
    const int n = max(-7, min(7, __float2int_rn(__fdiv_rn(x, s))));
    out |= (uint32_t)(n + 8) << (4 * i);
  }
  return out;
}

__device__ __forceinline__ uint32_t pack2(float a, float b) {
  __nv_bfloat162 v = __floats2bfloat162_rn(a, b);
  return *(uint32_t*)&v;
}
__device__ __forceinline__ uint32_t decode_e4m3x2(uint32_t two, float s) {
  const __half2_raw h = __nv_cvt_fp8x2_to_halfraw2((__nv_fp8x2_storage_t)(two & 0xffffu), __NV_E4M3);
  const float2 f = __half22float2(*(const __half2*)&h);
  return pack2(f.x * s, f.y * s);
}

// FMT: thinK_page_format.  E: bytes of an element (2 bf16, 4 fp32).
template <int D, int E, int FMT, bool WRITE>
__global__ void __launch_bounds__(kRowThreads) k_paged_rows(const PagedRowsParams p) {
  constexpr int LANES = D * E / 16;             // lanes of a row, 16 bytes of elements each
  constexpr int CH = 16 / E;                    // channels of a lane
  const int b = blockIdx.y;
  const int nrows_raw = p.rows ? __ldg(p.rows + b) : p.max_rows;
  const int nrows = min(nrows_raw, p.max_rows);
  if (blockIdx.x == 0 && threadIdx.x == 0 && nrows_raw > p.max_rows) atomicOr(p.error, kErrPage);
  if (nrows <= 0) return;
  const uint32_t r = blockIdx.x * (kRowThreads / LANES) + threadIdx.x / LANES;     // row of the entry, head fastest
  const uint32_t rl = p.by_heads.div(r), h = r - rl * p.g.N_kv;
  const uint32_t s = p.by_layers.div(rl), ll = rl - s * p.nlayers;
  if (blockIdx.x * (kRowThreads / LANES) >= (uint64_t)nrows * p.nlayers * p.g.N_kv) return;   // whole block: no row
  const bool on = s < (uint32_t)nrows;          // lanes of a row agree; idle rows still take part in the shuffles
  const int c = threadIdx.x % LANES;
  const int64_t tok = (int64_t)(p.pos ? __ldg(p.pos + b) : 0) + s;
  const int64_t ek = b * p.k.sb + (int64_t)s * p.k.ss + ll * p.k.sl + h * p.k.sn + c * CH;
  const int64_t ev = b * p.v.sb + (int64_t)s * p.v.ss + ll * p.v.sl + h * p.v.sn + c * CH;
  uint4* const kx = (uint4*)((uint8_t*)p.k.ptr + ek * E);
  uint4* const vx = (uint4*)((uint8_t*)p.v.ptr + ev * E);
  uint4 k = make_uint4(0u, 0u, 0u, 0u), v = k;
  if (WRITE && on) {
    k = __ldcs(kx);
    v = __ldcs(vx);
  }
  const int page = on ? page_of(p.table, p.g, b, tok, p.error) : -1;
  const bool ok = page >= 0;
  const int slot = (int)(tok & (kPageTokens - 1));
  uint8_t* const block = p.pages + page_block_offset(p.g, p.layer0 + (int)ll, ok ? page : 0, (int)h);
  uint8_t* const kc = block + slot * p.g.row_bytes;
  uint8_t* const vc = kc + kPageTokens * p.g.row_bytes;
  uint8_t* const ks = block + 2 * kPageTokens * p.g.row_bytes + slot * p.g.scale_bytes;
  uint8_t* const vs = ks + kPageTokens * p.g.scale_bytes;
  if (WRITE) {
    if (FMT == THINK_PAGE_PLAIN) {
      if (ok) {
        ((uint4*)kc)[c] = k;
        ((uint4*)vc)[c] = v;
      }
    } else if (FMT == THINK_PAGE_E4M3) {
      uint32_t ke, ve;
      bool kbad, vbad;
      const uint2 k8 = encode_e4m3<LANES>(k, ke, kbad), v8 = encode_e4m3<LANES>(v, ve, vbad);
      if (ok) {
        ((uint2*)kc)[c] = k8;
        ((uint2*)vc)[c] = v8;
        if (c == 0) {
          *ks = (uint8_t)ke;
          *vs = (uint8_t)ve;
          if (kbad || vbad) atomicOr(p.error, kErrNonFinite);
        }
      }
    } else {
      uint32_t ke, ve;
      bool kbad, vbad;
      const uint32_t k4 = encode_int4(k, ke, kbad), v4 = encode_int4(v, ve, vbad);
      if (ok) {
        ((uint32_t*)kc)[c] = k4;
        ((uint32_t*)vc)[c] = v4;
        if ((c & 3) == 0) {
          ((uint16_t*)ks)[c >> 2] = (uint16_t)ke;
          ((uint16_t*)vs)[c >> 2] = (uint16_t)ve;
          if (kbad || vbad) atomicOr(p.error, kErrNonFinite);
        }
      }
    }
  } else if (ok) {
    if (FMT == THINK_PAGE_PLAIN) {
      k = __ldcs((const uint4*)kc + c);
      v = __ldcs((const uint4*)vc + c);
    } else if (FMT == THINK_PAGE_E4M3) {
      const uint2 k8 = __ldcs((const uint2*)kc + c), v8 = __ldcs((const uint2*)vc + c);
      const float fk = e8m0(*ks), fv = e8m0(*vs);
      k = make_uint4(decode_e4m3x2(k8.x, fk), decode_e4m3x2(k8.x >> 16, fk), decode_e4m3x2(k8.y, fk), decode_e4m3x2(k8.y >> 16, fk));
      v = make_uint4(decode_e4m3x2(v8.x, fv), decode_e4m3x2(v8.x >> 16, fv), decode_e4m3x2(v8.y, fv), decode_e4m3x2(v8.y >> 16, fv));
    } else {
      const uint32_t k4 = __ldcs((const uint32_t*)kc + c), v4 = __ldcs((const uint32_t*)vc + c);
      const float fk = __uint_as_float((uint32_t)((const uint16_t*)ks)[c >> 2] << 16);
      const float fv = __uint_as_float((uint32_t)((const uint16_t*)vs)[c >> 2] << 16);
      auto two = [](uint32_t w, int i, float f) {
        return pack2((float)((int)(w >> (8 * i) & 15u) - 8) * f, (float)((int)(w >> (8 * i + 4) & 15u) - 8) * f);
      };
      k = make_uint4(two(k4, 0, fk), two(k4, 1, fk), two(k4, 2, fk), two(k4, 3, fk));
      v = make_uint4(two(v4, 0, fv), two(v4, 1, fv), two(v4, 2, fv), two(v4, 3, fv));
    }
    __stcs(kx, k);
    __stcs(vx, v);
  }
}

template <int D, int E, int FMT>
cudaError_t launch_rows(const PagedRowsParams& p, bool write, cudaStream_t s) {
  constexpr int rpb = kRowThreads / (D * E / 16);
  const int64_t rows = (int64_t)p.max_rows * p.nlayers * p.g.N_kv;
  const dim3 grid((unsigned)((rows + rpb - 1) / rpb), (unsigned)p.table.B);
  if (write) k_paged_rows<D, E, FMT, true><<<grid, kRowThreads, 0, s>>>(p);
  else k_paged_rows<D, E, FMT, false><<<grid, kRowThreads, 0, s>>>(p);
  return cudaGetLastError();
}

template <int D>
cudaError_t launch_rows_d(const PagedRowsParams& p, int dtype, int format, bool write, cudaStream_t s) {
  if (dtype == THINK_F32) return launch_rows<D, 4, THINK_PAGE_PLAIN>(p, write, s);
  switch (format) {
    case THINK_PAGE_PLAIN: return launch_rows<D, 2, THINK_PAGE_PLAIN>(p, write, s);
    case THINK_PAGE_E4M3: return launch_rows<D, 2, THINK_PAGE_E4M3>(p, write, s);
    case THINK_PAGE_INT4: return launch_rows<D, 2, THINK_PAGE_INT4>(p, write, s);
  }
  return cudaErrorInvalidValue;
}

}  // namespace

cudaError_t launch_paged_rows(const PagedRowsParams& p, int dtype, int format, bool write, cudaStream_t s) {
  if (p.g.D == 128) return launch_rows_d<128>(p, dtype, format, write, s);
  if (p.g.D == 64) return launch_rows_d<64>(p, dtype, format, write, s);
  return cudaErrorInvalidValue;
}

}  // namespace think
