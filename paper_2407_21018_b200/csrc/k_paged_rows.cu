// Rows of the paged cache: quantised as they are written, dequantised as they are read back.
//
// Both directions only move bytes (512 bytes of bf16 key and value against 258 or 144 stored ones a row at
// D = 128), so the DRAM stream is the bound and the kernels are one pass: a lane owns two 16-byte pieces of a row's
// elements (8 bf16 or 4 fp32 channels each) of the key AND of the value, all four loads in flight before
// anything waits (one piece a lane spent most of its instructions on addresses), the row's (or
// group's) maximum goes over the lanes of the row by shuffles, and codes leave from registers.  The lanes of a warp
// hold consecutive rows with the head running fastest, which is the order of the [b, s, l, n, d] tensors: loads are
// whole 128-byte lines, and the stores of a row are one contiguous piece of its page.
#include <cuda_fp8.h>

#include "paged_internal.h"

namespace think {
namespace {

constexpr int kRowThreads = 128;
constexpr int kPieces = 2;            // 16-byte pieces of a row that a lane holds, half a row apart

// largest |x| of 8 bf16, a NaN if there is one, as the integer of its bits: orders finite < infinite < NaN
__device__ __forceinline__ uint32_t amax_bits(const uint4& w) {
  auto mag = [](uint32_t x) { return __habs2(*(const __nv_bfloat162*)&x); };
  const __nv_bfloat162 t = __hmax2_nan(__hmax2_nan(mag(w.x), mag(w.y)), __hmax2_nan(mag(w.z), mag(w.w)));
  const uint32_t m = *(const uint32_t*)&t;
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

// A row's scale byte from its largest magnitude's bits; the factor 2^-k that brings it to codes.
// top = 1.m * 2^(E - 127): 448 = 1.75 * 2^8, so the scale's exponent k is E - 8, one more if 1.m > 1.75
__device__ __forceinline__ uint32_t scale_e4m3(uint32_t top, float& inv) {
  const int k = max((int)(top >> 7) - 127 - 8 + ((top & 0x7fu) > 0x60u ? 1 : 0), -126);
  inv = __uint_as_float((uint32_t)(127 - k) << 23);
  return (uint32_t)(k + 127);
}
// 8 bf16 -> 8 e4m3 codes: the products are exact, the codes round once
__device__ __forceinline__ uint2 encode_e4m3(const uint4& w, float inv) {
  return make_uint2(e4m3x4(bf16lo(w.x) * inv, bf16hi(w.x) * inv, bf16lo(w.y) * inv, bf16hi(w.y) * inv),
                    e4m3x4(bf16lo(w.z) * inv, bf16hi(w.z) * inv, bf16lo(w.w) * inv, bf16hi(w.w) * inv));
}

// 8 bf16 -> 8 4-bit codes; 4 lanes hold the group of 32 channels.  `sbits` receives the bf16 scale.
// x / s to the nearest integer, ties to even, without eight divisions: x and s have 8 significant bits, so a quotient
// that is no tie is at least 1 / 510 away from one.  x * (1 / s) is off by less than 2^-20; adding 1.5 * 2^11 rounds it
// to multiples of 2^-12, which makes ties exact again and moves nothing else across one.  A second addition makes that
// offset 1.5 * 2^23 + 8 and rounds to integers: n + 8 is in the low bits.  A scale below 2^-126 takes the division:
// its own rounding error is large there, and n needs its limits.
__device__ __forceinline__ uint32_t encode_int4(const uint4& w, uint32_t& sbits, bool& bad) {
  const uint32_t top = lane_max<4>(amax_bits(w));
  bad = top >= kInfBits;
  // amax / 7 to bf16: the quotient of an 8-bit number by 7 is never a tie and at least 2^-12 away from one, so the
  // product with 1 / 7 rounds the same
  const __nv_bfloat16 sb = __float2bfloat16_rn(__fmul_rn(__uint_as_float(top << 16), 1.f / 7.f));
  sbits = bad ? 0x7fc0u : (uint32_t)__bfloat16_as_ushort(sb);
  const float s = __bfloat162float(sb);
  if (bad || s == 0.f) return 0x88888888u;
  const uint32_t ws[4] = {w.x, w.y, w.z, w.w};
  uint32_t c[4];                                // two codes each in the low byte
  if (s >= 1.17549435e-38f) {
    float inv;                                  // within an ulp
    asm("rcp.approx.f32 %0, %1;" : "=f"(inv) : "f"(s));
    constexpr float kTo12 = 1.5f * 2048.f, kToInt = 12582920.f - kTo12;
    const f32x2 inv2 = two(inv, inv), to12 = two(kTo12, kTo12), to_int = two(kToInt, kToInt);
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      float a, b;
      split(add2(fma2(two(bf16lo(ws[i]), bf16hi(ws[i])), inv2, to12), to_int), a, b);
      c[i] = __float_as_uint(a) + (__float_as_uint(b) << 4);
    }
  } else {
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const int a = max(-7, min(7, __float2int_rn(__fdiv_rn(bf16lo(ws[i]), s))));
      const int b = max(-7, min(7, __float2int_rn(__fdiv_rn(bf16hi(ws[i]), s))));
      c[i] = (uint32_t)(a + 8) | (uint32_t)(b + 8) << 4;
    }
  }
  return __byte_perm(__byte_perm(c[0], c[1], 0x0040), __byte_perm(c[2], c[3], 0x0040), 0x5410);
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

// 8 4-bit codes times their scale to bf16: a code as the low byte of 2^23 + code, less 2^23 + 8
__device__ __forceinline__ uint4 decode_int4(uint32_t w, float f) {
  const uint32_t even = w & 0x0f0f0f0fu, odd = (w >> 4) & 0x0f0f0f0fu;
  const f32x2 f2 = two(f, f), off = two(-8388616.f, -8388616.f);
  uint32_t r[4];
#pragma unroll
  for (int i = 0; i < 4; ++i) {
    float a = __uint_as_float(__byte_perm(even, 0x4b000000u, 0x7440 | i)), b = __uint_as_float(__byte_perm(odd, 0x4b000000u, 0x7440 | i));
    split(mul2(add2(two(a, b), off), f2), a, b);
    r[i] = pack2(a, b);
  }
  return make_uint4(r[0], r[1], r[2], r[3]);
}
__device__ __forceinline__ uint4 decode_e4m3(const uint2& w, float f) {
  return make_uint4(decode_e4m3x2(w.x, f), decode_e4m3x2(w.x >> 16, f), decode_e4m3x2(w.y, f), decode_e4m3x2(w.y >> 16, f));
}

// FMT: thinK_page_format.  E: bytes of an element (2 bf16, 4 fp32).  A block takes kRowThreads / LANES consecutive
// rows of one entry (head fastest, then layer, then token).  SLOTS: a row's place is given, not looked up.  14 blocks an SM: the 4-bit kernels would take 40 registers
// and 12 blocks (3 prompts written and read back, replayed: 80.3 us, 79.2 so, although the 4-bit writer then keeps 28
// bytes a thread, 32 at D = 64, in local memory).
template <int D, int E, int FMT, bool WRITE, bool SLOTS = false>
__global__ void __launch_bounds__(kRowThreads, 14) k_paged_rows(PagedRowsParams p) {
  constexpr int P = kPieces;
  constexpr int LANES = D * E / 16 / P;         // lanes of a row
  constexpr int RPB = kRowThreads / LANES;
  constexpr int RB = FMT == THINK_PAGE_PLAIN ? D * E : FMT == THINK_PAGE_E4M3 ? D : D / 2;
  constexpr int SB = FMT == THINK_PAGE_PLAIN ? 0 : FMT == THINK_PAGE_E4M3 ? 1 : D / 16;
  begin_dependent();
  const int b = blockIdx.y;
  const int nrows_raw = p.rows ? load_now(p.rows + b) : p.max_rows;
  const int pos = p.pos ? load_now(p.pos + b) : 0;
  const int nrows = min(nrows_raw, p.max_rows);
  if (blockIdx.x == 0 && threadIdx.x == 0 && nrows_raw > p.max_rows) atomicOr(p.error, kErrPage);
  const uint32_t first = blockIdx.x * RPB;
  if (nrows <= 0 || first >= (uint64_t)nrows * p.nlayers * p.g.N_kv) return;      // whole block: no row
  const int c = threadIdx.x % LANES;
  const uint8_t* const kb = (const uint8_t*)p.k.ptr + (b * p.k.sb) * E + c * 16;
  const uint8_t* const vb = (const uint8_t*)p.v.ptr + (b * p.v.sb) * E + c * 16;
  const uint32_t r = first + threadIdx.x / LANES;
  const uint32_t rl = p.by_heads.div(r), h = r - rl * p.g.N_kv;
  const uint32_t s = p.by_layers.div(rl), ll = rl - s * p.nlayers;
  bool on = s < (uint32_t)nrows;                // lanes of a row agree; idle rows still take part in the shuffles
  uint4* const kx = (uint4*)(kb + (s * p.k.ss + ll * p.k.sl + h * p.k.sn) * E);
  uint4* const vx = (uint4*)(vb + (s * p.v.ss + ll * p.v.sl + h * p.v.sn) * E);
  uint4 k[P], v[P];
#pragma unroll
  for (int i = 0; i < P; ++i) {
    k[i] = v[i] = make_uint4(0u, 0u, 0u, 0u);
    if (WRITE && on) {
      k[i] = __ldcs(kx + i * LANES);
      v[i] = __ldcs(vx + i * LANES);
    }
  }
  int64_t tok = (int64_t)pos + s;
  int page;
  if constexpr (SLOTS) {
    tok = on ? load_now(p.slots + s) : -1;      // a negative one: the row goes nowhere
    page = (int)(tok >> 6);
    if (page >= p.g.num_pages) {
      atomicOr(p.error, kErrPage);
      page = -1;
    }
  } else {
    page = on ? page_of(p.table, p.g, b, tok, p.error) : -1;
  }
  on = page >= 0;
  const int slot = (int)(tok & (kPageTokens - 1));
  uint8_t* const block = p.pages + page_block_offset(p.g, p.layer0 + (int)ll, on ? page : 0, (int)h);
  uint8_t* const kc = block + slot * RB;        // values: 64 rows behind
  uint8_t* const ks = block + 2 * kPageTokens * RB + slot * SB;
  if (WRITE) {
    uint8_t* const vc = kc + kPageTokens * RB;
    uint8_t* const vs = ks + kPageTokens * SB;
    if (FMT == THINK_PAGE_PLAIN) {
      if (on) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
          ((uint4*)kc)[c + i * LANES] = k[i];
          ((uint4*)vc)[c + i * LANES] = v[i];
        }
      }
    } else if (FMT == THINK_PAGE_E4M3) {
      uint32_t kt = 0, vt = 0;
#pragma unroll
      for (int i = 0; i < P; ++i) {
        kt = max(kt, amax_bits(k[i]));
        vt = max(vt, amax_bits(v[i]));
      }
      kt = lane_max<LANES>(kt);
      vt = lane_max<LANES>(vt);
      float ki, vi;
      const uint32_t ke = scale_e4m3(kt, ki), ve = scale_e4m3(vt, vi);
      const bool kbad = kt >= kInfBits, vbad = vt >= kInfBits;
      const uint2 nan = make_uint2(0x7f7f7f7fu, 0x7f7f7f7fu);
      if (on) {
#pragma unroll
        for (int i = 0; i < P; ++i) {
          const uint2 k8 = encode_e4m3(k[i], ki), v8 = encode_e4m3(v[i], vi);
          ((uint2*)kc)[c + i * LANES] = kbad ? nan : k8;
          ((uint2*)vc)[c + i * LANES] = vbad ? nan : v8;
        }
        if (c == 0) {
          *ks = (uint8_t)(kbad ? 127u : ke);
          *vs = (uint8_t)(vbad ? 127u : ve);
          if (kbad || vbad) atomicOr(p.error, kErrNonFinite);
        }
      }
    } else {
#pragma unroll
      for (int i = 0; i < P; ++i) {
        uint32_t ke, ve;
        bool kbad, vbad;
        const uint32_t k4 = encode_int4(k[i], ke, kbad), v4 = encode_int4(v[i], ve, vbad);
        if (on) {
          ((uint32_t*)kc)[c + i * LANES] = k4;
          ((uint32_t*)vc)[c + i * LANES] = v4;
          if ((c & 3) == 0) {
            ((uint16_t*)ks)[(c + i * LANES) >> 2] = (uint16_t)ke;
            ((uint16_t*)vs)[(c + i * LANES) >> 2] = (uint16_t)ve;
            if (kbad || vbad) atomicOr(p.error, kErrNonFinite);
          }
        }
      }
    }
    return;
  }
  if (!on) return;
  uint32_t ke[P], ve[P];                        // scales' bits
  const uint8_t* const vc = kc + kPageTokens * RB;
  const uint8_t* const vs = ks + kPageTokens * SB;
#pragma unroll
  for (int i = 0; i < P; ++i) {
    const int ci = c + i * LANES;
    if (FMT == THINK_PAGE_PLAIN) {
      k[i] = __ldcs((const uint4*)kc + ci);
      v[i] = __ldcs((const uint4*)vc + ci);
    } else if (FMT == THINK_PAGE_E4M3) {
      *(uint2*)&k[i] = __ldcs((const uint2*)kc + ci);
      *(uint2*)&v[i] = __ldcs((const uint2*)vc + ci);
      ke[i] = i == 0 ? *ks : ke[0];
      ve[i] = i == 0 ? *vs : ve[0];
    } else {
      k[i].x = __ldcs((const uint32_t*)kc + ci);
      v[i].x = __ldcs((const uint32_t*)vc + ci);
      ke[i] = ((const uint16_t*)ks)[ci >> 2];
      ve[i] = ((const uint16_t*)vs)[ci >> 2];
    }
  }
#pragma unroll
  for (int i = 0; i < P; ++i) {
    if (FMT == THINK_PAGE_E4M3) {
      k[i] = decode_e4m3(make_uint2(k[i].x, k[i].y), e8m0(ke[i]));
      v[i] = decode_e4m3(make_uint2(v[i].x, v[i].y), e8m0(ve[i]));
    } else if (FMT == THINK_PAGE_INT4) {
      k[i] = decode_int4(k[i].x, __uint_as_float(ke[i] << 16));
      v[i] = decode_int4(v[i].x, __uint_as_float(ve[i] << 16));
    }
    __stcs(kx + i * LANES, k[i]);
    __stcs(vx + i * LANES, v[i]);
  }
}

template <int D, int E, int FMT>
cudaError_t launch_rows(const PagedRowsParams& p, bool write, cudaStream_t s) {
  constexpr int rpb = kRowThreads / (D * E / 16 / kPieces);
  const int64_t rows = (int64_t)p.max_rows * p.nlayers * p.g.N_kv;
  const dim3 grid((unsigned)((rows + rpb - 1) / rpb), (unsigned)p.table.B);
  if (p.slots) return launch_dependent(k_paged_rows<D, E, FMT, true, true>, grid, kRowThreads, 0, s, p);
  return launch_dependent(write ? k_paged_rows<D, E, FMT, true> : k_paged_rows<D, E, FMT, false>, grid, kRowThreads, 0, s, p);
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
