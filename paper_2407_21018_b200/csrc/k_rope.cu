// Rotary positions (host side and kernel).
//
//   (x_a, x_b) -> m (x_a cos t - x_b sin t, x_b cos t + x_a sin t),  t = position * frequency(j)
// for the R / 2 pairs of a row's first R channels; the transposed form turns by -t with the same factor m.
//
// Angles.  A position may be 2^31 and a frequency 1, so their product in fp32 would be off by whole turns.  Frequencies are
// kept as turns per token in 64-bit fixed point, 2^-64 of a turn a unit: the product modulo one turn is the low half of an
// integer product, exact but for the frequency's own rounding to an even unit (2^-64 * 2^31 = 2^-33 turns).  Its upper 32 bits are brought to the
// nearest quarter turn, which leaves at most an eighth to sine and cosine in fp32, with an angle error of 2^-27 turns.
// Bound: DRAM, each row read and written once: 8192 tokens of 40 heads of 128 in 31.6 us, 168 MB at 0.81 of the copy rate; heads of
// 64 with half their channels turned 0.83; small calls 2.7 us of launch, 10 with the host's part.  Sine and cosine are computed once
// a token and pair, into shared memory, for all heads and layers of queries and keys; a lane then turns 16-byte pieces (with their
// partners half a rotation away).  Two pieces with their partners a lane under way (56 registers) took 37 us, more tokens a block
// 35; interleaved pairs with one piece a lane 48 instead of 38 (heads of 64); pairs one by one where half a rotation is no whole piece 179
// instead of 51 (20 of 128 channels; what is left there is accesses of 4 bytes, of 2 where half a rotation is odd: 22 of 128, 62 us).
#include <math.h>
#include <string.h>

#include <new>

#include <nvtx3/nvToolsExt.h>

#include "paged_internal.h"
#include "paged_views.h"

namespace think {
namespace {

constexpr int kRopeThreads = 256;
constexpr int kRopeMaxD = 256;
constexpr int kRopeTable = 2048;        // (cos, sin) pairs a block holds

struct RopeSide {                       // queries or keys
  const uint8_t* x;
  uint8_t* y;
  int64_t xb, xs, xl, xn, yb, ys, yl, yn;   // strides in bytes
};
struct RopeParams {
  RopeSide side[2];
  int heads_q, heads;                   // heads of queries, of both, a layer
  int nlayers, S, R, D, pairs, table;   // pairs: R / 2; table: room for a token's, those of whole pieces
  int tokens, blocks_s;                 // tokens of a block, blocks of an entry
  int units, items;                     // units of a row, of a token (all layers and heads)
  int second;                           // 0, or pieces of a row that a unit's second is behind its first
  float m, sign;
  const int32_t* pos;
  int64_t pos_stride;                   // 0: position pos[b] + s
  const int32_t* rows;
  FastDiv by_items, by_units, by_heads, by_pairs, by_blocks;
  uint64_t turns[kRopeMaxD / 2];
};

__device__ __forceinline__ void turn(float a, float b, float c, float s, float& u, float& v) {
  const float x = fmaf(a, c, -(b * s));
  v = fmaf(b, c, a * s);
  u = x;
}

// 16 bytes of bf16 or fp32 as floats and back
template <int E>
__device__ __forceinline__ void open16(const uint4& w, float (&f)[16 / E]) {
  if constexpr (E == 2) {
    const uint32_t u[4] = {w.x, w.y, w.z, w.w};
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      f[2 * i] = bf16lo(u[i]);
      f[2 * i + 1] = bf16hi(u[i]);
    }
  } else {
    f[0] = __uint_as_float(w.x); f[1] = __uint_as_float(w.y); f[2] = __uint_as_float(w.z); f[3] = __uint_as_float(w.w);
  }
}
template <int E>
__device__ __forceinline__ uint4 close16(const float (&f)[16 / E]) {
  if constexpr (E == 2) {
    uint32_t u[4];
#pragma unroll
    for (int i = 0; i < 4; ++i) {
      const __nv_bfloat162 h = __floats2bfloat162_rn(f[2 * i], f[2 * i + 1]);
      u[i] = *(const uint32_t*)&h;
    }
    return make_uint4(u[0], u[1], u[2], u[3]);
  } else {
    return make_uint4(__float_as_uint(f[0]), __float_as_uint(f[1]), __float_as_uint(f[2]), __float_as_uint(f[3]));
  }
}

// What a unit is: a piece of 16 bytes and its partner half a rotation on; a piece and, where their number is even, the one half
// the pieces on (interleaved pairs lie within pieces); two or one channels and their partners, where half a rotation is no
// multiple of a piece (two channels where it is even).  Behind the units that turn are those that copy, by pieces.
enum RopeForm { kHalves, kPairs, kTwo, kOne };
template <int E, int FORM>
__global__ void __launch_bounds__(kRopeThreads) k_rope(const __grid_constant__ RopeParams p) {
  constexpr int V = 16 / E, kShift = FORM == kHalves ? (E == 2 ? 3 : 2) : FORM == kPairs ? (E == 2 ? 2 : 1) : 0, W = 1 << kShift;      // W: pairs of a piece
  __shared__ __align__(16) float2 s_cs[kRopeTable];
  __shared__ int s_on[64];
  begin_dependent();
  const int b = p.by_blocks.div(blockIdx.x), s0 = (blockIdx.x - b * p.blocks_s) * p.tokens;
  const int rows = p.rows ? min(load_now(p.rows + b), p.S) : p.S;
  const int n = min(p.tokens, rows - s0);
  if (n <= 0) return;                   // whole block
  const int across = p.table >> kShift;
  for (int i = threadIdx.x; i < n * p.pairs; i += kRopeThreads) {
    const int t = p.by_pairs.div(i), j = i - t * p.pairs;
    const int32_t pos = p.pos_stride ? load_now(p.pos + b * p.pos_stride + s0 + t)
                                     : (int32_t)((uint32_t)load_now(p.pos + b) + (uint32_t)(s0 + t));   // past 2^31: negative
    if (j == 0) s_on[t] = pos >= 0;
    const uint64_t f = p.turns[j];
    const uint32_t u = (uint32_t)pos * (uint32_t)(f >> 32) + __umulhi((uint32_t)pos, (uint32_t)f);    // 2^-32 turns
    const uint32_t quarter = (u + 0x20000000u) >> 30;
    const float r = (float)(int32_t)(u - (quarter << 30)) * 4.656612873077392578e-10f;                 // half turns
    float sn, cn;
    sincospif(r, &sn, &cn);
    const float c = quarter & 1 ? sn : cn, s = quarter & 1 ? cn : sn;     // signs: cos - + by quarters 1, 2; sin by 2, 3
    // two pairs of a piece, then the same two of the next: lanes with neighbouring pieces read neighbouring 16 bytes
    const int at = t * p.table + (W > 1 ? (j & (W - 2)) * across + 2 * (j >> kShift) + (j & 1) : j);
    s_cs[at] = make_float2((quarter + 1) & 2 ? -c * p.m : c * p.m, (quarter & 2 ? -s : s) * p.m * p.sign);
  }
  __syncthreads();
  for (int i = threadIdx.x; i < n * p.items; i += kRopeThreads) {
    const int t = p.by_items.div(i), item = i - t * p.items;
    if (!s_on[t]) continue;             // no position: the row stays
    const int lh = p.by_units.div(item), unit = item - lh * p.units;
    const int l = p.by_heads.div(lh), h0 = lh - l * p.heads;
    const bool key = h0 >= p.heads_q;
    const RopeSide& side = p.side[key];
    const int h = key ? h0 - p.heads_q : h0;
    const uint8_t* const x = side.x + b * side.xb + (s0 + t) * side.xs + l * side.xl + h * side.xn;
    uint8_t* const y = side.y + b * side.yb + (s0 + t) * side.ys + l * side.yl + h * side.yn;
    const float2* const cs = s_cs + t * p.table;
    if constexpr (FORM == kPairs) {
      auto turned = [&](const uint4& w, int piece) {
        if (piece * V >= p.R) return w;
        float f[V];
        open16<E>(w, f);
#pragma unroll
        for (int k = 0; k < V; k += 4) {
          const float4 c = *(const float4*)(cs + k / 2 * across + 2 * piece);
          if (piece * V + k < p.R) turn(f[k], f[k + 1], c.x, c.y, f[k], f[k + 1]);
          if (piece * V + k + 2 < p.R) turn(f[k + 2], f[k + 3], c.z, c.w, f[k + 2], f[k + 3]);
        }
        return close16<E>(f);
      };
      const uint4 wa = __ldcs((const uint4*)x + unit);
      if (p.second) {
        const uint4 wb = __ldcs((const uint4*)x + unit + p.second);
        __stcs((uint4*)y + unit + p.second, turned(wb, unit + p.second));
      }
      __stcs((uint4*)y + unit, turned(wa, unit));
    } else if constexpr (FORM == kHalves) {
      const int half = p.pairs / V;
      if (unit < half) {
        const uint4 wa = __ldcs((const uint4*)x + unit), wb = __ldcs((const uint4*)x + unit + half);
        float a[V], c[V];
        open16<E>(wa, a);
        open16<E>(wb, c);
#pragma unroll
        for (int k = 0; k < V; k += 2) {
          const float4 f = *(const float4*)(cs + k * across + 2 * unit);
          turn(a[k], c[k], f.x, f.y, a[k], c[k]);
          turn(a[k + 1], c[k + 1], f.z, f.w, a[k + 1], c[k + 1]);
        }
        __stcs((uint4*)y + unit, close16<E>(a));
        __stcs((uint4*)y + unit + half, close16<E>(c));
      } else {
        __stcs((uint4*)y + unit + half, __ldcs((const uint4*)x + unit + half));
      }
    } else {
      using T = typename std::conditional<E == 2, __nv_bfloat16, float>::type;
      struct alignas(sizeof(T) * (FORM == kTwo ? 2 : 1)) Some { T v[FORM == kTwo ? 2 : 1]; };
      constexpr int N = FORM == kTwo ? 2 : 1;
      const Some* const xe = (const Some*)x;
      Some* const ye = (Some*)y;
      const int turning = p.pairs / N, border = (p.R + V - 1) / V * V;
      if (unit < turning) {
        Some a = xe[unit], c = xe[unit + turning];
#pragma unroll
        for (int k = 0; k < N; ++k) {
          float u, v;
          turn((float)a.v[k], (float)c.v[k], cs[N * unit + k].x, cs[N * unit + k].y, u, v);
          a.v[k] = (T)u;
          c.v[k] = (T)v;
        }
        ye[unit] = a;
        ye[unit + turning] = c;
      } else {
        const int c = unit + turning, piece = border / V + c - border / N;
        if (c < border / N) ye[c] = xe[c];
        else __stcs((uint4*)y + piece, __ldcs((const uint4*)x + piece));
      }
    }
  }
}

struct Range {
  explicit Range(const char* name) { nvtxRangePushA(name); }
  ~Range() { nvtxRangePop(); }
};

}  // namespace
}  // namespace think

using namespace think;

struct thinK_rope {
  int D, R, layout, elem;
  float m;
  double radians[kRopeMaxD / 2];
  uint64_t turns[kRopeMaxD / 2];
};

namespace {

thinK_status rope_frequencies(const thinK_rope_config* c, thinK_rope* o) {
  if (!c) return THINK_ERR_INVALID_ARG;
  if (c->dtype != THINK_BF16 && c->dtype != THINK_F32) return THINK_ERR_UNSUPPORTED;
  o->elem = c->dtype == THINK_BF16 ? 2 : 4;
  if (c->D < 2 || c->rot_dim < 2 || c->rot_dim > c->D || c->rot_dim % 2 != 0) return THINK_ERR_INVALID_ARG;
  if (c->D > kRopeMaxD || c->D * o->elem % 16 != 0) return THINK_ERR_UNSUPPORTED;
  if (c->layout != THINK_ROPE_HALVES && c->layout != THINK_ROPE_PAIRS) return THINK_ERR_INVALID_ARG;
  if (c->scaling < THINK_ROPE_PLAIN || c->scaling > THINK_ROPE_BANDS) return THINK_ERR_INVALID_ARG;
  if (!(c->theta >= 1.0 && c->theta <= 1e30)) return THINK_ERR_INVALID_ARG;
  const bool scaled = c->scaling != THINK_ROPE_PLAIN, trained = c->scaling == THINK_ROPE_YARN || c->scaling == THINK_ROPE_BANDS;
  if (scaled && !(c->factor >= 1.0 && c->factor <= 1e6)) return THINK_ERR_INVALID_ARG;
  if (!(c->attention_factor >= 0.0 && c->attention_factor <= 1e6)) return THINK_ERR_INVALID_ARG;
  double slow = c->slow == 0.0 ? 1.0 : c->slow, fast = c->fast == 0.0 ? (c->scaling == THINK_ROPE_YARN ? 32.0 : 4.0) : c->fast;
  if (trained && (!(c->trained >= 1.0 && c->trained <= 1e12) || !(slow > 0.0 && slow < fast && fast <= 1e12))) return THINK_ERR_INVALID_ARG;
  if (c->scaling == THINK_ROPE_NTK && c->rot_dim < 4) return THINK_ERR_INVALID_ARG;
  if (c->scaling == THINK_ROPE_YARN && !(c->theta > 1.0)) return THINK_ERR_INVALID_ARG;      // divides by its logarithm
  constexpr long double kTwoPi = 6.283185307179586476925286766559L;
  const int R = c->rot_dim;
  o->D = c->D; o->R = R; o->layout = c->layout;
  long double m = c->attention_factor;
  if (m == 0) m = c->scaling == THINK_ROPE_YARN ? 0.1L * logl(c->factor) + 1 : 1;
  o->m = (float)m;
  long double theta = c->theta;
  if (c->scaling == THINK_ROPE_NTK) theta *= powl(c->factor, (long double)R / (R - 2));
  long double low = 0, high = 0;
  if (c->scaling == THINK_ROPE_YARN) {
    // the pair that makes so many turns over the trained context
    auto where = [&](double turns) { return R * logl(c->trained / (turns * kTwoPi)) / (2 * logl(theta)); };
    low = fmaxl(floorl(where(fast)), 0);
    high = fminl(ceill(where(slow)), R - 1);
  }
  for (int j = 0; j < R / 2; ++j) {
    long double f = powl(theta, -2.0L * j / R);
    if (c->scaling == THINK_ROPE_LINEAR) {
      f /= c->factor;
    } else if (c->scaling == THINK_ROPE_YARN) {
      const long double ramp = fminl(1, fmaxl(0, (j - low) / fmaxl(high - low, 0.001L)));
      f = f / c->factor * ramp + f * (1 - ramp);
    } else if (c->scaling == THINK_ROPE_BANDS) {
      const long double keep = fminl(1, fmaxl(0, (c->trained * f / kTwoPi - slow) / ((long double)fast - slow)));
      f = f / c->factor * (1 - keep) + f * keep;
    }
    o->radians[j] = (double)f;
    o->turns[j] = (uint64_t)llroundl(f / kTwoPi * 9223372036854775808.0L) << 1;       // f <= 1: below a sixth of a turn
  }
  return THINK_OK;
}

bool side_ok(const thinK_tensor5& t, int elem) {
  if (!t.ptr || ((uintptr_t)t.ptr & 15)) return false;
  const int64_t s[4] = {t.stride_b, t.stride_s, t.stride_l, t.stride_n};
  for (int i = 0; i < 4; ++i)
    if (s[i] < 0 || s[i] % (16 / elem) != 0) return false;
  return true;
}
bool same(const thinK_tensor5& a, const thinK_tensor5& b) {
  return a.ptr == b.ptr && a.stride_b == b.stride_b && a.stride_s == b.stride_s && a.stride_l == b.stride_l && a.stride_n == b.stride_n;
}

}  // namespace

extern "C" {

thinK_status thinK_rope_create(const thinK_rope_config* cfg, thinK_rope** out) {
  if (!out) return THINK_ERR_INVALID_ARG;
  *out = nullptr;
  thinK_rope* r = new (std::nothrow) thinK_rope();
  if (!r) return THINK_ERR_INVALID_ARG;
  const thinK_status st = rope_frequencies(cfg, r);
  if (st != THINK_OK) {
    delete r;
    return st;
  }
  *out = r;
  return THINK_OK;
}

double thinK_rope_frequency(const thinK_rope* r, int32_t pair) {
  return r && pair >= 0 && pair < r->R / 2 ? r->radians[pair] : -1.0;
}

thinK_status thinK_rope_apply(const thinK_rope* r, thinK_tensor5 q, thinK_tensor5 k, thinK_tensor5 q_out, thinK_tensor5 k_out,
                              int32_t B, int32_t S, int32_t nlayers, int32_t N_q, int32_t N_kv, const int32_t* pos,
                              int64_t pos_stride, const int32_t* rows, int32_t transpose, void* stream) {
  Range nvtx_range("thinK_rope_apply");
  if (!r || B < 0 || S < 0 || nlayers < 0 || N_q < 0 || N_kv < 0 || (transpose & ~1)) return THINK_ERR_INVALID_ARG;
  if (B == 0 || S == 0 || nlayers == 0 || N_q + (int64_t)N_kv == 0) return THINK_OK;      // views without rows may have no memory
  if (!pos || ((uintptr_t)pos & 3) || ((uintptr_t)rows & 3) || pos_stride < 0 || (pos_stride > 0 && B > 1 && pos_stride < S)) return THINK_ERR_INVALID_ARG;
  const thinK_tensor5 in[2] = {q, k}, to[2] = {q_out, k_out};
  const int heads[2] = {N_q, N_kv};
  const int V = 16 / r->elem;
  RowView iv[2], ov[2];
  for (int i = 0; i < 2; ++i) {
    if (heads[i] == 0) continue;
    if (!side_ok(in[i], r->elem) || !side_ok(to[i], r->elem)) return THINK_ERR_INVALID_ARG;
    auto view = [&](const thinK_tensor5& t) {
      return RowView{{t.stride_b / V, t.stride_s / V, t.stride_l / V, t.stride_n / V}, {B, S, nlayers, heads[i]}, r->D / V};
    };
    iv[i] = view(in[i]);
    ov[i] = view(to[i]);
    if (!iv[i].spread_ok() || !ov[i].spread_ok() || ov[i].shares_with_itself()) return THINK_ERR_INVALID_ARG;
  }
  // a row is stored by threads of its own, which read nothing but that row
  for (int i = 0; i < 2; ++i)
    for (int j = 0; j < 2; ++j) {
      if (heads[i] == 0 || heads[j] == 0) continue;
      if (!(i == j && same(in[i], to[i])) &&
          ov[i].shares_with(iv[j], (int64_t)((uintptr_t)in[j].ptr / 16) - (int64_t)((uintptr_t)to[i].ptr / 16))) return THINK_ERR_INVALID_ARG;
      if (i < j && ov[i].shares_with(ov[j], (int64_t)((uintptr_t)to[j].ptr / 16) - (int64_t)((uintptr_t)to[i].ptr / 16))) return THINK_ERR_INVALID_ARG;
    }
  const bool in_place = (!N_q || same(q, q_out)) && (!N_kv || same(k, k_out));
  const int form = r->layout == THINK_ROPE_PAIRS ? kPairs : (r->R / 2) % V == 0 ? kHalves : (r->R / 2) % 2 == 0 ? kTwo : kOne;
  RopeParams p;
  memset((void*)&p, 0, sizeof(p));
  for (int i = 0; i < 2; ++i) {
    if (heads[i] == 0) continue;
    p.side[i] = RopeSide{(const uint8_t*)in[i].ptr, (uint8_t*)to[i].ptr,
                         in[i].stride_b * r->elem, in[i].stride_s * r->elem, in[i].stride_l * r->elem, in[i].stride_n * r->elem,
                         to[i].stride_b * r->elem, to[i].stride_s * r->elem, to[i].stride_l * r->elem, to[i].stride_n * r->elem};
  }
  p.R = r->R; p.D = r->D; p.pairs = r->R / 2;
  const int border = (p.R + V - 1) / V * V, rest = in_place ? 0 : (p.D - border) / V;        // pieces that no pair touches
  if (form == kPairs) p.units = border / V + rest;
  else if (form == kHalves) p.units = p.pairs / V + rest;
  else p.units = (p.pairs + (in_place ? 0 : border - p.R)) / (form == kTwo ? 2 : 1) + rest;
  if (form == kPairs && p.units % 2 == 0) p.second = p.units /= 2;
  p.table = form == kPairs ? border / 2 : p.pairs;
  const int64_t heads_all = (int64_t)N_q + N_kv, items = heads_all * nlayers * p.units;
  if (items > (1 << 24)) return THINK_ERR_UNSUPPORTED;                 // item numbers of a block fit 31 bits
  p.heads_q = N_q; p.heads = (int)heads_all;
  p.nlayers = nlayers; p.S = S;
  p.items = (int)items;
  p.m = r->m; p.sign = transpose ? -1.f : 1.f;
  p.pos = pos; p.pos_stride = pos_stride; p.rows = rows;
  // Tokens of a block: enough for four items a thread, as long as there are four blocks an SM; a table's worth at most.
  int tokens = (int)((4 * kRopeThreads + items - 1) / items);
  const int64_t fill = (int64_t)B * S / (4 * kSMs);
  if (tokens > fill) tokens = (int)fill;
  if (tokens > kRopeTable / p.table) tokens = kRopeTable / p.table;
  if (tokens > 64) tokens = 64;
  if (tokens < 1) tokens = 1;
  p.tokens = tokens;
  p.blocks_s = (int)(((int64_t)S + tokens - 1) / tokens);
  if ((int64_t)p.blocks_s * B > INT32_MAX) return THINK_ERR_UNSUPPORTED;
  p.by_items = FastDiv((uint32_t)p.items);
  p.by_units = FastDiv((uint32_t)p.units);
  p.by_heads = FastDiv((uint32_t)p.heads);
  p.by_pairs = FastDiv((uint32_t)p.pairs);
  p.by_blocks = FastDiv((uint32_t)p.blocks_s);
  memcpy(p.turns, r->turns, sizeof(p.turns));
  static void (*const kernels[2][4])(const RopeParams) = {{k_rope<2, kHalves>, k_rope<2, kPairs>, k_rope<2, kTwo>, k_rope<2, kOne>},
                                                          {k_rope<4, kHalves>, k_rope<4, kPairs>, k_rope<4, kTwo>, k_rope<4, kOne>}};
  void (*const kernel)(const RopeParams) = kernels[r->elem == 4][form];
  return launch_dependent(kernel, dim3((unsigned)(p.blocks_s * B)), kRopeThreads, 0, (cudaStream_t)stream, p) == cudaSuccess ? THINK_OK
                                                                                                                             : THINK_ERR_CUDA;
}

thinK_status thinK_rope_destroy(thinK_rope* r) {
  if (!r) return THINK_ERR_INVALID_ARG;
  delete r;
  return THINK_OK;
}

}  // extern "C"
