// Host side of the paged key-value cache: validation, sizes, launches.
#include <float.h>
#include <math.h>
#include <string.h>

#include <new>

#include <nvtx3/nvToolsExt.h>

#include "paged_internal.h"
#include "paged_views.h"

using namespace think;

namespace {

struct Range {
  explicit Range(const char* name) { nvtxRangePushA(name); }
  ~Range() { nvtxRangePop(); }
};

inline size_t align_up(size_t x, size_t a) { return (x + a - 1) / a * a; }
inline bool overlap(const void* a, size_t na, const void* b, size_t nb) {
  return a && b && (uintptr_t)a < (uintptr_t)b + nb && (uintptr_t)b < (uintptr_t)a + na;
}
inline bool aligned(const void* p, size_t a) { return ((uintptr_t)p & (a - 1)) == 0; }

struct Geometry {
  PageGeom g;
  int N_q, G, dtype, format, max_batch, elem;
  float scale_log2;
};

// Offsets in the workspace (and in a scratch buffer, whose error word is not used).  Partial states lie at the same
// place and take the same room whatever the handle, tickets behind them: handles of any shape may take turns on one
// scratch buffer without a state of one landing on a ticket of another.
struct Layout {
  size_t records, counters, total;
};

thinK_status make_geometry(const thinK_paged_config* c, Geometry* o) {
  if (!c) return THINK_ERR_INVALID_ARG;
  if (c->L < 1 || c->N_kv < 1 || c->N_q < 1 || c->num_pages < 1 || c->max_batch < 1 || c->D < 1) return THINK_ERR_INVALID_ARG;
  if (c->N_q % c->N_kv != 0) return THINK_ERR_INVALID_ARG;
  if (c->dtype != THINK_BF16 && c->dtype != THINK_F32) return THINK_ERR_UNSUPPORTED;
  if (c->page_format < THINK_PAGE_PLAIN || c->page_format > THINK_PAGE_INT4) return THINK_ERR_INVALID_ARG;
  constexpr double kLog2e = 1.4426950408889634074;
  if (!(c->softmax_scale >= 0.0 && c->softmax_scale * kLog2e <= FLT_MAX)) return THINK_ERR_INVALID_ARG;      // fp32 below
  if (c->D != 64 && c->D != 128) return THINK_ERR_UNSUPPORTED;
  if (c->N_q / c->N_kv > kMaxPagedGroup) return THINK_ERR_UNSUPPORTED;
  if (c->dtype != THINK_BF16 && c->page_format != THINK_PAGE_PLAIN) return THINK_ERR_UNSUPPORTED;
  if (c->max_batch > kMaxPagedBatch) return THINK_ERR_UNSUPPORTED;
  // units of a call (batch * layers * key heads) and query rows are counted in 32 bits
  if ((int64_t)c->max_batch * c->L > (1 << 24) || (int64_t)c->max_batch * c->L * c->N_q > INT32_MAX) return THINK_ERR_UNSUPPORTED;
  Geometry r;
  r.N_q = c->N_q;
  r.G = c->N_q / c->N_kv;
  r.dtype = c->dtype;
  r.format = c->page_format;
  r.max_batch = c->max_batch;
  r.elem = c->dtype == THINK_BF16 ? 2 : 4;
  r.g.L = c->L; r.g.N_kv = c->N_kv; r.g.D = c->D; r.g.num_pages = c->num_pages;
  r.g.row_bytes = c->page_format == THINK_PAGE_PLAIN ? c->D * r.elem : c->page_format == THINK_PAGE_E4M3 ? c->D : c->D / 2;
  r.g.scale_bytes = c->page_format == THINK_PAGE_PLAIN ? 0 : c->page_format == THINK_PAGE_E4M3 ? 1 : 2 * (c->D / kGroupChannels);
  r.g.block_bytes = 2 * kPageTokens * (r.g.row_bytes + r.g.scale_bytes);
  // the pool's size in bytes has to fit a signed 64-bit offset
  if ((double)c->L * c->num_pages * c->N_kv * r.g.block_bytes > 4.0e18) return THINK_ERR_UNSUPPORTED;
  const double scale = c->softmax_scale == 0.0 ? 1.0 / sqrt((double)c->D) : c->softmax_scale;
  r.scale_log2 = (float)(scale * kLog2e);
  *o = r;
  return THINK_OK;
}

void make_layout(const Geometry& g, Layout* w) {
  w->records = 256;                                    // the error word is in front
  w->counters = align_up(w->records + paged_decode_record_bytes(kSMs), 256);
  w->total = align_up(w->counters + sizeof(uint32_t) * (size_t)g.max_batch * g.g.L * g.g.N_kv, 256);
}

bool table_ok(const Geometry& g, const thinK_page_table& t) {
  return t.table && aligned(t.table, 4) && t.B >= 1 && t.B <= g.max_batch && t.max_pages >= 1 &&
         t.max_pages <= INT32_MAX / kPageTokens && t.table_stride >= t.max_pages;
}

bool view_ok(const thinK_tensor5& t, int elem) {
  if (!t.ptr || !aligned(t.ptr, 16)) return false;
  const int64_t s[4] = {t.stride_b, t.stride_s, t.stride_l, t.stride_n};
  for (int i = 0; i < 4; ++i)
    if (s[i] < 0 || s[i] % (16 / elem) != 0) return false;
  return true;
}

// rows that are written must not share memory: each is stored by threads of its own
bool destinations_ok(const thinK_tensor5& k, const thinK_tensor5& v, const Geometry& g, int B, int rows, int layers) {
  const int unit = 16 / g.elem;                        // view_ok: pointers and strides are multiples of 16 bytes
  auto view = [&](const thinK_tensor5& t) {
    return RowView{{t.stride_b / unit, t.stride_s / unit, t.stride_l / unit, t.stride_n / unit}, {B, rows, layers, g.g.N_kv}, g.g.D / unit};
  };
  const RowView a = view(k), b = view(v);
  if (!a.spread_ok() || !b.spread_ok() || a.shares_with_itself() || b.shares_with_itself()) return false;
  return !a.shares_with(b, (int64_t)((uintptr_t)v.ptr / 16) - (int64_t)((uintptr_t)k.ptr / 16));
}

}  // namespace

struct thinK_paged {
  Geometry g;
  Layout w;
  uint8_t* pages;
  uint8_t* ws;
  int grid;
};

namespace {
bool layers_ok(const thinK_paged* p, int layer0, int nlayers) {
  return layer0 >= 0 && nlayers >= 1 && layer0 <= p->g.g.L && nlayers <= p->g.g.L - layer0;
}

thinK_status rows_impl(thinK_paged* p, const thinK_tensor5& k, const thinK_tensor5& v, const thinK_page_table& t,
                       const int32_t* pos, const int32_t* rows, int32_t max_rows, int32_t layer0, int32_t nlayers,
                       void* stream, bool write) {
  if (!p || !layers_ok(p, layer0, nlayers) || !table_ok(p->g, t)) return THINK_ERR_INVALID_ARG;
  if (max_rows < 0 || (int64_t)max_rows * p->g.g.N_kv > (1 << 30) || !aligned(pos, 4) || !aligned(rows, 4)) return THINK_ERR_INVALID_ARG;
  if (max_rows == 0) return THINK_OK;                  // views without rows may have no memory
  if (!view_ok(k, p->g.elem) || !view_ok(v, p->g.elem)) return THINK_ERR_INVALID_ARG;
  if (!write && !destinations_ok(k, v, p->g, t.B, max_rows, nlayers)) return THINK_ERR_INVALID_ARG;
  PagedRowsParams r;
  memset((void*)&r, 0, sizeof(r));
  r.g = p->g.g;
  r.pages = p->pages;
  r.table = PageTableView{t.table, t.table_stride, t.max_pages, t.B};
  r.pos = pos; r.rows = rows; r.max_rows = max_rows;
  r.by_heads = FastDiv((uint32_t)p->g.g.N_kv);
  r.error = (uint32_t*)p->ws;
  // row indices of an entry are 32 bits wide: as many layers per launch as fit
  const int64_t fit = (1 << 30) / ((int64_t)max_rows * p->g.g.N_kv);
  const int per = fit < nlayers ? (int)fit : nlayers;
  for (int l = 0; l < nlayers; l += per) {
    r.layer0 = layer0 + l;
    r.nlayers = per < nlayers - l ? per : nlayers - l;
    r.by_layers = FastDiv((uint32_t)r.nlayers);
    r.k = View5{(uint8_t*)k.ptr + l * k.stride_l * p->g.elem, k.stride_b, k.stride_s, k.stride_l, k.stride_n};
    r.v = View5{(uint8_t*)v.ptr + l * v.stride_l * p->g.elem, v.stride_b, v.stride_s, v.stride_l, v.stride_n};
    if (launch_paged_rows(r, p->g.dtype, p->g.format, write, (cudaStream_t)stream) != cudaSuccess) return THINK_ERR_CUDA;
  }
  return THINK_OK;
}
}  // namespace

extern "C" {

thinK_status thinK_paged_bytes(const thinK_paged_config* cfg, thinK_paged_sizes* out) {
  if (!out) return THINK_ERR_INVALID_ARG;
  Geometry g;
  const thinK_status st = make_geometry(cfg, &g);
  if (st != THINK_OK) return st;
  Layout w;
  make_layout(g, &w);
  out->block = (size_t)g.g.block_bytes;
  out->pages = (size_t)g.g.block_bytes * g.g.N_kv * g.g.num_pages * g.g.L;
  out->workspace = w.total;
  return THINK_OK;
}

thinK_status thinK_paged_create(const thinK_paged_config* cfg, const thinK_paged_sizes* sizes, void* pages,
                                void* workspace, thinK_paged** out) {
  if (!out) return THINK_ERR_INVALID_ARG;
  *out = nullptr;
  if (!sizes || !pages || !workspace) return THINK_ERR_INVALID_ARG;
  thinK_paged_sizes need;
  thinK_status st = thinK_paged_bytes(cfg, &need);
  if (st != THINK_OK) return st;
  if (sizes->pages < need.pages || sizes->workspace < need.workspace) return THINK_ERR_CAPACITY;
  if (!aligned(pages, 256) || !aligned(workspace, 256)) return THINK_ERR_INVALID_ARG;
  thinK_paged* p = new (std::nothrow) thinK_paged();
  if (!p) return THINK_ERR_INVALID_ARG;
  make_geometry(cfg, &p->g);
  make_layout(p->g, &p->w);
  p->pages = (uint8_t*)pages;
  p->ws = (uint8_t*)workspace;
  int dev = 0, sms = 0;
  if (cudaGetDevice(&dev) != cudaSuccess || cudaDeviceGetAttribute(&sms, cudaDevAttrMultiProcessorCount, dev) != cudaSuccess ||
      paged_decode_setup(p->g.dtype, p->g.format, p->g.g.D, p->g.G) != cudaSuccess ||
      cudaMemset(p->ws, 0, p->w.records) != cudaSuccess ||
      cudaMemset(p->ws + p->w.counters, 0, p->w.total - p->w.counters) != cudaSuccess || cudaStreamSynchronize(cudaStreamLegacy) != cudaSuccess) {
    delete p;
    return THINK_ERR_CUDA;
  }
  p->grid = sms < kSMs ? sms : kSMs;                 // one wave, one CTA an SM
  *out = p;
  return THINK_OK;
}

int64_t thinK_paged_offset(const thinK_paged_config* cfg, int32_t layer, int32_t page, int32_t head, int32_t slot,
                           int32_t part) {
  Geometry g;
  if (make_geometry(cfg, &g) != THINK_OK) return -1;
  if (layer < 0 || layer >= g.g.L || page < 0 || page >= g.g.num_pages || head < 0 || head >= g.g.N_kv || slot < 0 ||
      slot >= kPageTokens || part < THINK_PART_K || part > THINK_PART_V_SCALE)
    return -1;
  const int per = part <= THINK_PART_V ? g.g.row_bytes : g.g.scale_bytes;
  if (per == 0) return -1;
  return page_block_offset(g.g, layer, page, head) + page_part_offset(g.g, part) + slot * per;
}

thinK_status thinK_paged_write(thinK_paged* p, thinK_tensor5 k, thinK_tensor5 v, thinK_page_table table,
                               const int32_t* pos, const int32_t* rows, int32_t max_rows, int32_t layer0,
                               int32_t nlayers, void* stream) {
  Range nvtx_range("thinK_paged_write");
  return rows_impl(p, k, v, table, pos, rows, max_rows, layer0, nlayers, stream, true);
}

thinK_status thinK_paged_read(thinK_paged* p, thinK_tensor5 k, thinK_tensor5 v, thinK_page_table table,
                              const int32_t* pos, const int32_t* rows, int32_t max_rows, int32_t layer0,
                              int32_t nlayers, void* stream) {
  Range nvtx_range("thinK_paged_read");
  return rows_impl(p, k, v, table, pos, rows, max_rows, layer0, nlayers, stream, false);
}

thinK_status thinK_paged_decode_attn(thinK_paged* p, const void* q, void* out, float* lse, thinK_page_table table,
                                     const int32_t* seq_len, void* scratch, size_t scratch_bytes, int32_t layer0,
                                     int32_t nlayers, void* stream) {
  Range nvtx_range("thinK_paged_decode_attn");
  if (!p || !q || !out || !seq_len || !layers_ok(p, layer0, nlayers) || !table_ok(p->g, table)) return THINK_ERR_INVALID_ARG;
  if (!aligned(q, 16) || !aligned(out, 16) || !aligned(lse, 4) || !aligned(seq_len, 4)) return THINK_ERR_INVALID_ARG;
  if (scratch && !aligned(scratch, 256)) return THINK_ERR_INVALID_ARG;
  if (scratch && scratch_bytes < p->w.total) return THINK_ERR_CAPACITY;
  // queries are read until the last output is written
  const size_t heads = (size_t)table.B * nlayers * p->g.N_q, bytes = heads * p->g.g.D * p->g.elem;
  if (overlap(q, bytes, out, bytes) || overlap(lse, heads * 4, q, bytes) || overlap(lse, heads * 4, out, bytes)) return THINK_ERR_INVALID_ARG;
  // four places a tile and two a sequence are counted in 32 bits, over all layers and heads in 54
  const int64_t tiles = (int64_t)table.B * table.max_pages;
  if (4 * tiles + 2 * (int64_t)table.B > INT32_MAX || (double)tiles * nlayers * p->g.g.N_kv > 4.0e15) return THINK_ERR_UNSUPPORTED;
  uint8_t* const ws = scratch ? (uint8_t*)scratch : p->ws;
  PagedDecodeParams d;
  memset((void*)&d, 0, sizeof(d));
  d.g = p->g.g;
  d.pages = p->pages;
  d.q = q; d.out = out; d.lse = lse;
  d.table = PageTableView{table.table, table.table_stride, table.max_pages, table.B};
  d.seq_len = seq_len;
  d.N_q = p->g.N_q; d.G = p->g.G;
  d.layer0 = layer0; d.nlayers = nlayers;
  d.scale_log2 = p->g.scale_log2;
  d.error = (uint32_t*)p->ws;
  d.counters = (uint32_t*)(ws + p->w.counters);
  d.records = ws + p->w.records;
  d.grid = p->grid;
  if (launch_paged_decode(d, p->g.dtype, p->g.format, (cudaStream_t)stream) != cudaSuccess) return THINK_ERR_CUDA;
  return THINK_OK;
}

thinK_status thinK_paged_device_error(thinK_paged* p, int32_t* out_code) {
  if (!p || !out_code) return THINK_ERR_INVALID_ARG;
  uint32_t v = 0;
  if (cudaMemcpy(&v, p->ws, sizeof(v), cudaMemcpyDeviceToHost) != cudaSuccess) return THINK_ERR_CUDA;
  *out_code = (int32_t)v;
  return THINK_OK;
}

thinK_status thinK_paged_destroy(thinK_paged* p) {
  if (!p) return THINK_ERR_INVALID_ARG;
  delete p;
  return THINK_OK;
}

}  // extern "C"
