"""CPU checks of the paged cache's host side: sizes, offsets, refusals, and the kernels' index arithmetic compiled for
the host.  No kernel is launched here."""
import ctypes as C
import os
import subprocess

import pytest

ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def tk():
    from paper_2407_21018_b200 import build
    build.build()
    from paper_2407_21018_b200 import binding
    return binding


def cfg_of(tk, **kw):
    base = dict(L=2, N_q=8, N_kv=4, D=128, num_pages=10, max_batch=3, dtype=tk.BF16, page_format=tk.PAGE_PLAIN)
    base.update(kw)
    return tk.make_paged_config(**base)


@pytest.mark.parametrize("fmt,dtype,D,row,scale", [
    (0, 0, 128, 256, 0), (0, 0, 64, 128, 0), (0, 1, 128, 512, 0), (0, 1, 64, 256, 0),
    (1, 0, 128, 128, 1), (1, 0, 64, 64, 1), (2, 0, 128, 64, 8), (2, 0, 64, 32, 4),
])
def test_sizes_and_offsets(tk, fmt, dtype, D, row, scale):
    c = cfg_of(tk, page_format=fmt, dtype=dtype, D=D)
    s = tk.paged_bytes(c)
    block = 2 * 64 * (row + scale)
    assert s.block == block and s.pages == 2 * 10 * 4 * block and block % 16 == 0
    at = lambda *a: tk.paged_offset(c, *a)  # noqa: E731
    base = ((1 * 10 + 7) * 4 + 3) * block
    assert at(1, 7, 3, 5, tk.PART_K) == base + 5 * row
    assert at(1, 7, 3, 5, tk.PART_V) == base + 64 * row + 5 * row
    assert at(1, 7, 3, 63, tk.PART_K_SCALE) == (base + 128 * row + 63 * scale if scale else -1)
    assert at(1, 7, 3, 63, tk.PART_V_SCALE) == (base + 128 * row + 64 * scale + 63 * scale if scale else -1)
    for bad in ((2, 0, 0, 0, 0), (-1, 0, 0, 0, 0), (0, 10, 0, 0, 0), (0, -1, 0, 0, 0), (0, 0, 4, 0, 0), (0, 0, 0, 64, 0),
                (0, 0, 0, -1, 0), (0, 0, 0, 0, 4), (0, 0, 0, 0, -1)):
        assert at(*bad) == -1


def test_offsets_past_32_bits(tk):
    c = cfg_of(tk, L=32, N_kv=8, N_q=32, num_pages=100000)
    assert tk.paged_offset(c, 31, 99999, 7, 63, tk.PART_V) == ((31 * 100000 + 99999) * 8 + 7) * 32768 + 127 * 256
    assert tk.paged_bytes(c).pages == 32 * 100000 * 8 * 32768


@pytest.mark.parametrize("kw", [
    dict(D=96), dict(D=0), dict(N_q=6), dict(N_q=36), dict(L=0), dict(N_kv=0), dict(num_pages=0), dict(max_batch=0),
    dict(max_batch=4097), dict(dtype=7), dict(page_format=3), dict(page_format=-1), dict(softmax_scale=-1.0),
    dict(softmax_scale=float("nan")), dict(softmax_scale=float("inf")), dict(dtype=1, page_format=1),
    dict(dtype=1, page_format=2), dict(L=2 ** 30, num_pages=2 ** 30, N_kv=2 ** 20, N_q=2 ** 20),
])
def test_invalid_configs_are_refused(tk, kw):
    with pytest.raises(tk.ThinKError) as e:
        tk.paged_bytes(cfg_of(tk, **kw))
    assert e.value.status in (tk.ERR_INVALID_ARG, tk.ERR_UNSUPPORTED)


def test_create_refusals(tk):
    c = cfg_of(tk)
    need = tk.paged_bytes(c)
    h = C.c_void_p()
    create = tk.lib.thinK_paged_create
    ok = (C.byref(c), C.byref(need), 4096, 4096, C.byref(h))
    for i in range(5):
        a = list(ok)
        a[i] = None
        assert create(*a) == tk.ERR_INVALID_ARG
    for i in (2, 3):                                  # misaligned buffers
        a = list(ok)
        a[i] = 4096 + 16
        assert create(*a) == tk.ERR_INVALID_ARG
    for name in ("pages", "workspace"):
        have = tk.paged_bytes(c)
        setattr(have, name, getattr(have, name) - 1)
        assert create(C.byref(c), C.byref(have), 4096, 4096, C.byref(h)) == tk.ERR_CAPACITY
    assert not h.value
    assert tk.lib.thinK_paged_bytes(C.byref(c), None) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_paged_bytes(None, C.byref(need)) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_paged_destroy(None) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_paged_device_error(None, None) == tk.ERR_INVALID_ARG


def test_calls_without_a_handle(tk):
    t5, tab = tk.Tensor5(4096, 0, 0, 0, 0), tk.PageTable(4096, 4, 4, 1)
    for fn in (tk.lib.thinK_paged_write, tk.lib.thinK_paged_read):
        assert fn(None, t5, t5, tab, None, None, 1, 0, 1, None) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_paged_decode_attn(None, 4096, 4096, None, tab, 4096, None, 0, 0, 1, None) == tk.ERR_INVALID_ARG


def compile_and_run(tmp_path, source: str) -> str:
    src, exe = tmp_path / "probe.cu", tmp_path / "probe"
    src.write_text(source)
    nvcc = os.environ.get("NVCC", "/usr/local/cuda/bin/nvcc")
    subprocess.run([nvcc, "-std=c++17", "-O1", "-gencode", "arch=compute_100a,code=sm_100a", "-I",
                    os.path.join(ROOT, "include"), "-I", os.path.join(ROOT, "paper_2407_21018_b200", "csrc"), str(src),
                    "-o", str(exe)], check=True, capture_output=True)
    r = subprocess.run([str(exe)], check=True, capture_output=True, text=True, timeout=120)
    return r.stdout


def test_row_index_division(tmp_path):
    """The reciprocal division that splits a row index into token, layer and head is exact below 2^31."""
    out = compile_and_run(tmp_path, r"""
#include <stdio.h>
#include "paged_internal.h"
int main() {
  long bad = 0;
  uint32_t ds[] = {1, 2, 3, 4, 5, 6, 7, 8, 9, 12, 31, 32, 33, 80, 96, 127, 128, 1000, 4095, 65535, 65537, (1u << 30) - 1, 1u << 30};
  for (uint32_t d : ds) {
    think::FastDiv f(d);
    for (uint64_t i = 0; i < 400000; ++i) {
      uint64_t x[4] = {i, 0x7fffffffull - i, (i * 2654435761ull) & 0x7fffffffull, (i * (uint64_t)d) & 0x7fffffffull};
      for (uint64_t y : x)
        for (long o = -1; o <= 1; ++o) {
          long z = (long)y + o;
          if (z < 0 || z > 0x7fffffffl) continue;
          bad += f.div((uint32_t)z) != (uint32_t)z / d;
        }
    }
  }
  printf("%ld\n", bad);
}
""")
    assert out.strip() == "0"


def test_split_of_places(tmp_path):
    """Parts of a line are contiguous, differ by one place at most, and the owner of a place is the part that holds
    it - at lengths of a few places and of 2^50.  Tiles of a unit stand where `slot` says and are found again, and no
    part of a weighted line is without a tile."""
    out = compile_and_run(tmp_path, r"""
#include <stdio.h>
#include "paged_split.h"
using namespace think;
int main() {
  long bad = 0;
  for (int parts : {1, 2, 7, 8, 132, 148})
    for (int64_t n : {int64_t(1), int64_t(2), int64_t(7), int64_t(147), int64_t(148), int64_t(149), int64_t(1000), int64_t(54321), int64_t(1) << 50}) {
      bad += split_begin(n, parts, 0) != 0 || split_begin(n, parts, parts) != n;
      for (int i = 0; i < parts; ++i) {
        const int64_t a = split_begin(n, parts, i), b = split_begin(n, parts, i + 1);
        bad += b < a || b - a > n / parts + 1;
        for (int64_t f : {a, a + 1, (a + b) / 2, b - 1})
          if (f >= a && f < b) bad += split_owner(n, parts, f) != i;
      }
    }
  for (Weights w : {Weights{4, 1}, Weights{2, 2}, Weights{1, 1}, Weights{1, 0}})
    for (int nt = 1; nt < 40; ++nt) {
      bad += w.tiles(w.cost(nt)) != nt;
      for (int64_t x = -2; x < w.cost(nt) + 3; ++x) {
        int j = 0;
        while (j < nt && w.slot(j) < x) ++j;
        const int got = w.first_tile(x);
        bad += j < nt ? got != j : got < nt;
      }
      bad += w.slot(nt - 1) >= w.cost(nt);
    }
  // tile + unit places in a row always hold a tile's, across units of any length
  for (Weights w : {Weights{4, 1}, Weights{2, 2}})
    for (int a = 1; a < 6; ++a)
      for (int b = 1; b < 6; ++b) {
        bool at[64] = {};
        for (int j = 0; j < a; ++j) at[w.slot(j)] = true;
        for (int j = 0; j < b; ++j) at[w.cost(a) + w.slot(j)] = true;
        at[w.cost(a) + w.cost(b)] = true;                    // a third unit
        for (int i = 0; i < w.cost(a) + w.cost(b); ++i) {
          bool any = false;
          for (int k = 0; k < w.tile + w.unit; ++k) any |= at[i + k];
          bad += i + w.tile + w.unit <= w.cost(a) + w.cost(b) + 1 && !any;
        }
      }
  bad += weights_for({1, 1}, 100, 100, 148).unit != 0 || weights_for({1, 1}, 148, 148, 148).unit != 1 || weights_for({4, 1}, 184, 1, 148).unit != 0;
  printf("%ld\n", bad);
}
""")
    assert out.strip() == "0"


def test_views_that_share_memory(tmp_path):
    """Row views against marking every unit of memory: random strides, views of dense tensors in any order, pairs side by
    side, interleaved and overlapping; extents of millions; a search that is cut short says that they share."""
    out = compile_and_run(tmp_path, r"""
#include <stdio.h>
#include <string.h>
#include <chrono>
#include <random>
#include "paged_views.h"
using namespace think;
static uint8_t mem[1 << 20];
static long base = 4096;
static bool mark(const RowView& v, long at) {               // true: a unit was marked already
  bool twice = false;
  for (long a = 0; a < v.extent[0]; ++a) for (long b = 0; b < v.extent[1]; ++b) for (long c = 0; c < v.extent[2]; ++c)
    for (long d = 0; d < v.extent[3]; ++d) for (long r = 0; r < v.row; ++r) {
      uint8_t& m = mem[base + at + a * v.stride[0] + b * v.stride[1] + c * v.stride[2] + d * v.stride[3] + r];
      twice |= m; m = 1;
    }
  return twice;
}
int main() {
  std::mt19937 g(7);
  auto rnd = [&](int n) { return (int)(g() % n); };
  long bad = 0, cases = 0, shared = 0;
  for (int it = 0; it < 60000; ++it) {
    RowView a, b;
    for (RowView* v : {&a, &b}) {
      v->row = 1 + rnd(4);
      const bool dense = rnd(2);
      int order[4] = {0, 1, 2, 3};
      for (int i = 3; i > 0; --i) { int j = rnd(i + 1), t = order[i]; order[i] = order[j]; order[j] = t; }
      long at = v->row + (rnd(3) ? 0 : rnd(5));
      for (int i : order) {
        v->extent[i] = 1 + rnd(4);
        v->stride[i] = dense ? at : rnd(40);
        if (dense) at *= v->extent[i] + (rnd(3) ? 0 : 1);
      }
    }
    if (rnd(3) == 0) b = a;                                  // the same layout, shifted
    memset(mem, 0, sizeof(mem));
    const bool self = mark(a, 0);
    bad += a.shares_with_itself() != self;
    if (rnd(2)) b.row = a.row;
    const long apart = rnd(600) - 300;
    memset(mem, 0, sizeof(mem));
    mark(a, 0);
    bool both = false;
    for (long x = 0; x < b.extent[0]; ++x) for (long y = 0; y < b.extent[1]; ++y) for (long z = 0; z < b.extent[2]; ++z)
      for (long w = 0; w < b.extent[3]; ++w) for (long r = 0; r < b.row; ++r)
        both |= mem[base + apart + x * b.stride[0] + y * b.stride[1] + z * b.stride[2] + w * b.stride[3] + r];
    bad += a.shares_with(b, apart) != both || b.shares_with(a, -apart) != both;
    ++cases; shared += both + self;
  }
  // [4096][131072][80][8] rows of 16: dense, key and value rows interleaved, one row too many
  RowView big = {{131072ll * 80 * 8 * 32, 80 * 8 * 32, 8 * 32, 32}, {4096, 131072, 80, 8}, 16};
  auto t0 = std::chrono::steady_clock::now();
  bad += big.shares_with_itself() || big.shares_with(big, 16) || big.shares_with(big, -16) || !big.shares_with(big, 15) || big.shares_with(big, 48) || !big.shares_with(big, 40);
  RowView heads = {{131072ll * 80 * 8 * 32, 16, 131072ll * 8 * 16, 131072ll * 16}, {4096, 131072, 80, 8}, 16};      // b l n s
  RowView rows = {{131072ll * 80 * 8 * 32, 80 * 8 * 16, 8 * 16, 16}, {4096, 131072, 80, 8}, 16};                    // b s l n
  bad += heads.shares_with(rows, 131072ll * 80 * 8 * 16) || !heads.shares_with(rows, 131072ll * 80 * 8 * 16 - 1) || heads.shares_with_itself();
  bad += std::chrono::duration<double>(std::chrono::steady_clock::now() - t0).count() > 0.05;
  RowView wide = big;
  wide.extent[3] = 9;
  bad += !wide.shares_with_itself();
  RowView zero = big;
  zero.stride[2] = 0;
  bad += !zero.shares_with_itself();
  zero.extent[2] = 1;
  bad += zero.shares_with_itself();
  bad += !big.spread_ok();
  big.stride[1] = 1ll << 50;
  bad += big.spread_ok();
  RowView odd = {{1 << 20, (1 << 20) + 16, (1 << 20) + 48, (1 << 20) + 112}, {4000, 4000, 4000, 4000}, 16};      // long search
  bad += !odd.shares_with_itself();
  printf("%ld %d %d\n", bad, cases > 0, shared > cases / 10 && shared < cases * 19 / 10);
}
""")
    assert out.split() == ["0", "1", "1"]


def test_softmax_scale_in_base_2_stays_finite(tk):
    """The kernels take the scale times log2(e) in fp32."""
    top = 3.4028234e38 / 1.4426951
    assert tk.paged_bytes(cfg_of(tk, softmax_scale=top * 0.999999)).block > 0
    for scale in (top * 1.000001, 2.5e38, 3.0e38, 1e39):
        with pytest.raises(tk.ThinKError) as e:
            tk.paged_bytes(cfg_of(tk, softmax_scale=scale))
        assert e.value.status == tk.ERR_INVALID_ARG
