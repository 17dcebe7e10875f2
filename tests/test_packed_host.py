"""CPU checks of packed batches over the paged cache and of rotary positions: how attention of many new tokens is cut over
CTAs, frequencies, and the refusals of every entry point.  No kernel is launched here: the paged cache's host side is
compiled with launches that only count."""
import ctypes as C
import math
import os
import subprocess

import pytest
import torch

from test_paged_host import ROOT, compile_and_run, tk  # noqa: F401


def test_cut_of_a_line(tmp_path):
    """Shares, quotients, the places of tiles and items against plain arithmetic; every tile of random batches belongs to
    exactly one part, parts in order."""
    out = compile_and_run(tmp_path, r"""
#include <stdio.h>
#include <algorithm>
#include <random>
#include <vector>
#include "paged_prompt.h"
using namespace think;
int main() {
  std::mt19937_64 g(5);
  auto below = [&](int64_t n) { return (int64_t)(g() % (uint64_t)n); };
  long bad = 0, aligned = 0;
  for (int it = 0; it < 200000; ++it) {
    const int parts = 1 + (int)below(it & 1 ? 148 : 1 << 15);
    const int64_t n = below((int64_t)1 << (1 + below(62)));
    const PromptShare s(n, parts);
    for (int i : {0, 1, (int)below(parts + 1), parts - 1, parts}) bad += s.begin(i) != (int64_t)((__int128)n * i / parts);
    const int64_t len = 1 + below((int64_t)1 << (1 + below(50))), q = below(2147483647);
    if ((__int128)len * (q + 1) < (__int128)1 << 62) {
      bad += prompt_quotient(len * q, len) != q || prompt_quotient(len * q + len - 1, len) != q || prompt_quotient(len * q + below(len), len) != q;
    }
  }
  for (PromptCut cut : {PromptCut{384}, PromptCut{64}}) {
    for (int64_t x = -70; x < 2000; ++x) {
      const int64_t j = cut.first_tile(x);
      bad += cut.slot(j) < x || (j > 0 && cut.slot(j - 1) >= x);
    }
    for (int it = 0; it < 500; ++it) {
      const int B = 1 + (int)below(12), lh = 1 + (int)below(9), per = 1 + (int)below(256), most = 1 + (int)below(148);
      std::vector<PromptLine> line;
      std::vector<int> pos;
      int64_t W = 0, items = 0;
      for (int b = 0; b < B; ++b) {
        pos.push_back((int)below(3) ? (int)below(3000) : 0);
        line.push_back(PromptLine{(int64_t)cut.extra + pos[b], (int)below(4) ? (int)below(900) : 0, per});
        const PromptLine& l = line[b];
        int64_t sum = 0;
        for (int64_t i = 0; i < l.items(); ++i) {
          bad += l.begin(i) != sum || l.find(sum) != i || l.find(sum + l.cost(i) - 1) != i;
          bad += l.cost(i) != cut.extra + pos[b] + std::min<int64_t>((i + 1) * per, l.rows);
          sum += l.cost(i);
        }
        bad += sum != l.total();
        W += sum;
        items += l.items();
      }
      const int64_t total = W * lh;
      if (total == 0) continue;
      int64_t largest = 0;
      for (const PromptLine& l : line) if (l.items() > 0) largest = std::max(largest, l.cost(l.items() - 1));
      const int pieces = cut.pieces(total, items * lh, largest, most);
      bad += pieces * items * lh > most;
      aligned += pieces > 0;
      const PromptShare share(total, most);
      int64_t at = 0, tiles_seen = 0, tiles_all = 0, number = 0;
      for (int i = 0; i < lh; ++i)
        for (int b = 0; b < B; ++b)
          for (int k = 0; k < line[b].items(); ++k, ++number) {
            const int n = (int)(line[b].cost(k) - cut.extra), tiles = (n + 63) / 64;
            tiles_all += tiles;
            int64_t next = 0;
            const PromptShare own(line[b].cost(k), pieces ? pieces : 1);
            for (int c = pieces ? (int)number * pieces : 0; c < (pieces ? (int)(number + 1) * pieces : most); ++c) {
              const int64_t begin = pieces ? at + own.begin(c % pieces) : share.begin(c), end = pieces ? at + own.begin(c % pieces + 1) : share.begin(c + 1);
              const int64_t t0 = std::min<int64_t>(tiles, cut.first_tile(begin - at)), t1 = std::min<int64_t>(tiles, cut.first_tile(end - at));
              if (t0 == t1) continue;
              bad += t0 != next;
              next = t1;
              tiles_seen += t1 - t0;
            }
            bad += next != tiles;
            at += line[b].cost(k);
          }
      bad += at != total || tiles_seen != tiles_all;
    }
  }
  // the longest lines that a call may name
  const PromptLine longest{(int64_t)256 + 2147483000, 647, 32};
  bad += longest.total() <= 0;
  const PromptLine many{(int64_t)256, 1 << 30, 1};
  bad += many.total() != (int64_t)256 * (1 << 30) + ((int64_t)1 << 29) * ((1 << 30) + 1) || many.find(many.total() - 1) != (1 << 30) - 1;
  printf("%ld %d\n", bad, aligned > 20);
}
""")
    assert out.split() == ["0", "1"]


# ---- the paged cache's host side with launches that count
FAKE = r"""
#include "paged_internal.h"
#include "paged_prompt_walk.cuh"
using namespace think;
static int launches;
extern "C" {
cudaError_t CUDARTAPI cudaGetDevice(int* d) { *d = 0; return cudaSuccess; }
cudaError_t CUDARTAPI cudaDeviceGetAttribute(int* v, cudaDeviceAttr, int) { *v = 148; return cudaSuccess; }
cudaError_t CUDARTAPI cudaMemset(void*, int, size_t) { return cudaSuccess; }
cudaError_t CUDARTAPI cudaMemcpy(void*, const void*, size_t, cudaMemcpyKind) { return cudaSuccess; }
cudaError_t CUDARTAPI cudaStreamSynchronize(cudaStream_t) { return cudaSuccess; }
static CUresult map_ok(...) { return CUDA_SUCCESS; }
cudaError_t CUDARTAPI cudaGetDriverEntryPointByVersion(const char*, void** fn, unsigned, unsigned long long, cudaDriverEntryPointQueryResult* r) {
  *fn = (void*)map_ok;
  if (r) *r = cudaDriverEntryPointSuccess;
  return cudaSuccess;
}
int fake_launches() { const int n = launches; launches = 0; return n; }
}
namespace think {
cudaError_t launch_paged_rows(const PagedRowsParams&, int, int, bool, cudaStream_t) { ++launches; return cudaSuccess; }
cudaError_t launch_paged_plan(const PagedPlanParams&, cudaStream_t) { ++launches; return cudaSuccess; }
cudaError_t launch_paged_decode(const PagedDecodeParams&, int, int, cudaStream_t) { ++launches; return cudaSuccess; }
cudaError_t launch_paged_prompt(const PagedPromptParams&, int, int, const void*, cudaStream_t) { ++launches; return cudaSuccess; }
cudaError_t paged_decode_setup(int, int, int, int) { return cudaSuccess; }
cudaError_t paged_prompt_setup(int, int, int) { return cudaSuccess; }
size_t paged_decode_record_bytes(int ctas) { return 4096 * (size_t)ctas; }
int paged_prompt_rows(int dtype) { return dtype == THINK_BF16 ? 256 : 64; }
PromptCut paged_prompt_cut(int) { return PromptCut{384}; }
}
"""


@pytest.fixture(scope="module")
def fake(tk, tmp_path_factory):  # noqa: F811
    d = tmp_path_factory.mktemp("fake")
    (d / "fake.cpp").write_text("#include <cuda.h>\n" + FAKE)
    csrc = os.path.join(ROOT, "paper_2407_21018_b200", "csrc")
    so = str(d / "fake.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    "-I", "/usr/local/cuda/include", "-x", "c++", os.path.join(csrc, "paged_api.cu"), str(d / "fake.cpp"), "-o", so],
                   check=True, capture_output=True)
    lib = C.CDLL(so)
    for name in ("thinK_paged_create", "thinK_paged_plan", "thinK_paged_write_slots", "thinK_paged_prompt_attn", "thinK_paged_prompt_scratch",
                 "thinK_paged_bytes", "thinK_paged_destroy"):
        real = getattr(tk.lib, name)
        getattr(lib, name).argtypes, getattr(lib, name).restype = real.argtypes, real.restype
    return lib


def handle(tk, fake, **kw):  # noqa: F811
    base = dict(L=2, N_q=8, N_kv=4, D=128, num_pages=10, max_batch=8, dtype=tk.BF16, page_format=tk.PAGE_PLAIN)
    base.update(kw)
    cfg = tk.make_paged_config(**base)
    need, h = tk.PagedSizes(), C.c_void_p()
    assert fake.thinK_paged_bytes(C.byref(cfg), C.byref(need)) == 0
    assert fake.thinK_paged_create(C.byref(cfg), C.byref(need), 1 << 40, 1 << 41, C.byref(h)) == 0
    return h


def test_plan_refusals(tk, fake):  # noqa: F811
    h = handle(tk, fake)
    B, max_pages, tokens = 5, 4, 100
    at = lambda i: (1 << 30) + i * 4096  # noqa: E731
    names = ["table", "seq_len", "change", "free_pages", "free_count", "pos", "rows", "start", "token_pos", "slots", "seq_len_out", "free_left"]
    base = dict(table_stride=max_pages, max_pages=max_pages, B=B, max_tokens=tokens, **{n: at(i) for i, n in enumerate(names)})

    def call(**kw):
        st = fake.thinK_paged_plan(h, C.byref(tk.PagedStep(**{**base, **kw})), None)
        assert fake.fake_launches() == (st == 0)
        return st
    assert call() == 0
    assert fake.thinK_paged_plan(None, C.byref(tk.PagedStep(**base)), None) == tk.ERR_INVALID_ARG
    assert fake.thinK_paged_plan(h, None, None) == tk.ERR_INVALID_ARG
    for n in names:
        assert call(**{n: None}) == tk.ERR_INVALID_ARG, n
        assert call(**{n: base[n] + 2}) == tk.ERR_INVALID_ARG, n
    for n in ("token_pos", "slots"):
        assert call(**{n: base[n] + 4}) == tk.ERR_INVALID_ARG
        assert call(**{n: base[n] + 16}) == 0
    for kw in (dict(B=0), dict(B=9), dict(max_pages=0), dict(table_stride=3), dict(max_tokens=0), dict(max_tokens=(1 << 30) + 1), dict(B=-1)):
        assert call(**kw) == tk.ERR_INVALID_ARG, kw
    # in place: lengths and the count of free pages, those alone
    assert call(seq_len_out=base["seq_len"], free_left=base["free_count"]) == 0
    assert call(seq_len_out=base["seq_len"] + 4) == tk.ERR_INVALID_ARG
    assert call(seq_len_out=base["change"]) == tk.ERR_INVALID_ARG
    assert call(free_left=base["seq_len"]) == tk.ERR_INVALID_ARG
    sizes = dict(table=4 * B * max_pages, seq_len=4 * B, change=4 * B, free_pages=40, free_count=4, pos=4 * B, rows=4 * B, start=4 * B + 4,
                 token_pos=4 * tokens, slots=4 * tokens, seq_len_out=4 * B, free_left=4)
    given = ("seq_len", "change", "free_count")
    for a in names:                                   # results on one another or on arguments: the first and last bytes, and just behind
        for b in names:
            if a == b or a in given and b in given or a in ("token_pos", "slots"):
                continue
            if (a, b) in (("seq_len_out", "seq_len"), ("seq_len", "seq_len_out"), ("free_left", "free_count"), ("free_count", "free_left")):
                continue
            assert call(**{a: base[b] + sizes[b] - 4}) == tk.ERR_INVALID_ARG, (a, b)
            assert call(**{a: base[b] + sizes[b] + 2048}) == 0, (a, b)
            assert call(**{a: base[b] - sizes[a] + 4}) == tk.ERR_INVALID_ARG, (a, b)
            assert call(**{a: base[b] - sizes[a]}) == 0, (a, b)
    wide = handle(tk, fake, num_pages=1 << 25, L=1, N_kv=1, N_q=1, D=64)
    st = fake.thinK_paged_plan(wide, C.byref(tk.PagedStep(**{**base, "free_pages": 1 << 36})), None)
    assert st == tk.ERR_UNSUPPORTED and fake.fake_launches() == 0         # a slot would not fit 32 bits


def test_write_slots_refusals(tk, fake):  # noqa: F811
    h = handle(tk, fake)
    t = tk.Tensor5(1 << 30, 0, 8 * 128, 4 * 128, 128)
    u = tk.Tensor5(1 << 31, 0, 8 * 128, 4 * 128, 128)

    def call(k=t, v=u, slots=4096, tokens=7, layer0=0, nlayers=2, h=h):
        st = fake.thinK_paged_write_slots(h, k, v, slots, tokens, layer0, nlayers, None)
        assert fake.fake_launches() == (st == 0 and tokens > 0)
        return st
    assert call() == 0 and call(tokens=0, k=tk.Tensor5(), v=tk.Tensor5(), slots=None) == 0
    assert call(k=tk.Tensor5(1 << 30, -5, 8 * 128, 4 * 128, 128)) == 0    # (its b axis is not looked at)
    bad = [dict(h=None), dict(tokens=-1), dict(slots=None), dict(slots=4098), dict(layer0=-1), dict(layer0=1), dict(nlayers=0), dict(nlayers=3),
           dict(k=tk.Tensor5()), dict(v=tk.Tensor5())]
    bad += [dict(k=tk.Tensor5((1 << 30) + 8, 0, 1024, 512, 128)), dict(v=tk.Tensor5(1 << 30, 0, 1025, 512, 128)), dict(v=tk.Tensor5(1 << 30, 0, 1024, 512, -128))]
    for kw in bad:
        assert call(**kw) == tk.ERR_INVALID_ARG, kw


@pytest.mark.parametrize("dtype,fmt", [(0, 0), (0, 1), (0, 2), (1, 0)])
def test_prompt_refusals(tk, fake, dtype, fmt):  # noqa: F811
    h = handle(tk, fake, dtype=dtype, page_format=fmt)
    elem, B, S, N, L, D = 4 if dtype else 2, 3, 5, 8, 2, 128
    need = fake.thinK_paged_prompt_scratch(h)
    rows = 64 if dtype else 256
    assert need % 256 == 0 and 2 * 148 * rows * (D + 2) * 4 <= need < 2 * 148 * rows * (D + 2) * 4 + 8192
    assert fake.thinK_paged_prompt_scratch(None) == 0
    dense = (S * L * N * D, L * N * D, N * D, D)
    q, out = tk.Tensor5(1 << 30, *dense), tk.Tensor5(1 << 31, *dense)
    tab = tk.PageTable(4096, 4, 4, B)

    def call(q=q, out=out, lse=1 << 33, tab=tab, pos=4096, rows=4096, start=None, max_rows=S, scratch=1 << 34, size=need, layer0=0, nlayers=2, h=h):
        st = fake.thinK_paged_prompt_attn(h, q, out, lse, tab, pos, rows, start, max_rows, scratch, size, layer0, nlayers, None)
        assert fake.fake_launches() == (st == 0 and max_rows > 0)
        return st
    flat = tk.Tensor5(1 << 31, -1, *dense[1:])
    assert call() == 0 and call(lse=None, pos=None, rows=None) == 0 and call(start=4096, out=flat) == 0
    assert call(max_rows=0, q=tk.Tensor5(), out=tk.Tensor5(), scratch=None, size=0) == 0
    bad = [dict(h=None), dict(max_rows=-1), dict(scratch=None), dict(scratch=(1 << 34) + 128), dict(lse=(1 << 33) + 2), dict(pos=4097), dict(rows=4098),
           dict(start=4098), dict(start=4096, rows=None), dict(layer0=1), dict(nlayers=0), dict(layer0=-1), dict(q=tk.Tensor5()), dict(out=tk.Tensor5())]
    bad += [dict(tab=tk.PageTable(*a)) for a in ((None, 4, 4, B), (4098, 4, 4, B), (4096, 3, 4, B), (4096, 4, 0, B), (4096, 4, 4, 0), (4096, 4, 4, 9))]
    view = lambda at, *s: tk.Tensor5(at, *s)  # noqa: E731
    bad += [dict(q=view((1 << 30) + 8, *dense)), dict(q=view(1 << 30, dense[0], dense[1], dense[2], D + 1)), dict(q=view(1 << 30, -dense[0], *dense[1:]))]
    # rows of out that share memory: with one another, with queries, with lse
    bad += [dict(out=view(1 << 31, 0, *dense[1:])), dict(out=view(1 << 31, dense[0], 0, *dense[2:])), dict(out=view(1 << 31, *dense[:3], D - 16)),
            dict(out=q), dict(out=view((1 << 30) + 16, *dense)), dict(out=view((1 << 30) + (B * dense[0] - D) * elem, *dense)),
            dict(lse=1 << 30), dict(lse=(1 << 31) + 4), dict(lse=(1 << 31) - 4)]
    for kw in bad:
        assert call(**kw) == tk.ERR_INVALID_ARG, kw
    assert call(out=view((1 << 30) + B * dense[0] * elem, *dense)) == 0
    assert call(q=view(1 << 30, 0, 0, 0, 0)) == 0                         # queries may repeat
    assert call(size=need - 1) == tk.ERR_CAPACITY
    # positions, and the places of all items, are counted in 31 and 62 bits
    far = dict(q=tk.Tensor5(1 << 45, 1 << 36, *dense[1:]), out=tk.Tensor5(1 << 50, 1 << 36, *dense[1:]), lse=None)
    most = tk.PageTable(1 << 35, (1 << 25) - 1, (1 << 25) - 1, B)
    assert call(**far, max_rows=63, tab=most) == 0 and call(**far, max_rows=64, tab=most) == tk.ERR_UNSUPPORTED
    assert call(**far, max_rows=1 << 20, tab=tk.PageTable(1 << 35, 1 << 24, 1 << 24, B)) == 0
    # (a billion rows over a billion tokens, 3 sequences, 2 layers, 4 heads: 2^30 / rows * G items of up to 2^31 places)
    assert call(**far, start=4096, max_rows=1 << 30, tab=tk.PageTable(1 << 35, 1 << 24, 1 << 23, B)) == tk.ERR_UNSUPPORTED


def test_calls_without_a_handle(tk):  # noqa: F811
    t5, tab = tk.Tensor5(4096, 0, 0, 0, 0), tk.PageTable(4096, 4, 4, 1)
    assert tk.lib.thinK_paged_plan(None, C.byref(tk.PagedStep()), None) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_paged_write_slots(None, t5, t5, 4096, 1, 0, 1, None) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_paged_prompt_attn(None, t5, t5, None, tab, None, None, None, 1, 4096, 1 << 30, 0, 1, None) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_paged_prompt_scratch(None) == 0


# ---- rotary positions
def rope_of(tk, **kw):  # noqa: F811
    base = dict(D=128, rot_dim=128, layout=tk.ROPE_HALVES, scaling=tk.ROPE_PLAIN, dtype=tk.BF16, theta=1e4, factor=1.0, trained=0.0, slow=0.0,
                fast=0.0, attention_factor=0.0)
    base.update(kw)
    h = C.c_void_p()
    return tk.lib.thinK_rope_create(C.byref(tk.RopeConfig(**base)), C.byref(h)), h


@pytest.mark.parametrize("kw", [
    dict(D=0), dict(rot_dim=0), dict(rot_dim=3), dict(rot_dim=130), dict(rot_dim=-2), dict(layout=2), dict(layout=-1), dict(scaling=5), dict(scaling=-1),
    dict(theta=0.5), dict(theta=float("nan")), dict(theta=float("inf")), dict(theta=-1e4), dict(attention_factor=-1.0), dict(attention_factor=float("nan")),
    dict(scaling=1, factor=0.5), dict(scaling=1, factor=float("nan")), dict(scaling=1, factor=float("inf")), dict(scaling=2, factor=2.0, rot_dim=2),
    dict(scaling=3, factor=2.0), dict(scaling=4, factor=2.0), dict(scaling=3, factor=2.0, trained=0.5), dict(scaling=3, factor=2.0, trained=float("nan")),
    dict(scaling=3, factor=2.0, trained=4096, theta=1.0), dict(scaling=4, factor=2.0, trained=4096, slow=4.0, fast=4.0),
    dict(scaling=4, factor=2.0, trained=4096, slow=-1.0), dict(scaling=4, factor=2.0, trained=4096, fast=float("inf")),
])
def test_rope_configs_that_are_refused(tk, kw):  # noqa: F811
    st, h = rope_of(tk, **kw)
    assert st == tk.ERR_INVALID_ARG and not h.value


def test_rope_limits(tk):  # noqa: F811
    for kw in (dict(dtype=7), dict(D=258, rot_dim=8), dict(D=260, rot_dim=8, dtype=1), dict(D=12, rot_dim=4), dict(D=6, rot_dim=4, dtype=1)):
        assert rope_of(tk, **kw)[0] == tk.ERR_UNSUPPORTED, kw
    assert tk.lib.thinK_rope_create(None, C.byref(C.c_void_p())) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_rope_create(C.byref(tk.RopeConfig()), None) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_rope_destroy(None) == tk.ERR_INVALID_ARG
    assert tk.lib.thinK_rope_frequency(None, 0) == -1.0
    for kw in (dict(D=256, rot_dim=256), dict(D=8, rot_dim=2), dict(D=4, rot_dim=4, dtype=1), dict(theta=1.0)):
        st, h = rope_of(tk, **kw)
        assert st == 0 and tk.lib.thinK_rope_frequency(h, 0) == 1.0
        assert tk.lib.thinK_rope_frequency(h, -1) == tk.lib.thinK_rope_frequency(h, kw.get("rot_dim", 128) // 2) == -1.0
        assert tk.lib.thinK_rope_destroy(h) == 0


@pytest.mark.parametrize("R,theta,trained,factor", [(128, 1e4, 4096, 8.0), (64, 5e5, 8192, 32.0), (20, 1e4, 2048, 1.0), (256, 1e6, 32768, 4.0)])
def test_rope_frequencies(tk, R, theta, trained, factor):  # noqa: F811
    """Against the formulas in fp64: 1e-13 is a thousand roundings."""
    def of(**kw):
        st, h = rope_of(tk, D=256, rot_dim=R, theta=theta, factor=factor, trained=trained, **kw)
        assert st == 0
        f = [tk.lib.thinK_rope_frequency(h, j) for j in range(R // 2)]
        tk.lib.thinK_rope_destroy(h)
        return f
    plain = [theta ** (-2.0 * j / R) for j in range(R // 2)]
    where = lambda turns: R * math.log(trained / (turns * 2 * math.pi)) / (2 * math.log(theta))  # noqa: E731
    low, high = max(math.floor(where(32.0)), 0), min(math.ceil(where(1.0)), R - 1)
    ramp = [min(1.0, max(0.0, (j - low) / max(high - low, 0.001))) for j in range(R // 2)]
    keep = [min(1.0, max(0.0, (trained * f / (2 * math.pi) - 1.0) / 3.0)) for f in plain]
    want = {tk.ROPE_PLAIN: plain, tk.ROPE_LINEAR: [f / factor for f in plain],
            tk.ROPE_NTK: [(theta * factor ** (R / (R - 2))) ** (-2.0 * j / R) for j in range(R // 2)],
            tk.ROPE_YARN: [f / factor * r + f * (1 - r) for f, r in zip(plain, ramp)],
            tk.ROPE_BANDS: [f / factor * (1 - k) + f * k for f, k in zip(plain, keep)]}
    for scaling, w in want.items():
        assert of(scaling=scaling) == pytest.approx(w, rel=1e-13, abs=0)
    for scaling, slow, fast in ((tk.ROPE_BANDS, 1.0, 4.0), (tk.ROPE_YARN, 1.0, 32.0)):
        assert of(scaling=scaling, slow=slow, fast=fast) == of(scaling=scaling)          # the defaults


def test_rope_apply_refusals(tk):  # noqa: F811
    st, h = rope_of(tk)
    assert st == 0
    B, S, L, N, K, D = 3, 5, 2, 8, 4, 128
    dq, dk = (S * L * N * D, L * N * D, N * D, D), (S * L * K * D, L * K * D, K * D, D)
    T = tk.Tensor5
    q, k, qo, ko = T(1 << 30, *dq), T(1 << 31, *dk), T(1 << 32, *dq), T(1 << 33, *dk)

    def call(q=q, k=k, qo=qo, ko=ko, B=B, S=S, L=L, N=N, K=K, pos=4096, stride=0, rows=None, transpose=0, h=h):
        return tk.lib.thinK_rope_apply(h, q, k, qo, ko, B, S, L, N, K, pos, stride, rows, transpose, None)
    none = T()
    for kw in (dict(B=0), dict(S=0), dict(L=0), dict(N=0, K=0)):          # nothing to do
        assert call(q=none, k=none, qo=none, ko=none, pos=None, **kw) == 0
    bad = [dict(h=None), dict(B=-1), dict(S=-1), dict(L=-1), dict(N=-1), dict(K=-1), dict(transpose=2), dict(transpose=-1), dict(pos=None), dict(pos=4098),
           dict(rows=4097), dict(stride=-1), dict(stride=S - 1), dict(q=none), dict(k=none), dict(qo=none), dict(ko=none)]
    bad += [dict(q=T((1 << 30) + 8, *dq)), dict(k=T(1 << 31, dk[0], dk[1], dk[2], D + 4)), dict(qo=T(1 << 32, -dq[0], *dq[1:])),
            dict(ko=T(1 << 33, dk[0], dk[1], dk[2], D + 1))]
    # results that share memory: rows with one another, with queries, with keys, with the other result
    bad += [dict(qo=T(1 << 32, 0, *dq[1:])), dict(ko=T(1 << 33, dk[0], dk[1], dk[2], D - 8)), dict(qo=T((1 << 30) + 16, *dq)),
            dict(qo=T(1 << 31, *dq)), dict(ko=T(1 << 30, *dk)), dict(qo=T(1 << 33, *dq)), dict(ko=T((1 << 32) + (B * dq[0] - D) * 2, *dk)),
            dict(qo=T(1 << 30, dq[0], dq[1], dq[2] // 2, D)), dict(q=T(1 << 30, 0, *dq[1:]), qo=T(1 << 30, 0, *dq[1:]))]
    for kw in bad:
        assert call(**kw) == tk.ERR_INVALID_ARG, kw
    assert call(L=1 << 20, q=T(1 << 30, 0, 0, 0, 0), N=32, K=0, B=1, S=1, qo=T(1 << 32, 0, 0, 32 * D, D)) == tk.ERR_UNSUPPORTED
    tk.lib.thinK_rope_destroy(h)


def test_rope_binding_refusals(tk):  # noqa: F811
    r = tk.Rope(128, torch.bfloat16)
    x, pos = torch.zeros(2, 3, 1, 4, 128, dtype=torch.bfloat16), torch.zeros(2, dtype=torch.int32)
    for args, kw in (((x, None, pos), {}), ((None, None, pos), {}), ((x, None, pos), dict(k_out=x)), ((None, x, pos), dict(q_out=x))):
        with pytest.raises(tk.ThinKError) as e:
            r.apply(*args, **kw)
        assert e.value.status == tk.ERR_INVALID_ARG
    with pytest.raises(tk.ThinKError):
        tk.Rope(100, torch.bfloat16)
    for B, n in ((0, 4), (1 << 13, 4), (4, 0), (4, (1 << 30) + 1)):
        with pytest.raises(tk.ThinKError):
            tk.PagePlan(B, n, device="cpu")
