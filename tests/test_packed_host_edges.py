"""CPU checks of packed batches where a call or a kernel goes wrong: what the host side of an entry point answers, and what a
kernel may trust."""
import ctypes as C
import os
import subprocess

import pytest

from test_packed_host import FAKE
from test_paged_host import ROOT, compile_and_run, tk  # noqa: F401


def test_descriptors_that_nobody_wrote(tmp_path):
    """The join of cut items takes a descriptor for an item only if its sequence, its layer and head and its number exist: random
    bytes and the values next to every limit."""
    out = compile_and_run(tmp_path, r"""
#include <stdio.h>
#include <string.h>
#include <random>
#include "paged_prompt.h"
using namespace think;
int main() {
  std::mt19937_64 g(1);
  long bad = 0, taken = 0;
  auto check = [&](const PromptDesc& d, int B, int heads) {
    const bool in = d.begins && 0 <= d.b && d.b < B && 0 <= d.lh && d.lh < heads && 0 <= d.item;
    bad += d.names_item(B, heads) != in;
    taken += in;
  };
  for (int it = 0; it < 300000; ++it) {
    PromptDesc d;
    uint32_t w[sizeof(d) / 4];
    for (uint32_t& x : w) x = (uint32_t)g();
    memcpy((void*)&d, w, sizeof(d));
    const int B = 1 + (int)(g() % 4096), heads = 1 + (int)(g() % 1000);
    check(d, B, heads);
    for (int b : {-1, 0, B - 1, B}) for (int lh : {-1, 0, heads - 1, heads}) for (int item : {-2147483647 - 1, -1, 0, 2147483647})
      for (int16_t begins : {0, 1, -1}) check(PromptDesc{lh, b, item, begins, d.carries}, B, heads);
    bad += PromptDesc{0, 0, 0, 0, 0}.names_item(B, heads);
  }
  // an item's number against the sequence's: none of a sequence without rows, and what numbers stand for stays within rows
  for (int rows = 0; rows < 600; ++rows)
    for (int per : {1, 7, 64, 256}) {
      const int items = PromptLine{0, rows, per}.items();
      bad += rows == 0 ? items != 0 : (items - 1) * per >= rows || items * per < rows;
    }
  bad += PromptLine{0, 2147483647, 1}.items() != 2147483647;
  printf("%ld %d\n", bad, taken > 1000);
}
""")
    assert out.split() == ["0", "1"]


def test_scale_of_the_logits(tmp_path):
    """The power of two on the queries times what is left on the logits is the scale, at every exponent; what is left is never 0 and
    is 1 to 2 wherever the scale is below 1 and has an exponent of fp32."""
    out = compile_and_run(tmp_path, r"""
#include <stdio.h>
#include "paged_prompt.h"
using namespace think;
int main() {
  long bad = 0;
  for (int e = -1074; e <= 127; ++e)
    for (double f : {1.0, 1.25, 1.9999}) {
      const double x = ldexp(f, e);
      if (x == 0 || x > 3.4e38) continue;
      const PromptScale s(x);
      bad += s.queries > 0 || s.queries < -126 || !(s.logits >= 1.17549435e-38f) || s.logits > 3.4028235e38f;
      if (e >= -126) bad += fabs(ldexp((double)s.logits, s.queries) / x - 1) > ldexp(1, -24);
      if (e >= -126 && e < 0) bad += s.logits < 1 || s.logits >= 2.0001f || s.queries != e;
      if (e >= 0) bad += s.queries != 0;
    }
  printf("%ld\n", bad);
}
""")
    assert out.split() == ["0"]


@pytest.mark.parametrize("broken", ["setup", "map"])
@pytest.mark.parametrize("dtype,fmt", [(0, 0), (0, 1), (0, 2), (1, 0)])
def test_a_cache_without_prompt_attention(tk, tmp_path, broken, dtype, fmt):  # noqa: F811
    """Where the attention's kernel or the map of the pool cannot be set up, that call alone is refused."""
    fake = FAKE.replace("paged_prompt_setup(int, int, int) { return cudaSuccess; }", "paged_prompt_setup(int, int, int) { return cudaErrorLaunchOutOfResources; }"
                        ) if broken == "setup" else FAKE.replace("return CUDA_SUCCESS; }", "return CUDA_ERROR_INVALID_VALUE; }")
    assert fake != FAKE
    (tmp_path / "fake.cpp").write_text("#include <cuda.h>\n" + fake)
    csrc, so = os.path.join(ROOT, "paper_2407_21018_b200", "csrc"), str(tmp_path / "fake.so")
    subprocess.run(["g++", "-std=c++17", "-O1", "-shared", "-fPIC", "-Wl,-Bsymbolic", "-I", os.path.join(ROOT, "include"), "-I", csrc,
                    "-I", "/usr/local/cuda/include", "-x", "c++", os.path.join(csrc, "paged_api.cu"), str(tmp_path / "fake.cpp"), "-o", so],
                   check=True, capture_output=True)
    lib = C.CDLL(so)
    for name in ("thinK_paged_bytes", "thinK_paged_create", "thinK_paged_write", "thinK_paged_decode_attn", "thinK_paged_prompt_attn",
                 "thinK_paged_prompt_scratch"):
        real = getattr(tk.lib, name)
        getattr(lib, name).argtypes, getattr(lib, name).restype = real.argtypes, real.restype
    cfg, need, h = tk.make_paged_config(2, 8, 4, 128, 10, 8, dtype, fmt), tk.PagedSizes(), C.c_void_p()
    assert lib.thinK_paged_bytes(C.byref(cfg), C.byref(need)) == 0
    assert lib.thinK_paged_create(C.byref(cfg), C.byref(need), 1 << 40, 1 << 41, C.byref(h)) == 0
    rows, table = tk.Tensor5(1 << 30, 4096, 1024, 512, 128), tk.PageTable(4096, 4, 4, 3)
    assert lib.thinK_paged_write(h, rows, tk.Tensor5(1 << 31, 4096, 1024, 512, 128), table, None, None, 4, 0, 2, None) == 0
    assert lib.thinK_paged_decode_attn(h, 1 << 30, 1 << 31, None, table, 4096, None, 0, 0, 2, None) == 0
    q, out = tk.Tensor5(1 << 30, 4 * 2048, 2048, 1024, 128), tk.Tensor5(1 << 31, 4 * 2048, 2048, 1024, 128)
    refused = broken == "setup" or (dtype, fmt) == (0, 0)         # (only bf16 pages of plain rows have a map)
    assert lib.thinK_paged_prompt_attn(h, q, out, None, table, None, None, None, 4, 1 << 34, lib.thinK_paged_prompt_scratch(h), 0, 2, None) == (
        tk.ERR_UNSUPPORTED if refused else 0)
