"""GPU tests of the paged key-value cache at the edges of what its documentation allows: buffers shared between caches,
values and logits at the ends of their ranges, destinations, streams.  Oracle and harness are test_gpu_paged's."""
import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from test_gpu_paged import FMT, IDS, KINDS, PAGE, Paged, binding, bounds, gen

pytestmark = pytest.mark.gpu


# ---------------------------------------------------------------------------
# one scratch buffer, several caches
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("d_small,d_large", [(128, 64), (64, 128), (128, 128), (64, 64)])
def test_one_scratch_for_caches_of_different_shapes(d_small, d_large):
    """Two caches (bf16 and 4-bit layers, say) that take turns on one scratch buffer; all of their sequences are split
    over CTAs, so each call leaves partial states and tickets in it."""
    bf16 = torch.bfloat16
    small = Paged("plain", bf16, [20000], N_kv=1, G=4, D=d_small)
    large = Paged("int4", bf16, [130] * 60 + [3000, 5000, 700, 9000], L=3, N_kv=8, G=2, D=d_large, max_batch=64)
    scratch = torch.zeros(max(int(p.cache.sizes.workspace) for p in (small, large)), dtype=torch.uint8, device="cuda")
    calls = []
    for p in (small, large):
        k, v = p.rows(3)
        p.cache.write(k, v, p.table, rows=p.seq)
        q = torch.randn(len(p.lens), p.L, p.N_kv * p.G, p.D, generator=gen(5), device="cuda").to(bf16)
        calls.append((p, q) + p.cache.decode_attn(q, p.table, p.seq, return_lse=True))
    for i in (0, 1, 0, 0, 1, 1, 0, 1):
        p, q, want, wlse = calls[i]
        out, lse = torch.full_like(want, float("nan")), torch.full_like(wlse, float("nan"))
        p.cache.decode_attn(q, p.table, p.seq, out=out, lse=lse, scratch=scratch)
        assert torch.equal(out, want) and torch.equal(lse, wlse)
    # a cache's own workspace is such a buffer too
    if large.cache.sizes.workspace >= small.cache.sizes.workspace:
        p, q, want, _ = calls[0]
        assert torch.equal(p.cache.decode_attn(q, p.table, p.seq, scratch=large.cache.workspace), want)
        p, q, want, _ = calls[1]
        assert torch.equal(p.cache.decode_attn(q, p.table, p.seq), want)
    assert small.cache.device_error() == 0 and large.cache.device_error() == 0
