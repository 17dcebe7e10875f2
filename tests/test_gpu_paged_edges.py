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


# ---------------------------------------------------------------------------
# destinations of the read-back
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_read_refuses_destinations_that_share_memory(fmt, dtype):
    tk = binding()
    lens = [70, 33]
    p = Paged(fmt, dtype, lens, L=2, N_kv=2, G=2)
    k, v = p.rows(3)
    p.cache.write(k, v, p.table, rows=p.seq)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)

    def refused(a, b):
        with pytest.raises(tk.ThinKError) as e:
            p.cache.read(a, b, p.table, rows=p.seq)
        assert e.value.status == tk.ERR_INVALID_ARG

    one = torch.zeros(2, 70, 2, 2, 128, dtype=dtype, device="cuda")
    refused(one, one)                                             # the same rows for keys and values
    refused(one[:, :1].expand_as(one), vo)                        # one row for all tokens
    refused(ko, one[:, :, :1].expand_as(one))                     # for all layers
    refused(one[:1].expand_as(one), vo)                           # for all sequences
    refused(one[:, :, :, :1].expand_as(one), vo)                  # for all heads
    mem = torch.zeros(2 * one.numel(), dtype=dtype, device="cuda")
    refused(mem.as_strided(one.shape, (70 * 512, 512, 256, 120, 1)), vo)            # rows that run into one another
    refused(mem.as_strided(one.shape, (69 * 512, 512, 256, 128, 1)), vo)            # sequences that do
    half = one.numel() - 512
    refused(mem[:one.numel()].view_as(one), mem[half:half + one.numel()].view_as(one))
    assert not (ko.any() or vo.any() or one.any() or mem.any()) and p.cache.device_error() == 0
    # disjoint views of one buffer
    p.cache.read(ko, vo, p.table, rows=p.seq)
    want = torch.cat([ko, vo], -1)
    wide = torch.zeros(2, 70, 2, 2, 256, dtype=dtype, device="cuda")
    p.cache.read(wide[..., :128], wide[..., 128:], p.table, rows=p.seq)
    assert torch.equal(wide, want)
    wide = torch.zeros(2, 2, 2, 2, 70, 128, dtype=dtype, device="cuda")             # [b][key, value][layer][head][token]
    a, b = (wide[:, i].permute(0, 3, 1, 2, 4) for i in (0, 1))
    p.cache.read(a, b, p.table, rows=p.seq)
    assert torch.equal(a, ko) and torch.equal(b, vo)
    wide = torch.zeros(2, 2, 2, 70, 2, 128, dtype=dtype, device="cuda")             # different orders within a sequence
    a, b = wide[:, 0].permute(0, 2, 1, 3, 4), wide[:, 1].view(2, 70, 2, 2, 128)
    p.cache.read(a, b, p.table, rows=p.seq)
    assert torch.equal(a, ko) and torch.equal(b, vo)
    # an index of one value may have any stride
    k1, v1 = torch.zeros_like(k[:1, :, :1]), torch.zeros_like(v[:1, :, :1])
    p.cache.read(k1.as_strided(k1.shape, (0, 256, 0, 128, 1)), v1.as_strided(v1.shape, (8, 256, 8, 128, 1)), p.table, rows=p.seq, nlayers=1)
    assert torch.equal(k1, ko[:1, :, :1]) and torch.equal(v1, vo[:1, :, :1])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=IDS[:2])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_infinite_values(dtype, D):
    """A plain page may hold infinities.  A value of +-infinity with a weight makes its channel +-infinity, both signs a
    NaN, and no other channel sees it; behind the sequence's end it counts nothing."""
    lens = [1, 2, 63, 70, 3000]
    p = Paged("plain", dtype, [n + 1 for n in lens], N_kv=2, G=4, D=D)
    k, v = p.rows(19)
    inf = float("inf")
    for b, n in enumerate(lens):
        v[b, n // 2, 0, 0, 3] = inf
        v[b, n // 2, 0, 0, 9] = -inf
        v[b, 0, 0, 0, 17], v[b, n - 1, 0, 0, 17] = inf, -inf
        v[b, n] = inf
    p.cache.write(k, v, p.table)
    q = (0.1 * torch.randn(len(lens), 1, 8, D, generator=gen(23), device="cuda")).to(dtype)
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    out, lse = p.cache.decode_attn(q, p.table, seq, return_lse=True)
    mine = out[:, 0, :4].float()
    assert (mine[..., 3] == inf).all() and (mine[..., 9] == -inf).all()
    assert torch.isnan(mine[1:, :, 17]).all() and (mine[0, :, 17] == -inf).all()
    # the rest as without them (the oracle reads the pool: put finite values there)
    keep = [c for c in range(D) if c not in (3, 9, 17)]
    v = torch.where(torch.isfinite(v), v, torch.ones_like(v))
    p.cache.write(k, v, p.table)
    want = p.cache.decode_attn(q, p.table, seq)
    assert torch.equal(out[:, :, :4][..., keep], want[:, :, :4][..., keep]) and torch.equal(out[:, :, 4:], want[:, :, 4:])
    p.check(q, want, lse, lens=lens)
