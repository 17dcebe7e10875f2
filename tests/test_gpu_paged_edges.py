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


# ---------------------------------------------------------------------------
# attention: values, scales and logits at the ends of their ranges
# ---------------------------------------------------------------------------
def own_bounds(out, lse, sizes, n, D, dtype, same_keys=False, floor=1e-30):
    """As test_gpu_paged.bounds, but every channel by its own magnitudes (absv): a weight times its value's scale is kept
    as a pair of bf16, the first cut (2^-7 left at most), the second to the nearest (2^-9 of that), 2^-16 in all, plus
    2^-23 that the second is raised by.  Weights below 2^-117 of the largest may vanish.  Equal keys have equal logits,
    whatever their rounding: the weights are then exact up to exp2."""
    u = 2.0 ** -23
    delta = (D + 4) * u * sizes["qk"] + (2.0 ** -39 * sizes["q_max"] if dtype == torch.bfloat16 else 0.0)
    weights = (0.0 if same_keys else 2 * delta) + 2.0 ** -21 + (2.0 ** -16 + u if dtype == torch.bfloat16 else 0.0) + 2 * (n + 8) * u
    tol = torch.finfo(dtype).eps / 2 * np.abs(out) + np.reshape(weights, (-1, 1)) * sizes["absv"] * (1 + 2.0 ** -7) + floor
    ltol = delta + (n + 8) * u + 2.0 ** -21 + 4 * u * np.abs(np.where(np.isfinite(lse), lse, 0.0))
    return tol, ltol


def check_own(p, q, out, lse, same_keys=False, floor=lambda b: 1e-30):
    q64, o64, l64 = (x.double().cpu().numpy() for x in (q, out, lse))
    for b in range(q.shape[0]):
        for l in range(p.L):
            for h in range(p.N_kv):
                hs = slice(h * p.G, (h + 1) * p.G)
                k, v = p.stored(b, l, h, p.lens[b])
                r = po.attention(q64[b, l, hs], k, v, p.scale)
                tol, ltol = own_bounds(*r, p.lens[b], p.D, p.dtype, same_keys, floor(b))
                err, e = np.abs(o64[b, l, hs] - r[0]), np.abs(l64[b, l, hs] - r[1])
                assert (err <= tol).all(), f"{(b, l, hs)}: {(err / tol).max():.3g} of the bound at channel {(err / tol).max(0).argmax()}"
                assert (e <= ltol).all(), f"lse {(b, l, hs)}: {e.max():.3g} > {ltol.min():.3g}"


@pytest.mark.parametrize("fmt", ["plain", "e4m3", "int4"])
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("power", [10, 20, 30, 45, 60])
def test_attention_channels_far_apart(fmt, D, power):
    """Value channels whose magnitudes differ by 2^10 to 2^60 in a row (4 bits: its groups), and one token that is
    2^power larger than all others, in its first channel alone: the other channels keep their share."""
    p = Paged(fmt, torch.bfloat16, [200, 200, 3000], N_kv=2, G=3, D=D)
    k, v = p.rows(7)
    v = v.float()
    if fmt != "e4m3":                                 # (an e4m3 row has one scale: such channels would be stored as zeros)
        v[0, :, :, :, 32:64] *= 2.0 ** -power
    v[1, 90, :, :, 1:] = 0
    v[1, 90, :, :, 0] = 2.0 ** power
    v[2, 1700, :, :, 1:] = 0
    v[2, 1700, :, :, 0] = -(2.0 ** power)
    p.cache.write(k, v.bfloat16(), p.table, rows=p.seq)
    q = torch.randn(3, 1, 6, D, generator=gen(11), device="cuda").bfloat16()
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    check_own(p, q, out, lse)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("power", [0, 8, 16, 24, 40])
def test_attention_large_logits_of_equal_keys(fmt, dtype, power):
    """Logits of any size, the same for every token of a sequence (one token's is): the output is the mean of the values,
    whatever a logit's rounding is."""
    lens = [1, 1, 2, 40, 300, 5000]
    p = Paged(fmt, dtype, lens, N_kv=2, G=4)
    k, v = p.rows(13)
    k = k[:, :1].expand_as(k)
    mags = 2.0 ** torch.randint(-20, 21, v.shape[:4] + (1,), generator=gen(37), device="cuda").float()
    v = (v.float() * mags).to(dtype)
    p.cache.write(k, v, p.table, rows=p.seq)
    q = (torch.randn(len(lens), 1, 8, 128, generator=gen(17), device="cuda") * 2.0 ** power).to(dtype)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    check_own(p, q, out, lse, same_keys=True)


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32], ids=IDS[:2])
@pytest.mark.parametrize("D", [64, 128])
def test_attention_logits_of_minus_infinity(dtype, D):
    """Keys of -infinity.  A sequence whose every logit is -infinity has no softmax: NaN, not the zeros of a sequence
    without tokens (the sum's logarithm is -infinity for both); one finite logit takes all of the weight."""
    inf = float("inf")
    lens = [1, 70, 5000, 1, 70, 5000, 0]
    p = Paged("plain", dtype, lens, N_kv=2, G=4, D=D)
    k, v = p.rows(29)
    k[:, :, :, 0, 5] = -inf
    last = [n - 1 for n in lens]
    for b in (3, 4, 5):
        k[b, last[b], 0, 0, 5] = 1
    p.cache.write(k, v, p.table, rows=p.seq)
    q = torch.randn(len(lens), 1, 8, D, generator=gen(31), device="cuda").to(dtype)
    q[..., 5] = q[..., 5].abs() + 1
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    assert torch.isnan(out[:3, 0, :4]).all() and torch.isneginf(lse[:3, 0, :4]).all()
    assert (out[6] == 0).all() and torch.isneginf(lse[6]).all()
    for b in (3, 4, 5):
        assert torch.equal(out[b, 0, :4], v[b, last[b], 0, 0].expand(4, D)) and torch.isfinite(lse[b]).all()
    p.check(q, out, lse, units={(b, 0, 1) for b in range(6)})


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("q_pow,k_pow,scale", [(-120, 120, 0.0), (-90, 91, 0.0), (-100, 118, 2.0 ** -20), (110, -109, 0.0), (60, -80, 2.0 ** 20)])
def test_attention_tiny_queries_and_huge_keys(fmt, dtype, q_pow, k_pow, scale):
    """Queries and keys at opposite ends of the exponent range, logits of ordinary size."""
    p = Paged(fmt, dtype, [1, 150], N_kv=2, G=4, scale=scale)
    k, v = p.rows(43, outliers=False)
    p.cache.write((k.float() * 2.0 ** k_pow).to(dtype), v, p.table, rows=p.seq)
    q = (torch.randn(2, 1, 8, 128, generator=gen(47), device="cuda") * 2.0 ** q_pow).to(dtype)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    assert (lse[0].abs() > 2.0 ** -8).all()
    p.check(q, out, lse)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("power", [-104, -112, -120, -126])
def test_attention_tiny_values(fmt, dtype, power):
    """Values down to the smallest ordinary numbers: outputs are as exact as those of any size, up to half a step of
    bf16's smallest numbers where all of a sequence's values are tiny.  Sequences 1 and 2 hold one token of ordinary values that has next to no weight, in front
    of all others and behind them; sequences 3 and 5 one that has weight."""
    p = Paged(fmt, dtype, [1, 300, 300, 300, 5000, 5000], N_kv=2, G=4)
    k, v = p.rows(83)
    v = v.float() * 2.0 ** power
    q = torch.randn(6, 1, 8, 128, generator=gen(89), device="cuda").to(dtype)
    for b, t, like in ((1, 0, -4.0), (2, 299, -4.0), (3, 150, 0.5), (5, 2600, 0.0)):
        v[b, t] = torch.randn(1, 2, 128, generator=gen(91), device="cuda")
        k[b, t, 0] = (like * q[b, 0].view(2, 4, 128).float().sum(1)).to(dtype)
    p.cache.write(k, v.to(dtype), p.table, rows=p.seq)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    # Half a step of the smallest outputs; fp32 sums of numbers below 2^-126 miss half of 2^-149 a token, weights (and so
    # the sums) may be 2^-8 of what they are divided by.  Beside the ordinary token of those sequences (which flips the
    # reference of the weights) a token's weight * scale may be below 2^-117: a pair of bf16 then misses up to 2^-133 of
    # it, times its code (448 or 7 at most), divided by a sum of 2^-8 at least: 2^-125 code a token.  That shows in
    # channels in which the ordinary token's code is 0, and absv with it of the tiny ones' size.
    half, code = (2.0 ** -134 if dtype == torch.bfloat16 else 2.0 ** -150), {"plain": 0.0, "e4m3": 448.0, "int4": 7.0}[fmt]

    def floor(b):
        return half + p.lens[b] * (2.0 ** -142 + (code * 2.0 ** -125 if b in (1, 2, 3, 5) else 0.0))

    check_own(p, q, out, lse, floor=floor)


@pytest.mark.parametrize("byte", [0, 1, 254, 255])
@pytest.mark.parametrize("D", [64, 128])
def test_scale_bytes_at_the_ends(byte, D):
    """Scale bytes 0 (2^-127) and 255 (NaN) are never written, but mean the same to attention as to the read-back, as the
    ends of the ordinary range do."""
    tk = binding()
    p = Paged("e4m3", torch.bfloat16, [1, 1, 70, 70], N_kv=2, G=3, D=D)
    k, v = p.rows(41)
    k[:2] *= 2.0 ** -6                                # codes far below 448: 2^127 times them stays in range
    v[:2] *= 2.0 ** -6
    p.cache.write(k, v, p.table, rows=p.seq)

    def patch(b, tok, part):
        page = int(p.table_cpu[b, tok // PAGE])
        at = tk.paged_offset(p.cfg, 0, page, 0, tok % PAGE, part)
        p.pool[at] = byte
        if byte == 254:                               # codes that 2^127 keeps in bf16's range
            row = tk.paged_offset(p.cfg, 0, page, 0, tok % PAGE, part - 2)
            p.pool[row:row + D] = torch.tensor([0x38, 0xb8, 0x08, 0x00], dtype=torch.uint8, device="cuda").repeat(D // 4)

    patch(0, 0, tk.PART_V_SCALE)
    patch(1, 0, tk.PART_K_SCALE)
    patch(2, 66, tk.PART_V_SCALE)
    patch(3, 5, tk.PART_K_SCALE)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    p.cache.read(ko, vo, p.table, rows=p.seq)
    small = byte >= 254                               # queries that bring the patched keys' logits to order 1
    q = torch.randn(4, 1, 6, D, generator=gen(43), device="cuda")
    q[1] *= 2.0 ** (-125 if small else 110)
    q[3] *= 2.0 ** (-125 if small else 0)
    q = q.bfloat16()
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    if byte == 255:
        assert torch.isnan(vo[0, 0, 0, 0]).all() and torch.isnan(ko[1, 0, 0, 0]).all()
        assert torch.isnan(out[[0, 1, 2, 3], 0, :3]).all()
        assert torch.isnan(lse[[1, 3], 0, :3]).all() and torch.isfinite(lse[[0, 2]]).all()
    else:
        assert torch.isfinite(out).all() and torch.isfinite(lse).all()
        # the only token's value as it is read back
        assert torch.equal(out[0, 0, :3], vo[0, 0, 0, 0].expand(3, D)) and out[0, 0, :3].abs().sum() > 0
        q64 = q.double().cpu().numpy()
        for b in (1, 3):
            kk, vv = p.stored(b, 0, 0, p.lens[b])
            r = po.attention(q64[b, 0, :3], kk, vv, p.scale)
            tol, ltol = bounds(*r, p.lens[b], D, "e4m3", torch.bfloat16)
            assert (np.abs(out[b, 0, :3].double().cpu().numpy() - r[0]) <= tol).all()
            assert (np.abs(lse[b, 0, :3].double().cpu().numpy() - r[1]) <= ltol).all()
            if b == 1:
                assert (lse[b, 0, :3].abs() > 2.0 ** -20).all()
    other = slice(3, 6)
    q0 = q[:, :, other]
    for b in range(4):
        kk, vv = p.stored(b, 0, 1, p.lens[b])
        r = po.attention(q0[b, 0].double().cpu().numpy(), kk, vv, p.scale)
        tol, _ = bounds(*r, p.lens[b], D, "e4m3", torch.bfloat16)
        assert (np.abs(out[b, 0, other].double().cpu().numpy() - r[0]) <= tol).all()


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("power", [-110, 0, 100])
def test_log_sums_of_equal_logits(fmt, dtype, power):
    """Logits of zero: the logarithm of the sum is that of the length, whatever weights are relative to (which goes by the
    values).  The sums are exact; log2 of a number between 1 and 2 is off by 2^-23 at most, the sum with its exponent and
    the product with ln 2 by half a step each, ln 2 itself by 2^-25: 2 u |lse| + u."""
    lens = [1, 2, 3, 5, 7, 11, 100, 300, 5000, 12345]
    p = Paged(fmt, dtype, lens, N_kv=1, G=4)
    k, v = p.rows(83)
    p.cache.write(k, (v.float() * 2.0 ** power).to(dtype), p.table, rows=p.seq)
    q = torch.zeros(len(lens), 1, 4, 128, dtype=dtype, device="cuda")
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    want = np.log(np.array(lens, dtype=np.float64)).reshape(-1, 1, 1)
    u = 2.0 ** -23
    err = np.abs(lse.double().cpu().numpy() - want)
    assert (err <= 2 * u * want + u).all(), f"{(err / (2 * u * want + u)).max():.3g} of the bound"


# ---------------------------------------------------------------------------
# streams
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("by_argument", [True, False], ids=["argument", "current"])
def test_a_cache_may_be_dropped_while_another_stream_uses_it(by_argument):
    """The memory that a cache allocated is not handed out again before the calls on all of its streams are done."""
    tk = binding()
    lens = [9000, 5000]
    cfg = tk.make_paged_config(1, 8, 2, 128, 232, 2, torch.bfloat16, tk.PAGE_PLAIN)
    table = torch.full((2, 150), -1, dtype=torch.int32, device="cuda")
    table[0, :141] = torch.arange(141, dtype=torch.int32, device="cuda")
    table[1, :79] = torch.arange(141, 220, dtype=torch.int32, device="cuda")
    seq = torch.tensor(lens, dtype=torch.int32, device="cuda")
    g = gen(3)
    k = torch.randn(2, 9000, 1, 2, 128, generator=g, device="cuda").bfloat16()
    v = torch.randn(2, 9000, 1, 2, 128, generator=g, device="cuda").bfloat16()
    q = torch.randn(2, 1, 8, 128, generator=g, device="cuda").bfloat16()
    ref = tk.PagedKVCache(cfg)
    ref.write(k, v, table, rows=seq)
    want = ref.decode_attn(q, table, seq)
    cache = tk.PagedKVCache(cfg)
    cache.write(k, v, table, rows=seq)
    out = torch.zeros_like(q)
    sizes = (cache.pages.numel(), cache.workspace.numel())
    side = torch.cuda.Stream()
    torch.full((16,), 85, dtype=torch.uint8, device="cuda")        # (a kernel's first use may wait for the device)
    torch.cuda.synchronize()
    with torch.cuda.stream(side):
        torch.cuda._sleep(1_000_000_000)              # about 0.6 s: the call is still waiting when the cache goes
    if by_argument:
        cache.decode_attn(q, table, seq, out=out, stream=side)
    else:
        with torch.cuda.stream(side):
            cache.decode_attn(q, table, seq, out=out)
    cache.close()
    del cache
    taken = [torch.full((n,), 85, dtype=torch.uint8, device="cuda") for n in sizes for _ in range(2)]
    torch.cuda.synchronize()
    assert torch.equal(out, want) and len(taken) == 4


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_one_layer_of_one_sequence(fmt, dtype):
    """A call over a single layer of a single sequence out of a larger cache, against the oracle."""
    p = Paged(fmt, dtype, [100, 260], L=3, N_kv=2, G=2, D=64, scale=0.31, max_batch=5)
    k, v = p.rows(23)
    p.cache.write(k, v, p.table, rows=p.seq)
    q = torch.randn(2, 3, 4, 64, generator=gen(29), device="cuda").to(dtype)
    for b in range(2):
        for l in range(3):
            out, lse = p.cache.decode_attn(q[b:b + 1, l:l + 1].contiguous(), p.table[b:], p.seq[b:], layer0=l, nlayers=1, return_lse=True)
            for h in range(2):
                hs = slice(2 * h, 2 * h + 2)
                r = po.attention(q[b, l, hs].double().cpu().numpy(), *p.stored(b, l, h, p.lens[b]), 0.31)
                tol, ltol = bounds(*r, p.lens[b], 64, fmt, dtype)
                assert (np.abs(out[0, 0, hs].double().cpu().numpy() - r[0]) <= tol).all()
                assert (np.abs(lse[0, 0, hs].double().cpu().numpy() - r[1]) <= ltol).all()
    assert p.cache.device_error() == 0
