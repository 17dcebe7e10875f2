"""GPU tests of the paged key-value cache against the fp64 oracle: stored bytes and read-back bit-exact, attention
within bounds that are derived from the kernels' roundings (see `bounds`)."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from paper_2407_21018_b200 import workloads as wl

pytestmark = pytest.mark.gpu

FMT = {"plain": 0, "e4m3": 1, "int4": 2}
PAGE = 64
KINDS = [("plain", torch.bfloat16), ("plain", torch.float32), ("e4m3", torch.bfloat16), ("int4", torch.bfloat16)]
IDS = ["bf16", "f32", "e4m3", "int4"]


def binding():
    from paper_2407_21018_b200 import binding as tk
    return tk


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


class Paged:
    """A cache over a pool full of 0xff bytes (NaN in every format), with a shuffled page table whose entries behind
    a sequence's end are invalid."""

    def __init__(self, fmt, dtype, lens, L=1, N_kv=2, G=4, D=128, extra_pages=2, seed=0, scale=0.0, width=None, num_pages=None,
                 first_page=0, max_batch=None):
        tk = binding()
        self.fmt, self.dtype, self.lens, self.L, self.N_kv, self.G, self.D = fmt, dtype, list(lens), L, N_kv, G, D
        need = [-(-n // PAGE) for n in lens]
        self.width = width or max(1, max(need))
        used = sum(need)
        self.num_pages = num_pages or first_page + used + extra_pages
        self.cfg = tk.make_paged_config(L, N_kv * G, N_kv, D, self.num_pages, max_batch or max(1, len(lens)), dtype, FMT[fmt], scale)
        self.scale = scale or D ** -0.5
        sizes = tk.paged_bytes(self.cfg)
        if num_pages is None:
            self.pool = torch.full((int(sizes.pages),), 255, dtype=torch.uint8, device="cuda")
        else:
            self.pool = torch.empty((int(sizes.pages),), dtype=torch.uint8, device="cuda")
        self.cache = tk.PagedKVCache(self.cfg, pages=self.pool)
        order = first_page + torch.from_numpy(np.random.default_rng(seed).permutation(used + extra_pages)).to(torch.int32)
        table = torch.full((len(lens), self.width), -7, dtype=torch.int32)
        at = 0
        for b, n in enumerate(need):
            table[b, :n] = order[at:at + n]
            at += n
        self.table_cpu = table
        self.table = table.cuda()
        self.seq = torch.tensor(self.lens, dtype=torch.int32, device="cuda")

    def rows(self, seed, S=None, outliers=True):
        S = max(self.lens) if S is None else S
        g = gen(seed)
        k = torch.randn(len(self.lens), S, self.L, self.N_kv, self.D, generator=g, device="cuda")
        v = torch.randn(len(self.lens), S, self.L, self.N_kv, self.D, generator=g, device="cuda")
        if outliers:
            k[..., :3] *= 8
        return k.to(self.dtype), v.to(self.dtype)

    def block(self, l, page, h):
        n = int(binding().paged_bytes(self.cfg).block)
        o = ((l * self.num_pages + page) * self.N_kv + h) * n
        return self.pool[o:o + n].cpu().numpy()

    def parts(self, raw):
        e = 2 if self.dtype == torch.bfloat16 else 4
        row = {"plain": self.D * e, "e4m3": self.D, "int4": self.D // 2}[self.fmt]
        sc = {"plain": 0, "e4m3": 1, "int4": 2 * self.D // 32}[self.fmt]
        a, b = PAGE * row, PAGE * sc
        cut = lambda o, n: raw[o:o + n].reshape(PAGE, -1) if n else None  # noqa: E731
        return cut(0, a), cut(a, a), cut(2 * a, b), cut(2 * a + b, b)

    def stored(self, b, l, h, n):
        """The first n tokens of sequence b as the oracle reads the pool's bytes: (k, v) [n, D] in 64 bits."""
        ks, vs = [], []
        for j in range(-(-n // PAGE)):
            kc, vc, ksc, vsc = self.parts(self.block(l, int(self.table_cpu[b, j]), h))
            m = min(PAGE, n - j * PAGE)
            for out, c, s in ((ks, kc, ksc), (vs, vc, vsc)):
                if self.fmt == "plain":
                    t = torch.from_numpy(c[:m].copy()).view(self.dtype).double().numpy()
                    out.append(t)
                else:
                    out.append(np.stack([po.decode_row(c[i], s[i], self.fmt) for i in range(m)]))
        z = np.zeros((0, self.D))
        return (np.concatenate(ks) if ks else z), (np.concatenate(vs) if vs else z)

    def want(self, q, lens=None, units=None):
        """Oracle attention; yields (b, l, heads slice, out, lse, tol_out, tol_lse)."""
        lens = self.lens if lens is None else lens
        q64 = q.double().cpu().numpy()
        for b in range(q.shape[0]):
            for l in range(self.L):
                for h in range(self.N_kv):
                    if units is not None and (b, l, h) not in units:
                        continue
                    hs = slice(h * self.G, (h + 1) * self.G)
                    k, v = self.stored(b, l, h, lens[b])
                    r = po.attention(q64[b, l, hs], k, v, self.scale)
                    yield (b, l, hs, r[0], r[1]) + bounds(*r, lens[b], self.D, self.fmt, self.dtype)

    def check(self, q, out, lse=None, lens=None, units=None):
        o64 = out.double().cpu().numpy()
        l64 = None if lse is None else lse.double().cpu().numpy()
        worst = 0.0
        for b, l, hs, want, wlse, tol, ltol in self.want(q, lens, units):
            err = np.abs(o64[b, l, hs] - want)
            assert np.isfinite(o64[b, l, hs]).all(), (b, l, hs)
            assert (err <= tol).all(), f"{(b, l, hs)}: {(err / np.maximum(tol, 1e-300)).max():.3g} of the bound, max-abs {err.max():.3g}"
            worst = max(worst, float((err / np.maximum(tol, 1e-30)).max()))
            if l64 is not None:
                if np.isneginf(wlse).any():
                    assert np.isneginf(l64[b, l, hs]).all()
                else:
                    e = np.abs(l64[b, l, hs] - wlse)
                    assert (e <= ltol).all(), f"lse {(b, l, hs)}: {e.max():.3g} > {ltol.min():.3g}"
        return worst


def bounds(out, lse, sizes, n, D, fmt, dtype):
    """Error bounds of one head, first order in the roundings; the sizes are oracle.attention's.

    With u = 2^-23 (one fp32 operation, also where the tensor core's adder truncates):
      logit     a dot product of D terms whose magnitudes sum to qk: error <= (D + 4) u qk, the scale in base 2 and the
                maximum's subtraction included.  A weight exp(x) then carries twice that (its own and the
                denominator's) relative error, plus 2^-21 for exp2 and 2^-11 where weights are rounded to 16 bits.
      sums      n terms added in fp32 in any order: n u, numerator and denominator.
      16 bits   a 16-bit weight has a smallest step of 2^-24, with the largest weight * scale between 2^7 and 2^15:
                each token is off by at most 2^-32 of that product, whose codes are at most 448 (7) of a scale of
                which the row's largest value has at least 224 (7/2): 2^-31 of top.
      query     of quantised pages: f16 with the row's largest channel in [2^14, 2^15) and a smallest step of 2^-24, so
                a channel is off by at most 2^-39 of the largest: 2^-39 q_max.
    Weighted with |v| the weights' errors are relative to absv.  The output is rounded once to its type: half a step,
    finfo.eps / 2 relative."""
    u = 2.0 ** -23
    delta = (D + 4) * u * sizes["qk"]
    if fmt != "plain":
        delta = delta + 2.0 ** -39 * sizes["q_max"]
    weights = 2 * delta + 2.0 ** -21 + (2.0 ** -11 if dtype == torch.bfloat16 else 0.0) + 2 * (n + 8) * u
    tol = torch.finfo(dtype).eps / 2 * np.abs(out) + weights[:, None] * sizes["absv"] * (1 + 2.0 ** -7) + 1e-30
    if dtype == torch.bfloat16:
        tol = tol + n * 2.0 ** -31 * sizes["top"][:, None]
    ltol = delta + (n + 8) * u + 2.0 ** -21 + 4 * u * np.abs(np.where(np.isfinite(lse), lse, 0.0))
    return tol, ltol


# ---------------------------------------------------------------------------
# write and read
# ---------------------------------------------------------------------------
def expected_block_rows(p, x):
    """Oracle bytes of a row (codes, scales)."""
    if p.fmt == "plain":
        return x.cpu().contiguous().view(torch.uint8).numpy(), None
    return po.encode_row(x.double().cpu().numpy(), p.fmt)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("D,N_kv", [(128, 2), (64, 3), (128, 1)])
def test_write_is_bit_exact_and_read_reverses(fmt, dtype, D, N_kv):
    lens = [1, 64, 130, 0, 65]
    p = Paged(fmt, dtype, [n + 5 for n in lens], L=2, N_kv=N_kv, D=D)
    S = max(lens) + 3
    k, v = p.rows(3, S)
    rows = torch.tensor(lens, dtype=torch.int32, device="cuda")
    pos = torch.tensor([5, 0, 3, 1, 5], dtype=torch.int32, device="cuda")
    k[0, 0, 0, 0, :] = 0                              # an empty row
    k[1, 3, 0, 0, 7] = 2.0 ** -130                    # subnormal next to ordinary values
    k[1, 4, 0, 0, :] = 0
    k[1, 4, 0, 0, 5] = -(2.0 ** -133)                 # nothing but the smallest bf16
    v[2, 0, 1, 0, :] *= 2.0 ** 120                    # near the largest bf16
    v[2, 1, 1, 0, :] *= 2.0 ** -120
    k[1, 5, 1, 0, :] = 3.5                            # quotients that are ties
    before = p.pool.clone()
    kin = k.clone()
    for b, n in enumerate(lens):                      # rows that are not named are not looked at
        kin[b, n:] = float("nan")
    p.cache.write(kin, v, p.table, pos=pos, rows=rows)
    assert p.cache.device_error() == 0
    want = before.cpu().numpy()
    block = int(p.cache.sizes.block)
    for b, n in enumerate(lens):
        for s in range(n):
            t = int(pos[b]) + s
            page, slot = int(p.table_cpu[b, t // PAGE]), t % PAGE
            for l in range(2):
                for h in range(N_kv):
                    o = ((l * p.num_pages + page) * N_kv + h) * block
                    parts = p.parts(want[o:o + block])
                    for x, c, z in ((k, parts[0], parts[2]), (v, parts[1], parts[3])):
                        codes, scales = expected_block_rows(p, x[b, s, l, h])
                        c[slot] = codes
                        if z is not None:
                            z[slot] = scales
    got = p.pool.cpu().numpy()
    assert np.array_equal(got, want), f"{int((got != want).sum())} bytes differ"
    # read back into views with NaN around: named rows only
    ko, vo = torch.full_like(k, float("nan")), torch.full_like(v, float("nan"))
    p.cache.read(ko, vo, p.table, pos=pos, rows=rows)
    assert p.cache.device_error() == 0
    for b, n in enumerate(lens):
        assert torch.isnan(ko[b, n:]).all() and torch.isnan(vo[b, n:]).all()
        for s in range(n):
            for l in range(2):
                for h in range(N_kv):
                    for x, y in ((k, ko), (v, vo)):
                        if fmt == "plain":
                            assert torch.equal(x[b, s, l, h], y[b, s, l, h])
                        else:
                            w = torch.from_numpy(po.decode_row(*po.encode_row(x[b, s, l, h].double().cpu().numpy(), fmt), fmt))
                            w = torch.from_numpy(po.round_bf16(w.numpy()))
                            assert torch.equal(w, y[b, s, l, h].double().cpu()), (b, s, l, h)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_write_strided_views_layers_and_defaults(fmt, dtype):
    """Heads-first views, a layer range, no pos and no rows; the layers outside stay as they were."""
    p = Paged(fmt, dtype, [70, 70], L=4, N_kv=2, D=64)
    k, v = p.rows(5)
    other = Paged(fmt, dtype, [70, 70], L=4, N_kv=2, D=64)
    other.cache.write(k, v, other.table)
    hk = k[:, :, 1:3].permute(0, 3, 2, 1, 4).contiguous().permute(0, 3, 2, 1, 4)     # [b][n][l][s][d] in memory
    wide = torch.zeros(2, 70, 2, 2, 80, dtype=dtype, device="cuda")
    wide[..., :64] = v[:, :, 1:3]
    p.cache.write(hk, wide[..., :64], p.table, layer0=1, nlayers=2)
    a, b = p.pool.view(4, -1), other.pool.view(4, -1)
    assert torch.equal(a[1:3], b[1:3]) and (a[0] == 255).all() and (a[3] == 255).all()
    ko = torch.zeros_like(hk)
    vo = torch.zeros_like(wide)
    p.cache.read(ko, vo[..., :64], p.table, layer0=1, nlayers=2)
    k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
    other.cache.read(k2, v2, other.table)
    assert torch.equal(ko, k2[:, :, 1:3]) and torch.equal(vo[..., :64], v2[:, :, 1:3]) and (vo[..., 64:] == 0).all()
    # a broadcast row: the same key row for every token
    one = k[:, :1].expand(2, 70, 4, 2, 64)
    p.cache.write(one, v, p.table)
    p.cache.read(k2, v2, p.table)
    assert torch.equal(k2, k2[:, :1].expand_as(k2))


@pytest.mark.parametrize("fmt,dtype", KINDS[2:], ids=IDS[2:])
@pytest.mark.parametrize("bad", [float("nan"), float("inf"), -float("inf")])
def test_non_finite_rows(fmt, dtype, bad):
    p = Paged(fmt, dtype, [66], N_kv=2)
    k, v = p.rows(1)
    k[0, 65, 0, 1, 40] = bad
    p.cache.write(k, v, p.table)
    assert p.cache.device_error() == binding().ERR_BIT_NON_FINITE
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    p.cache.read(ko, vo, p.table)
    hit = torch.zeros_like(k, dtype=torch.bool)
    hit[0, 65, 0, 1, slice(None) if fmt == "e4m3" else slice(32, 64)] = True
    assert torch.equal(torch.isnan(ko), hit) and not torch.isnan(vo).any()
    # attention over the tokens in front of it does not see it
    q = torch.randn(1, 1, 8, 128, device="cuda").to(dtype)
    n = torch.tensor([65], dtype=torch.int32, device="cuda")
    out, lse = p.cache.decode_attn(q, p.table, n, return_lse=True)
    p.check(q, out, lse, lens=[65])


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("where", ["key", "value", "only key"])
def test_a_nan_that_counts_is_seen(fmt, dtype, where):
    """A stored NaN reaches the outputs of its own key head (a quantised row or group is NaN as a whole) and no other;
    also where it is the only token."""
    n = 1 if where == "only key" else 200
    p = Paged(fmt, dtype, [n, n], N_kv=2, G=2)
    k, v = p.rows(1)
    x = v if where == "value" else k
    x[1, n // 2, 0, 1, 40] = float("nan")
    p.cache.write(k, v, p.table)
    q = torch.randn(2, 1, 4, 128, generator=gen(5), device="cuda").to(dtype)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    p.check(q, out, lse, units={(0, 0, 0), (0, 0, 1), (1, 0, 0)})
    mine = out[1, 0, 2:].float()
    if where == "value":
        hit = {"plain": slice(40, 41), "e4m3": slice(None), "int4": slice(32, 64)}[fmt]
        assert torch.isnan(mine[:, hit]).all() and torch.isfinite(lse).all()
        if fmt == "plain":
            assert torch.isfinite(mine[:, :40]).all() and torch.isfinite(mine[:, 41:]).all()
    else:
        assert torch.isnan(mine).all() and torch.isnan(lse[1, 0, 2:]).all() and torch.isfinite(lse[0]).all()


@pytest.mark.parametrize("D", [64, 128])
def test_every_bf16_mantissa(D):
    """Codes and scales for largest magnitudes of every mantissa, in ordinary, large and subnormal binades, beside
    values from all over the range below them: the same bytes as the definitions give in 64 bits."""
    tops, rows = [], []
    g = np.random.default_rng(3)
    for e in (1, 2, 40, 126, 127, 200, 253, 254):                # exponent fields; 0 (subnormal) below
        tops += [(e << 7) | m for m in range(128)]
    tops += list(range(0, 128))
    for t in tops:
        below = g.integers(0, t + 1, D - 1)
        near = np.clip(t - g.integers(0, 260, D - 1), 0, t)       # half of them within two binades of the top
        bits = np.concatenate([[t], np.where(g.random(D - 1) < 0.5, near, below)]) | (g.integers(0, 2, D) << 15)
        rows.append(g.permutation(bits))
    n = len(rows)
    x = torch.from_numpy(np.stack(rows).astype(np.uint16).view(np.int16)).view(torch.bfloat16).cuda().view(1, n, 1, 1, D)
    x64 = x.double().cpu().numpy().reshape(n, D)
    for fmt in ("e4m3", "int4"):
        p = Paged(fmt, torch.bfloat16, [n], N_kv=1, G=1, D=D)
        p.cache.write(x, x.flip(1), p.table)
        assert p.cache.device_error() == 0
        for j in range(-(-n // PAGE)):
            kc, vc, ks, vs = p.parts(p.block(0, int(p.table_cpu[0, j]), 0))
            for s in range(min(PAGE, n - j * PAGE)):
                t = j * PAGE + s
                for c, z, row in ((kc, ks, x64[t]), (vc, vs, x64[n - 1 - t])):
                    wc, wz = po.encode_row(row, fmt)
                    assert np.array_equal(c[s], wc) and np.array_equal(z[s], wz), (fmt, t)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_bad_pages_positions_and_counts(fmt, dtype):
    tk = binding()
    p = Paged(fmt, dtype, [200, 200, 200], N_kv=2, L=1)
    k, v = p.rows(2)
    p.table[1, 1] = p.num_pages                       # out of the pool
    p.table[2, 2] = -1
    before = p.pool.clone()
    rows = torch.tensor([201, 130, -3], dtype=torch.int32, device="cuda")      # cut to 200; page 1 left out; none
    p.cache.write(k, v, p.table, rows=rows)
    assert p.cache.device_error() == tk.ERR_BIT_PAGE
    good = Paged(fmt, dtype, [200, 200, 200], N_kv=2, L=1)
    n = torch.tensor([200, 64, 0], dtype=torch.int32, device="cuda")
    good.cache.write(k, v, good.table, rows=n)
    tail = torch.tensor([0, 2, 0], dtype=torch.int32, device="cuda")
    good.cache.write(k[:, 128:], v[:, 128:], good.table, rows=tail, pos=torch.full_like(tail, 128))
    assert good.cache.device_error() == 0
    assert torch.equal(p.pool, good.pool) and not torch.equal(p.pool, before)
    # reading: the same rows are left out
    ko = torch.full_like(k, 512.0)                    # far above every value
    vo = torch.full_like(v, 512.0)
    p.cache.read(ko, vo, p.table, rows=rows)
    assert (ko[1, 64:128] == 512).all() and (ko[2] == 512).all() and (vo[1, 130:] == 512).all()
    assert not (ko[1, 128:130] == 512).any() and not (vo[0] == 512).any()
    # positions outside of the table
    q = Paged(fmt, dtype, [64], N_kv=2)
    k1, v1 = q.rows(3, 4)
    q.cache.write(k1, v1, q.table, pos=torch.tensor([62], dtype=torch.int32, device="cuda"))
    assert q.cache.device_error() == tk.ERR_BIT_PAGE
    ref = Paged(fmt, dtype, [64], N_kv=2)
    ref.cache.write(k1[:, :2], v1[:, :2], ref.table, pos=torch.tensor([62], dtype=torch.int32, device="cuda"))
    assert ref.cache.device_error() == 0 and torch.equal(q.pool, ref.pool)
    q.cache.write(k1, v1, q.table, pos=torch.tensor([-2], dtype=torch.int32, device="cuda"))
    ref.cache.write(k1[:, 2:], v1[:, 2:], ref.table)
    assert torch.equal(q.pool, ref.pool)
    q.cache.write(k1, v1, q.table, pos=torch.tensor([2 ** 31 - 2], dtype=torch.int32, device="cuda"))
    assert torch.equal(q.pool, ref.pool)


def test_no_rows():
    p = Paged("e4m3", torch.bfloat16, [64])
    k, v = p.rows(3, 0)
    p.cache.write(k, v, p.table)
    p.cache.read(k, v, p.table)
    assert (p.pool == 255).all() and p.cache.device_error() == 0


# ---------------------------------------------------------------------------
# attention
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("D,G,N_kv", [(128, 4, 2), (64, 1, 3), (128, 8, 1), (64, 8, 2), (128, 1, 4), (128, 3, 2), (64, 7, 1), (128, 2, 2)])
def test_attention(fmt, dtype, D, G, N_kv):
    """Lengths around every border (16, 32 and 64 tokens), none and one token, pages in any order, NaN behind the end."""
    lens = [0, 1, 15, 16, 17, 31, 33, 63, 64, 65, 127, 129, 700, 0, 95]
    p = Paged(fmt, dtype, lens, L=2, N_kv=N_kv, G=G, D=D)
    k, v = p.rows(7)
    p.cache.write(k, v, p.table, rows=p.seq)
    q = torch.randn(len(lens), 2, N_kv * G, D, generator=gen(9), device="cuda").to(dtype)
    out = torch.full_like(q, float("nan"))
    lse = torch.full(q.shape[:3], float("nan"), device="cuda")
    r = p.cache.decode_attn(q, p.table, p.seq, out=out, lse=lse)
    assert r[0] is out and r[1] is lse
    assert p.cache.device_error() == 0
    p.check(q, out, lse)
    assert (out[0] == 0).all() and torch.isneginf(lse[13]).all()
    again = p.cache.decode_attn(q, p.table, p.seq)    # no lse; the same bits
    assert torch.equal(again, out)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("lens,N_kv,G", [([20000], 2, 4), ([5000, 3, 9000], 1, 8), ([129] * 300, 2, 2)])
def test_attention_split_and_many(fmt, dtype, lens, N_kv, G):
    """One sequence over many CTAs, uneven ones, and more sequences than workers."""
    p = Paged(fmt, dtype, lens, N_kv=N_kv, G=G)
    k, v = p.rows(17)
    p.cache.write(k, v, p.table, rows=p.seq)
    q = torch.randn(len(lens), 1, N_kv * G, 128, generator=gen(19), device="cuda").to(dtype)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    units = None if len(lens) < 10 else {(b, 0, b % N_kv) for b in range(0, len(lens), 23)}
    p.check(q, out, lse, units=units)
    for _ in range(3):
        o2, l2 = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
        assert torch.equal(o2, out) and torch.equal(l2, lse)
    assert p.cache.device_error() == 0


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_attention_layers_scale_and_strided_table(fmt, dtype):
    p = Paged(fmt, dtype, [100, 260], L=3, N_kv=2, G=2, D=64, scale=0.31, max_batch=5)
    k, v = p.rows(23)
    p.cache.write(k, v, p.table, rows=p.seq)
    q = torch.randn(2, 3, 4, 64, generator=gen(29), device="cuda").to(dtype)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    p.check(q, out, lse)
    wide = torch.full((2, 11), 10 ** 6, dtype=torch.int32, device="cuda")      # rows of a larger table
    wide[:, :p.width] = p.table
    o2 = p.cache.decode_attn(q[:, 1:].contiguous(), wide[:, :p.width], p.seq, layer0=1)
    assert torch.equal(o2, out[:, 1:])
    o3 = p.cache.decode_attn(q[1:, 2:].contiguous(), p.table[1:], p.seq[1:], layer0=2, nlayers=1)
    assert torch.allclose(o3.float(), out[1:, 2:].float(), rtol=2 ** -6, atol=1e-3)
    p.check(q[1:, 2:].contiguous(), o3, units=set())


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_attention_large_logits_and_uneven_scales(fmt, dtype):
    """Logits of several hundred (nearly one-hot weights), keys that grow along the sequence so that the running
    maximum moves at every step, and value rows whose magnitudes differ by 2^40 between tokens."""
    n = 300
    p = Paged(fmt, dtype, [n, n], N_kv=2, G=4)
    k, v = p.rows(31)
    grow = torch.linspace(0.1, 12.0, n, device="cuda").view(1, n, 1, 1, 1)
    k = (k.float() * grow).to(dtype)
    mags = 2.0 ** torch.randint(-20, 21, (2, n, 1, 2, 1), generator=gen(37), device="cuda").float()
    v = (v.float() * mags).to(dtype)
    p.cache.write(k, v, p.table, rows=p.seq)
    q = (3 * torch.randn(2, 1, 8, 128, generator=gen(41), device="cuda")).to(dtype)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    p.check(q, out, lse)
    # the large rows get no weight (the queries dislike their keys): what is left are the small ones
    k2 = k.clone()
    k2[:, ::2] = torch.where(mags[:, ::2] > 1, -q[:, 0].view(2, 1, 1, 2, 4, 128)[:, :, :, :, 0].expand_as(k2[:, ::2]).to(dtype), k2[:, ::2])
    p.cache.write(k2, v, p.table, rows=p.seq)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    p.check(q, out, lse)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("power", [-100, 100, 118])
def test_attention_values_of_any_magnitude(fmt, dtype, power):
    """All value rows near the ends of the exponent range: small weights keep their share."""
    p = Paged(fmt, dtype, [300], N_kv=1, G=4)
    k, v = p.rows(83)
    v = (v.float() * 2.0 ** power).to(dtype)
    p.cache.write(k, v, p.table)
    assert p.cache.device_error() == 0
    q = torch.randn(1, 1, 4, 128, generator=gen(89), device="cuda").to(dtype)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    if power < 0:                                     # bounds in units of the values
        for b, l, hs, want, wlse, tol, ltol in p.want(q):
            err = np.abs(out.double().cpu().numpy()[b, l, hs] - want) * 2.0 ** -power
            assert (err <= (tol - 1e-30) * 2.0 ** -power + 1e-6).all() and (np.abs(lse.double().cpu().numpy()[b, l, hs] - wlse) <= ltol).all()
    else:
        p.check(q, out, lse)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_attention_query_magnitudes(fmt, dtype):
    """Queries far from 1: all zero, tiny, and large against tiny keys; channels 2^30 apart in one row."""
    p = Paged(fmt, dtype, [150], N_kv=1, G=4)
    k, v = p.rows(43, outliers=False)
    k[..., 64:] *= 2.0 ** -20
    p.cache.write(k, v, p.table)
    q = torch.randn(1, 1, 4, 128, generator=gen(47), device="cuda")
    q[0, 0, 0] = 0
    q[0, 0, 1] *= 2.0 ** -60
    q[0, 0, 2, 64:] *= 2.0 ** 20
    q[0, 0, 3, :64] *= 2.0 ** -25
    q = q.to(dtype)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    p.check(q, out, lse)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_attention_bad_pages_and_lengths(fmt, dtype):
    """A page outside of the pool has no weight; lengths are cut to the table; negative ones mean none."""
    tk = binding()
    lens = [200, 200, 64, 10, 130]
    p = Paged(fmt, dtype, lens, N_kv=2, G=2)
    k, v = p.rows(53)
    p.cache.write(k, v, p.table, rows=p.seq)
    assert p.cache.device_error() == 0
    q = torch.randn(5, 1, 4, 128, generator=gen(59), device="cuda").to(dtype)
    full, flse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    t = p.table.clone()
    t[0, 1] = p.num_pages + 12345
    t[2, 0] = -(2 ** 31)
    t[4, 2] = 2 ** 31 - 1
    seq = torch.tensor([200, -5, 64, 10, 130], dtype=torch.int32, device="cuda")
    out, lse = p.cache.decode_attn(q, t, seq, return_lse=True)
    assert p.cache.device_error() == tk.ERR_BIT_PAGE
    assert torch.equal(out[3], full[3]) and (out[1:3] == 0).all() and torch.isneginf(lse[1:3]).all()
    q64 = q.double().cpu().numpy()
    for b, keep in ((0, np.r_[0:64, 128:200]), (4, np.r_[0:128])):
        for h in range(2):
            hs = slice(2 * h, 2 * h + 2)
            kk, vv = p.stored(b, 0, h, lens[b])
            r = po.attention(q64[b, 0, hs], kk[keep], vv[keep], p.scale)
            w, wl_ = r[:2]
            tol, ltol = bounds(*r, len(keep), 128, fmt, dtype)
            assert (np.abs(out[b, 0, hs].double().cpu().numpy() - w) <= tol).all()
            assert (np.abs(lse[b, 0, hs].double().cpu().numpy() - wl_) <= ltol).all()
    # longer than the table
    r = Paged(fmt, dtype, [128], N_kv=2, G=2)
    k, v = r.rows(61)
    r.cache.write(k, v, r.table)
    long = torch.tensor([2 ** 31 - 1], dtype=torch.int32, device="cuda")
    qq = q[:1].contiguous()
    out, lse = r.cache.decode_attn(qq, r.table, long, return_lse=True)
    assert r.cache.device_error() == tk.ERR_BIT_PAGE
    r.check(qq, out, lse, lens=[128])


def test_rows_behind_the_batch_stay():
    """A call over the first sequences of padded tensors leaves the rows behind them as they were."""
    tk = binding()
    p = Paged("e4m3", torch.bfloat16, [70, 80, 90], N_kv=2, G=2)
    k, v = p.rows(3)
    p.cache.write(k, v, p.table, rows=p.seq)
    q = torch.randn(4, 1, 4, 128, generator=gen(5), device="cuda").bfloat16()
    out = torch.full((4, 1, 4, 128), 7.0, dtype=torch.bfloat16, device="cuda")
    lse = torch.full((4, 1, 4), 7.0, device="cuda")
    p.cache.decode_attn(q[:2], p.table, p.seq, out=out[:2], lse=lse[:2])
    assert (out[2:] == 7).all() and (lse[2:] == 7).all()
    p.check(q[:2], out[:2], lse[:2])
    assert tk.PAGE_TOKENS == PAGE


def test_pool_past_32_bits():
    """Blocks behind 2^32 bytes of the pool."""
    p = Paged("plain", torch.bfloat16, [130, 65], L=2, N_kv=8, G=2, num_pages=12000, first_page=11900)
    k, v = p.rows(3)
    p.cache.write(k, v, p.table, rows=p.seq)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    p.cache.read(ko, vo, p.table, rows=p.seq)
    assert torch.equal(ko[0], k[0]) and torch.equal(vo[1, :65], v[1, :65])
    q = torch.randn(2, 2, 16, 128, generator=gen(5), device="cuda").bfloat16()
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    assert p.cache.device_error() == 0
    p.check(q, out, lse, units={(0, 1, 7), (1, 1, 7), (0, 0, 0), (1, 0, 3)})


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_largest_batch(fmt, dtype):
    """4096 sequences, most of them empty or a token long, a few of several pages."""
    g = np.random.default_rng(5)
    lens = [int(x) for x in g.choice([0, 0, 1, 2, 3], size=4096)]
    for b, n in ((0, 130), (1000, 65), (4095, 300)):
        lens[b] = n
    p = Paged(fmt, dtype, lens, N_kv=1, G=5, D=64)
    k, v = p.rows(3)
    p.cache.write(k, v, p.table, rows=p.seq)
    q = torch.randn(4096, 1, 5, 64, generator=gen(5), device="cuda").to(dtype)
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    assert p.cache.device_error() == 0
    p.check(q, out, lse, units={(b, 0, 0) for b in (*range(0, 4096, 97), 1000, 4095)})
    none = torch.tensor(lens, device="cuda") == 0
    assert (out[none] == 0).all() and torch.isneginf(lse[none]).all() and torch.isfinite(lse[~none]).all()
    # all of them empty
    zero = torch.zeros(4096, dtype=torch.int32, device="cuda")
    out, lse = p.cache.decode_attn(q, p.table, zero, return_lse=True)
    assert (out == 0).all() and torch.isneginf(lse).all()
    assert torch.equal(p.cache.decode_attn(q, p.table, p.seq)[~none], p.cache.decode_attn(q, p.table, p.seq)[~none])


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_shared_pages_and_explicit_stream(fmt, dtype):
    """Two sequences that begin with the same page, and one whose table names a page twice; a stream by argument."""
    p = Paged(fmt, dtype, [64, 200, 128], N_kv=2, G=6)
    k, v = p.rows(3)
    p.cache.write(k, v, p.table, rows=p.seq)
    p.table[1, 0] = p.table[0, 0]
    p.table_cpu[1, 0] = p.table_cpu[0, 0]
    p.table[2, 1] = p.table[2, 0]
    p.table_cpu[2, 1] = p.table_cpu[2, 0]
    q = torch.randn(3, 1, 12, 128, generator=gen(5), device="cuda").to(dtype)
    side = torch.cuda.Stream()
    torch.cuda.synchronize()
    out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True, stream=side)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    side.synchronize()
    torch.cuda.synchronize()
    p.cache.read(ko, vo, p.table, rows=p.seq, stream=side)
    side.synchronize()
    p.check(q, out, lse)
    assert torch.equal(ko[1, :64], ko[0, :64]) and torch.equal(vo[2, 64:128], vo[2, :64])
    assert p.cache.device_error() == 0


def test_many_layers_and_rows_in_one_call():
    """A call whose row count takes more than one launch (layers are split), with almost all rows unused."""
    L, S = 160, 1 << 20
    p = Paged("e4m3", torch.bfloat16, [40], L=L, N_kv=8, G=1, D=64)
    k, v = (x.expand(1, 3, L, 8, 64).contiguous() for x in p.rows(3, 1))
    n = torch.tensor([3], dtype=torch.int32, device="cuda")
    p.cache.write(k[:, :1].expand(1, S, L, 8, 64), v[:, :1].expand(1, S, L, 8, 64), p.table, rows=n)
    ko, vo = torch.zeros_like(k), torch.zeros_like(v)
    p.cache.read(ko, vo, p.table, rows=n)
    ref = Paged("e4m3", torch.bfloat16, [40], L=L, N_kv=8, G=1, D=64)
    ref.cache.write(k, v, ref.table)
    kr, vr = torch.zeros_like(k), torch.zeros_like(v)
    ref.cache.read(kr, vr, ref.table)
    assert torch.equal(p.pool, ref.pool) and torch.equal(ko, kr) and torch.equal(vo, vr)
    assert p.cache.device_error() == 0


@pytest.mark.parametrize("lens,N_kv,G", [
    ([1028, 5000, 2391, 112, 5000, 5000, 1136], 8, 4),      # most CTAs share a unit with the one before and the one behind
    ([1028, 5000, 2391, 112, 5000, 5000, 1136], 8, 1),
    ([700, 90, 1500, 64] * 12, 4, 2),
    ([20000, 9000], 2, 8),                                   # units of many CTAs
    ([30000], 3, 3)])
@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_results_do_not_depend_on_timing(fmt, dtype, lens, N_kv, G):
    p = Paged(fmt, dtype, lens, N_kv=N_kv, G=G)
    k, v = p.rows(3)
    p.cache.write(k, v, p.table, rows=p.seq)
    q = torch.randn(len(lens), 1, N_kv * G, 128, generator=gen(5), device="cuda").to(dtype)
    want, wlse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    assert torch.isfinite(want).all()
    differ = torch.zeros((), dtype=torch.int64, device="cuda")
    for _ in range(200):
        out, lse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
        differ += (out != want).sum() + (lse != wlse).sum()
    assert differ.item() == 0


# ---------------------------------------------------------------------------
# streams, graphs, use together
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_two_streams_with_a_scratch_each(fmt, dtype):
    p = Paged(fmt, dtype, [3000, 2000], N_kv=2, G=4)
    k, v = p.rows(3)
    p.cache.write(k, v, p.table, rows=p.seq)
    qs = [torch.randn(2, 1, 8, 128, generator=gen(5 + i), device="cuda").to(dtype) for i in range(2)]
    want = [p.cache.decode_attn(q, p.table, p.seq) for q in qs]
    streams, scratch = [torch.cuda.Stream() for _ in qs], [p.cache.new_scratch() for _ in qs]
    torch.cuda.synchronize()
    got = [[], []]
    for _ in range(20):
        for i in range(2):
            with torch.cuda.stream(streams[i]):
                got[i].append(p.cache.decode_attn(qs[i], p.table, p.seq, scratch=scratch[i]))
    torch.cuda.synchronize()
    for i in range(2):
        assert all(torch.equal(x, want[i]) for x in got[i])
    assert p.cache.device_error() == 0


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_decode_loop_in_a_graph(fmt, dtype):
    """A captured step (append one row a sequence, attend, lengths advance on the device) replayed over page borders
    gives what eager calls give; sequences that are padding (count 0) stay empty."""
    start = [62, 0, 127, 0]
    live = torch.tensor([1, 1, 1, 0], dtype=torch.int32, device="cuda")
    steps = 5
    ends = [n + steps * a for n, a in zip(start, [1, 1, 1, 0])]
    a = Paged(fmt, dtype, [max(1, e) for e in ends], N_kv=2, G=4, L=2)
    b = Paged(fmt, dtype, [max(1, e) for e in ends], N_kv=2, G=4, L=2)
    k, v = a.rows(3, max(ends))
    first = torch.tensor(start, dtype=torch.int32, device="cuda")
    for p in (a, b):
        p.cache.write(k, v, p.table, rows=first)
    g = gen(11)
    new = [(torch.randn(4, 1, 2, 2, 128, generator=g, device="cuda").to(dtype), torch.randn(4, 1, 2, 2, 128, generator=g, device="cuda").to(dtype),
            torch.randn(4, 2, 8, 128, generator=g, device="cuda").to(dtype)) for _ in range(steps)]
    want = []
    lens = first.clone()
    for kn, vn, q in new:
        a.cache.write(kn, vn, a.table, pos=lens, rows=live)
        lens = lens + live
        want.append(a.cache.decode_attn(q, a.table, lens))
    kn, vn, q = (torch.zeros_like(x) for x in new[0])
    out = torch.zeros_like(q)
    seq, seq_after = first.clone(), torch.zeros_like(first)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    graph = torch.cuda.CUDAGraph()
    scratch = b.cache.new_scratch()
    torch.cuda.synchronize()
    with torch.cuda.graph(graph, stream=side):
        b.cache.write(kn, vn, b.table, pos=seq, rows=live)
        torch.add(seq, live, out=seq_after)
        b.cache.decode_attn(q, b.table, seq_after, out=out, scratch=scratch)
        seq.copy_(seq_after)
    for i, (x, y, z) in enumerate(new):
        kn.copy_(x), vn.copy_(y), q.copy_(z)
        graph.replay()
        assert torch.equal(out, want[i]), f"step {i}"
    assert torch.equal(a.pool, b.pool) and seq.tolist() == ends
    assert (out[3] == 0).all()
    a.lens = ends
    a.check(new[-1][2], out)
    assert a.cache.device_error() == 0 and b.cache.device_error() == 0


def test_paged_prompt_is_thinned():
    """A running prompt lives in pages; when it is to be thinned its rows are read back into the tensors that the
    prefill takes, and the thinned cache is the one that the original tensors give.  Until then, attention over the
    pages and over a cache that keeps every channel agree."""
    tk = binding()
    w = wl.shrink(wl.get_config("c2"), S=400, L=2, B=2, steps=3)
    data = wl.make_prefill(w, device="cuda")
    K, V, Q = data["K"], data["V"], data["Q_obs"]
    p = Paged("plain", torch.bfloat16, [n + 8 for n in w.seq_lens], L=w.L, N_kv=w.N_kv, G=w.N_q // w.N_kv, D=w.D)
    rows = torch.tensor(w.seq_lens, dtype=torch.int32, device="cuda")
    p.cache.write(K, V, p.table, rows=rows)
    k2, v2 = torch.zeros_like(K), torch.zeros_like(V)
    p.cache.read(k2, v2, p.table, rows=rows)
    caches = []
    for kk, vv in ((K, V), (k2, v2)):
        cfg = tk.make_config(w.B, w.L, w.N_q, w.N_kv, w.D, w.S_max, w.S_obs, w.recent, w.steps, w.lam, w.torch_dtype)
        c = tk.ThinKCache(cfg, w.seq_lens)
        c.k_thin.zero_()
        c.prefill(Q, kk, vv)
        caches.append(c)
    assert torch.equal(caches[0].idx_tensor(), caches[1].idx_tensor())
    assert torch.equal(caches[0].k_thin, caches[1].k_thin)
    dense = tk.ThinKCache(tk.make_config(w.B, w.L, w.N_q, w.N_kv, w.D, w.S_max, w.S_obs, w.recent, w.steps, 0.0, w.torch_dtype), w.seq_lens)
    dense.prefill(Q, K, V)
    lens = rows.clone()
    for t in range(w.steps):
        st = wl.make_step(w, t, device="cuda")
        p.cache.write(st["k_new"].unsqueeze(1), st["v_new"].unsqueeze(1), p.table, pos=lens)
        lens = lens + 1
        paged = p.cache.decode_attn(st["q"], p.table, lens)
        dense.append(st["k_new"], st["v_new"])
        full = dense.decode_attn(st["q"])
        # both are within half a bf16 step plus 2^-8 (weights rounded to bf16 in the dense kernel) of the same value
        d = (paged.float() - full.float()).abs()
        assert (d <= 2.0 ** -7 * full.float().abs() + 2.0 ** -7 * 4).all()
        assert torch.equal(caches[0].append_decode(st["k_new"], st["v_new"], st["q"]), caches[1].append_decode(st["k_new"], st["v_new"], st["q"]))
    p.check(st["q"], paged, lens=[int(x) for x in lens], units={(0, 0, 0), (1, 1, w.N_kv - 1)})
    assert p.cache.device_error() == 0


def test_lse_joins_two_parts():
    """Attention over two page ranges, joined by their log sums, is attention over both."""
    p = Paged("e4m3", torch.bfloat16, [64 * 5 + 9], N_kv=2, G=4)
    k, v = p.rows(3)
    p.cache.write(k, v, p.table)
    q = torch.randn(1, 1, 8, 128, generator=gen(5), device="cuda").bfloat16()
    whole, wlse = p.cache.decode_attn(q, p.table, p.seq, return_lse=True)
    cut = 128
    n0 = torch.tensor([cut], dtype=torch.int32, device="cuda")
    o0, l0 = p.cache.decode_attn(q, p.table, n0, return_lse=True)
    o1, l1 = p.cache.decode_attn(q, p.table[:, cut // 64:], p.seq - cut, return_lse=True)
    assert torch.allclose(torch.logaddexp(l0, l1), wlse, rtol=0, atol=1e-5)
    w0, w1 = torch.exp(l0 - wlse).unsqueeze(-1), torch.exp(l1 - wlse).unsqueeze(-1)
    joined = w0 * o0.float() + w1 * o1.float()
    # each part carries half a bf16 step of itself, the whole half a step of itself
    tol = 2.0 ** -8 * (w0 * o0.float().abs() + w1 * o1.float().abs() + whole.float().abs()) * 1.01 + 2.0 ** -10
    assert ((joined - whole.float()).abs() <= tol).all()


def test_buffers_that_overlap_and_counts_past_32_bits_are_refused():
    tk = binding()
    p = Paged("plain", torch.float32, [70, 80], L=2, N_kv=2, G=2)
    c, n = p.cache, 2 * 2 * 4 * 128
    mem = torch.zeros(2 * n, device="cuda")
    q = mem[:n].view(2, 2, 4, 128)
    before = p.pool.clone()

    def refused(call):
        with pytest.raises(tk.ThinKError) as e:
            call()
        assert e.value.status == tk.ERR_INVALID_ARG

    refused(lambda: c.decode_attn(q, p.table, p.seq, out=q))
    refused(lambda: c.decode_attn(q, p.table, p.seq, out=mem[n - 4:2 * n - 4].view(q.shape)))
    refused(lambda: c.decode_attn(q, p.table, p.seq, lse=mem[n - 1:n + 15].view(2, 2, 4)))
    refused(lambda: c.decode_attn(q, p.table, p.seq, out=mem[n:].view(q.shape), lse=mem[2 * n - 16:].view(2, 2, 4)))
    k, v = p.rows(3)
    long = k[:, :1].expand(2, 1 << 32, 2, 2, 128)
    refused(lambda: c.write(long, long, p.table))
    refused(lambda: c.write(k, v, p.table, layer0=1 << 32, nlayers=2))
    refused(lambda: c.decode_attn(q, p.table, p.seq, layer0=1 << 32, nlayers=2))
    wide = p.table[:, :1].expand(2, 1 << 32)
    refused(lambda: c.write(k, v, wide))
    assert torch.equal(p.pool, before) and c.device_error() == 0
    # side by side is not overlapping (the pool was NaN so far)
    c.write(k, v, p.table, rows=p.seq)
    got = c.decode_attn(q, p.table, p.seq, out=mem[n:].view(q.shape))
    assert torch.isfinite(got).all() and torch.equal(got, c.decode_attn(q, p.table, p.seq))


@pytest.mark.parametrize("fmt,dtype", [("plain", "float32"), ("int4", "bfloat16")])
def test_first_calls_of_a_process_in_a_captured_graph(fmt, dtype):
    """Nothing of a call depends on an earlier one: kernels that never ran may be captured."""
    code = f"""
import torch
from paper_2407_21018_b200 import binding as tk
dt = torch.{dtype}
cfg = tk.make_paged_config(2, 4, 2, 128, 8, 2, dt, tk.PAGE_{fmt.upper()})
c = tk.PagedKVCache(cfg)
g = torch.Generator().manual_seed(3)
k, v = (torch.randn(2, 90, 2, 2, 128, generator=g).to(dt).cuda() for _ in range(2))
k2, v2 = torch.zeros_like(k), torch.zeros_like(v)
q = torch.randn(2, 2, 4, 128, generator=g).to(dt).cuda()
out = torch.zeros_like(q)
table = torch.arange(4, dtype=torch.int32).view(2, 2).cuda()
seq = torch.tensor([90, 33], dtype=torch.int32).cuda()
graph = torch.cuda.CUDAGraph()
torch.cuda.synchronize()
with torch.cuda.graph(graph):
    c.write(k, v, table, rows=seq)
    c.decode_attn(q, table, seq, out=out)
    c.read(k2, v2, table, rows=seq)
graph.replay()
torch.cuda.synchronize()
want = c.decode_attn(q, table, seq)
assert torch.equal(out, want) and out.abs().sum() > 0 and c.device_error() == 0
k3, v3 = torch.zeros_like(k), torch.zeros_like(v)
c.read(k3, v3, table, rows=seq)
assert torch.equal(k2, k3) and torch.equal(v2, v3) and k2[0].abs().sum() > 0 and not k2[1, 33:].any()
print("same")
"""
    root = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))
    r = subprocess.run([sys.executable, "-c", code], cwd=root, capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and "same" in r.stdout, r.stdout + r.stderr


def test_refusals():
    tk = binding()
    p = Paged("plain", torch.bfloat16, [70, 80], L=2, N_kv=2, G=2)
    k, v = p.rows(3)
    q = torch.zeros(2, 2, 4, 128, dtype=torch.bfloat16, device="cuda")
    c = p.cache
    before = p.pool.clone()

    def refused(call, status=tk.ERR_INVALID_ARG):
        with pytest.raises(tk.ThinKError) as e:
            call()
        assert e.value.status == status

    refused(lambda: c.write(k.float(), v, p.table))
    refused(lambda: c.write(k[:, :, :1], v, p.table))
    refused(lambda: c.write(k, v[:, :5], p.table))
    refused(lambda: c.write(k.cpu(), v, p.table))
    refused(lambda: c.write(k, v, p.table.long()))
    refused(lambda: c.write(k, v, p.table[:1]))
    refused(lambda: c.write(k, v, p.table[0]))
    refused(lambda: c.write(k, v, p.table[:1].expand(2, -1)))          # one row for all: its stride is 0
    refused(lambda: c.write(k[0], v, p.table))
    refused(lambda: c.write(k, v[0], p.table))
    refused(lambda: c.decode_attn(q[0], p.table, p.seq))
    refused(lambda: c.write(k, v, p.table.cpu()))
    refused(lambda: c.write(k, v, p.table.t().contiguous().t()))
    refused(lambda: c.write(k, v, p.table, pos=p.seq[:1]))
    refused(lambda: c.write(k, v, p.table, rows=p.seq.long()))
    refused(lambda: c.write(k, v, p.table, layer0=1))
    refused(lambda: c.write(k, v, p.table, layer0=-1, nlayers=2))
    refused(lambda: c.write(k, v, p.table, layer0=1, nlayers=2))
    refused(lambda: c.read(k, v.float(), p.table))
    odd = torch.zeros(2, 80, 2, 2, 129, dtype=torch.bfloat16, device="cuda")[..., :128]      # rows off 16 bytes
    refused(lambda: c.write(odd, v, p.table))
    off = torch.zeros(q.numel() + 1, dtype=q.dtype, device="cuda")[1:].view(q.shape)        # not on 16 bytes
    refused(lambda: c.decode_attn(off, p.table, p.seq))
    refused(lambda: c.decode_attn(q, p.table, p.seq, out=off))
    refused(lambda: c.decode_attn(q, p.table, p.seq, layer0=2, nlayers=0))
    refused(lambda: c.write(k.as_strided((2, 1 << 30, 2, 2, 128), (0, 0, 0, 0, 1)), v.as_strided((2, 1 << 30, 2, 2, 128), (0, 0, 0, 0, 1)), p.table))
    refused(lambda: c.decode_attn(q.float(), p.table, p.seq))
    refused(lambda: c.decode_attn(q[:, :1], p.table, p.seq))
    refused(lambda: c.decode_attn(q[:, :, :2], p.table, p.seq))
    refused(lambda: c.decode_attn(q, p.table, p.seq.long()))
    refused(lambda: c.decode_attn(q, p.table, p.seq[:1]))
    refused(lambda: c.decode_attn(q, p.table, p.seq, out=torch.zeros_like(q).float()))
    refused(lambda: c.decode_attn(q, p.table, p.seq, lse=torch.zeros(2, 2, 3, device="cuda")))
    refused(lambda: c.decode_attn(torch.cat([q, q]), torch.cat([p.table, p.table]), torch.cat([p.seq, p.seq])))
    refused(lambda: c.decode_attn(q, p.table, p.seq, scratch=torch.zeros(256, dtype=torch.uint8, device="cuda")), tk.ERR_CAPACITY)
    refused(lambda: c.decode_attn(q, p.table, p.seq, scratch=c.new_scratch()[16:]))
    refused(lambda: tk.PagedKVCache(p.cfg, device="cpu"))
    refused(lambda: tk.PagedKVCache(p.cfg, pages=p.pool[:-256]), tk.ERR_CAPACITY)
    refused(lambda: tk.PagedKVCache(p.cfg, pages=p.pool.view(torch.int8)))
    assert torch.equal(p.pool, before) and c.device_error() == 0
