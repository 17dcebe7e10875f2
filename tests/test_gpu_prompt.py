"""GPU tests of the attention of many new tokens over the paged cache against the fp64 oracle, row by row, within bounds that
are derived from the kernels' roundings (see `bounds`)."""
import numpy as np
import pytest
import torch

from oracle import packed_oracle as ko
from oracle import paged_oracle as po

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


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def bounds(sizes, n, D, dtype, lse):
    """Error bounds of one row's heads, first order in the roundings; sizes as in paged_oracle.attention, u = 2^-23 (one
    fp32 operation, also where the tensor core's adder truncates).
      logit   D products (exact: stored values have at most 11 bits, in two parts of 8; queries 8) summed in fp32, the scale in base
              2 and the reference taken off: error dx <= (D + 8) u qk.  A weight exp(x) carries it twice, its own and the
              denominator's, and 2^-21 for exp2 (2^-22 at most for each way of computing it).
      weight  rounded to bf16 once it meets the values, 2^-8 of itself, fp32 caches none; below 2^-118 it may be lost.
      sums    n products added in fp32 in any order: n u.
      output  one division (u) and the rounding to its type."""
    u, half = 2.0 ** -23, torch.finfo(dtype).eps / 2
    w = 2.0 ** -8 if dtype == torch.bfloat16 else 0.0
    dx = (D + 8) * u * sizes["qk"]
    rel = np.expm1(2 * dx) + 2 * 2.0 ** -21 + w + 2 * (n + 16) * u
    lost = n * 2.0 ** -118 * sizes["vmax"]
    out = rel[:, None] * sizes["absv"] + lost
    return out, half, dx + 2.0 ** -21 + (n + 16) * u + 4 * u * np.abs(lse)


class Prompt:
    """A cache over a pool full of 0xff bytes (NaN in every format) that holds `held[b]` + `rows[b]` written tokens of each
    sequence, and queries for the last rows[b]."""

    def __init__(self, fmt, dtype, rows, held, L=1, N_kv=2, G=4, D=128, packed=True, seed=0, scale=0.0, k_edit=None, v_edit=None, width=0,
                 extra_rows=0, max_rows=None):
        tk = binding()
        self.fmt, self.dtype, self.rows, self.held, self.L, self.N_kv, self.G, self.D, self.packed = fmt, dtype, rows, held, L, N_kv, G, D, packed
        B = len(rows)
        n = [a + b for a, b in zip(rows, held)]
        need = [ko.pages_of(x) for x in n]
        pages = sum(need) + 2
        self.cfg = tk.make_paged_config(L, N_kv * G, N_kv, D, pages, B, dtype, FMT[fmt], scale)
        self.scale = scale or D ** -0.5
        self.pool = torch.full((int(tk.paged_bytes(self.cfg).pages),), 255, dtype=torch.uint8, device="cuda")
        self.cache = tk.PagedKVCache(self.cfg, pages=self.pool)
        order = np.random.default_rng(seed).permutation(pages).tolist()
        width = width or max(1, max(need))
        table, at = [], 0
        for m in need:
            table.append(order[at:at + m] + [-5] * (width - m))
            at += m
        self.table = ints(table)
        g = gen(seed)
        S = max(1, max(n))
        k = torch.randn(B, S, L, N_kv, D, generator=g, device="cuda")
        v = torch.randn(B, S, L, N_kv, D, generator=g, device="cuda")
        k[..., :3] *= 8
        k, v = k.to(dtype), v.to(dtype)
        if k_edit:
            k_edit(k)
        if v_edit:
            v_edit(v)
        self.cache.write(k, v, self.table, rows=ints(n))
        self.cache.read(k, v, self.table, rows=ints(n))
        self.k, self.v = k, v
        if fmt == "int4":                       # read-back rounds to bf16; the oracle wants n * s
            self.k, self.v = self.exact_int4()
        self.first = [sum(rows[:b]) + b * extra_rows for b in range(B)]
        total = sum(rows) + B * extra_rows
        heads = N_kv * G
        shape = (max(1, total), L, heads, D) if packed else (B, max_rows or max(1, max(rows)), L, heads, D)
        self.q = torch.randn(shape, generator=g, device="cuda").to(dtype)
        self.pos, self.nrows, self.start = ints(held), ints(rows), ints(self.first) if packed else None

    def exact_int4(self):
        """Keys and values of the pages in 64 bits."""
        tk = binding()
        raw = self.pool.cpu().numpy()
        block = int(tk.paged_bytes(self.cfg).block)
        D, out = self.D, []
        table = self.table.cpu().numpy()
        rb, sb = D // 2, 2 * D // 32
        for part in (0, 1):
            x = np.zeros(self.k.shape)
            for b in range(x.shape[0]):
                n = self.rows[b] + self.held[b]
                for l in range(self.L):
                    for h in range(self.N_kv):
                        for j in range(ko.pages_of(n)):
                            o = ((l * self.cfg.num_pages + int(table[b, j])) * self.N_kv + h) * block
                            m = min(PAGE, n - j * PAGE)
                            codes = raw[o + part * PAGE * rb:][:PAGE * rb].reshape(PAGE, rb)[:m]
                            sc = raw[o + 2 * PAGE * rb + part * PAGE * sb:][:PAGE * sb].reshape(PAGE, sb)[:m]
                            q = np.empty((m, D))
                            q[:, 0::2], q[:, 1::2] = (codes & 15).astype(int) - 8, (codes >> 4).astype(int) - 8
                            s = (np.ascontiguousarray(sc).view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
                            x[b, j * PAGE:j * PAGE + m, l, h] = q * np.repeat(s, 32, axis=1)
            out.append(torch.from_numpy(x).cuda())
        return out

    def call(self, out=None, lse=None, **kw):
        if out is None:
            out = torch.full_like(self.q, 7.0)
        if lse is None:
            lse = torch.full(self.q.shape[:-1], 7.0, dtype=torch.float32, device="cuda")
        return self.cache.prompt_attn(self.q, self.table, self.pos, rows=self.nrows, start=self.start, out=out, lse=lse, **kw)

    def at(self, x, b):
        return x[self.first[b]:self.first[b] + self.rows[b]] if self.packed else x[b, :self.rows[b]]

    def check(self, out, lse, rows=None):
        """Every row, or those that `rows` (a function of sequence and row) names."""
        seen = torch.zeros(out.shape[:-3], dtype=torch.bool, device="cuda")
        worst = 0.0
        for b in range(len(self.rows)):
            if self.rows[b] == 0:
                continue
            self.at(seen, b)[:] = True
            q, o, z = (self.at(x, b).double().cpu().numpy() for x in (self.q, out, lse))
            for l in range(self.L):
                for h in range(self.N_kv):
                    hs = slice(h * self.G, (h + 1) * self.G)
                    k, v = self.k[b, :, l, h].double().cpu().numpy(), self.v[b, :, l, h].double().cpu().numpy()
                    for s in range(self.rows[b]):
                        if rows is not None and not rows(b, s):
                            continue
                        n = self.held[b] + s + 1
                        want, wlse, sizes = po.attention(q[s, l, hs], k[:n], v[:n], self.scale)
                        sizes["vmax"] = np.abs(v[:n]).max()
                        tol, half, ltol = bounds(sizes, n, self.D, self.dtype, wlse)
                        tol = tol + half * (np.abs(want) + tol)
                        err = np.abs(o[s, l, hs] - want)
                        assert (err <= tol).all(), f"{(b, s, l, h)}: {(err / tol).max():.3g} of the bound, {err.max():.3g}"
                        worst = max(worst, (err / tol).max())
                        le = np.abs(z[s, l, hs] - wlse)
                        assert (le <= ltol).all(), f"lse {(b, s, l, h)}: {le.max():.3g} > {ltol.min():.3g}"
        assert (out[~seen] == 7).all() and (lse[~seen] == 7).all(), "rows that no sequence has"
        return worst


def some(n):
    """The borders of items and tiles, and a few in between."""
    return lambda b, s: s < 3 or s % 61 == 0 or s % 64 in (0, 63) or s % 85 in (0, 84) or s >= n - 2


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("rows,held", [
    ([1], [0]), ([1], [63]), ([1], [64]), ([2], [127]), ([64], [0]), ([65], [0]), ([127], [1]), ([129], [128]), ([5, 0, 1], [0, 9, 300]),
    ([33, 1, 70], [100, 4000, 64]), ([300], [77]),
], ids=str)
def test_prompt_attn(fmt, dtype, D, rows, held):
    p = Prompt(fmt, dtype, rows, held, D=D, N_kv=2, G=4)
    out, lse = p.call()
    p.check(out, lse, some(max(rows)))
    assert p.cache.device_error() == 0


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("G", [1, 2, 3, 5, 6, 7, 8])
def test_prompt_attn_group_sizes(fmt, dtype, G):
    p = Prompt(fmt, dtype, [200, 3], [70, 900], D=64 if G % 2 else 128, N_kv=1, G=G, L=2, packed=G % 3 != 0, seed=G)
    out, lse = p.call()
    p.check(out, lse, some(200))


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_prompt_attn_longer(fmt, dtype):
    """Items that many CTAs share, and sequences of many items."""
    p = Prompt(fmt, dtype, [1100, 8], [0, 20000], D=128, N_kv=1, G=8, seed=3)
    out, lse = p.call()
    p.check(out, lse, lambda b, s: b == 1 and s % 3 == 0 or b == 0 and s % 173 == 0)
    again = [p.call() for _ in range(5)]
    assert all(torch.equal(out, x[0]) and torch.equal(lse, x[1]) for x in again)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_prompt_attn_equals_decode_attn_on_last_rows(fmt, dtype):
    """The last row of each sequence is what the one-token call computes, up to both calls' bounds."""
    p = Prompt(fmt, dtype, [40, 1, 130], [0, 500, 3], D=128, N_kv=2, G=4)
    out, lse = p.call()
    last = torch.stack([p.at(p.q, b)[-1] for b in range(3)])
    o1, l1 = p.cache.decode_attn(last.contiguous(), p.table, p.pos + p.nrows, return_lse=True)
    o2, l2 = torch.stack([p.at(out, b)[-1] for b in range(3)]), torch.stack([p.at(lse, b)[-1] for b in range(3)])
    vmax = float(p.v.abs().max())
    assert (o1.double() - o2.double()).abs().max() <= vmax * (2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -13)
    assert (l1 - l2).abs().max() <= 2.0 ** -13


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_prompt_attn_views_layers_and_gaps(fmt, dtype):
    """Strided queries and outputs, a range of layers, packed rows with gaps, a table with spare columns."""
    p = Prompt(fmt, dtype, [30, 66], [10, 0], L=3, D=64, N_kv=2, G=2, extra_rows=5, width=9)
    want, wl = p.call()
    p.check(want, wl, some(66))
    wide = torch.randn(p.q.shape[0], 3, 6, 64, generator=gen(1), device="cuda").to(dtype)
    wide[:, :, 1:5] = p.q
    dst = torch.full((3, p.q.shape[0], 4, 64), 7.0, dtype=dtype, device="cuda").permute(1, 0, 2, 3)
    out, lse = p.cache.prompt_attn(wide[:, 1:, 1:5], p.table, p.pos, rows=p.nrows, start=p.start, out=dst[:, 1:],
                                   lse=torch.full((p.q.shape[0], 2, 4), 7.0, device="cuda"), layer0=1)
    assert (dst[:, 0] == 7).all()
    one, z = p.cache.prompt_attn(p.q[:, 1:2], p.table, p.pos, rows=p.nrows, start=p.start, layer0=1, nlayers=1, return_lse=True)
    # (bits may differ: where items are cut depends on all that a call names)
    for layers, o, zz in ((slice(1, 3), out, lse), (slice(1, 2), one, z)):
        full, fl = want.clone(), wl.clone()
        for b in range(2):
            p.at(full, b)[:, layers] = p.at(o, b)
            p.at(fl, b)[:, layers] = p.at(zz, b)
        p.check(full, fl, some(66))
    # padded, the same rows
    pad = torch.zeros(2, 70, 3, 4, 64, dtype=dtype, device="cuda")
    for b in range(2):
        pad[b, :p.rows[b]] = p.at(p.q, b)
    o2 = p.cache.prompt_attn(pad, p.table, p.pos, rows=p.nrows)
    for b in range(2):
        assert torch.equal(o2[b, :p.rows[b]], p.at(want, b))       # (the same items, cut at the same places)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_what_a_row_does_not_see_does_not_reach_it(fmt, dtype, value):
    """A key and a value of NaN or infinity at token 40 of a prompt of 100: rows in front of it are as without; rows from it
    on hold what the formula gives."""
    t = 40

    def edit(x):
        x[0, t, 0, 0, 5] = value

    clean = Prompt(fmt, dtype, [100], [0], N_kv=1, G=4, D=64)
    want, wl = clean.call()
    for which in ("k", "v"):
        p = Prompt(fmt, dtype, [100], [0], N_kv=1, G=4, D=64, **{which + "_edit": edit})
        out, lse = p.call()
        assert torch.equal(out[:t], want[:t]) and torch.equal(lse[:t], wl[:t])
        if which == "v":
            assert torch.equal(lse, wl)
            whole = fmt != "plain"                       # a quantised row (or group) with a NaN or an infinity is all NaN
            bad = out[t:, 0, :, :32] if fmt == "int4" else out[t:, 0] if whole else out[t:, 0, :, 5]
            assert bad.isnan().all() if whole or value != value else (bad == value).all()
            if not whole:
                keep = [c for c in range(64) if c != 5]
                assert torch.equal(out[:, 0, :, keep], want[:, 0, :, keep])
            elif fmt == "int4":
                assert torch.equal(out[:, 0, :, 32:], want[:, 0, :, 32:])
        elif fmt != "plain" or value != value:
            assert out[t:].isnan().all() and lse[t:].isnan().all()
        else:                                            # an infinite key: its logit has the sign of the query's channel
            up = p.q[t:, 0, :, 5].float() * value > 0
            assert out[t:, 0][up].isnan().all()
            assert not out[t:, 0][~up].isnan().any()     # weight 0, everything else as it is
        assert (out != 7).any(-1).all()


@pytest.mark.parametrize("fmt,dtype", KINDS[:2], ids=IDS[:2])
def test_rows_whose_logits_are_all_minus_infinity(fmt, dtype):
    """Keys of -infinity where all queries are positive: the first rows have nothing else; later ones see a finite key."""
    def edit(k):
        k[0, :5] = 0
        k[0, :5, :, :, 0] = -float("inf")

    p = Prompt(fmt, dtype, [9], [0], N_kv=1, G=2, D=64, k_edit=edit)
    p.q.abs_().add_(0.5)
    out, lse = p.call()
    assert out[:5].isnan().all() and (lse[:5] == -float("inf")).all()
    assert out[5:].isfinite().all() and lse[5:].isfinite().all()


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
def test_bad_tables_positions_and_counts(fmt, dtype):
    """Pages outside the pool are left out, positions and counts are cut; the error word says so."""
    tk = binding()
    p = Prompt(fmt, dtype, [100, 20], [60, 0], N_kv=1, G=4, D=128)
    table = p.table.clone()
    table[0, 1] = 10 ** 6                                # tokens 64 .. 127
    out, lse = p.cache.prompt_attn(p.q, table, p.pos, rows=p.nrows, start=p.start, return_lse=True)
    assert p.cache.device_error() == tk.ERR_BIT_PAGE
    q, k, v = p.q.double().cpu().numpy(), p.k.double().cpu().numpy(), p.v.double().cpu().numpy()
    for s in (0, 3, 4, 50, 99):
        n = 61 + s
        keep = [t for t in range(n) if not 64 <= t < 128]
        want, wl, sizes = po.attention(q[s, 0], k[0, keep, 0, 0], v[0, keep, 0, 0], p.scale)
        sizes["vmax"] = np.abs(v).max()
        tol, half, ltol = bounds(sizes, n, 128, dtype, wl)
        assert (np.abs(out[s, 0].double().cpu().numpy() - want) <= tol + half * (np.abs(want) + tol)).all()
        assert (np.abs(lse[s, 0].double().cpu().numpy() - wl) <= ltol).all()
    table[:] = -1                                        # no page at all: rows without tokens
    out, lse = p.cache.prompt_attn(p.q, table, p.pos, rows=p.nrows, start=p.start, return_lse=True)
    assert (out == 0).all() and (lse == -float("inf")).all()
    for pos, rows, start, kept in (([-30, 0], [100, 20], [0, 100], None), ([10 ** 9, 2 ** 31 - 1], [100, 20], [0, 100], None), ([0, 0], [1000, 20], [0, 100], None),
                                   ([0, 0], [100, 20], [0, 110], 10), ([0, 0], [100, 20], [0, -3], 0), ([0, 0], [100, 20], [0, 2 ** 31 - 1], 0)):
        q = Prompt(fmt, dtype, [100, 20], [60, 0], N_kv=1, G=4, D=128)
        guard = torch.full((140, 1, 4, 128), 7.0, dtype=dtype, device="cuda")
        out = guard[10:130]
        q.cache.prompt_attn(q.q, q.table, ints(pos), rows=ints(rows), start=ints(start), out=out)
        assert q.cache.device_error() == tk.ERR_BIT_PAGE
        assert (guard[:10] == 7).all() and (guard[130:] == 7).all()
        if kept is not None:
            assert (out[100:] == 7).flatten(1).all(1).sum() == 20 - kept
        if pos[0] == -30:
            assert (out[:30] == 0).all() and (out[30:100] != 0).any(-1).all()


def test_graphs_streams_and_scratch():
    """Captured and replayed with other lengths and pages; two streams with a scratch buffer each."""
    p = Prompt("plain", torch.bfloat16, [90, 7], [100, 900], N_kv=2, G=4)
    want, wl = p.call()
    out, lse = torch.full_like(p.q, 7.0), torch.full(p.q.shape[:-1], 7.0, device="cuda")
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        p.call(out=out, lse=lse)
    graph.replay()
    assert torch.equal(out, want) and torch.equal(lse, wl)
    p.nrows.copy_(ints([3, 7]))
    out.fill_(7)
    graph.replay()
    assert (out[3:90] == 7).all()
    p.rows = [3, 7]
    full, fl = torch.full_like(out, 7.0), torch.full_like(lse, 7.0)
    for b in range(2):
        p.at(full, b).copy_(p.at(out, b))
        p.at(fl, b).copy_(p.at(lse, b))
    p.check(full, fl)
    p.nrows.copy_(ints([90, 7]))
    streams = [torch.cuda.Stream() for _ in range(2)]
    scratch = [p.cache.new_prompt_scratch() for _ in range(2)]
    torch.cuda.synchronize()
    outs = [[p.call(stream=streams[i], scratch=scratch[i])[0] for _ in range(20)] for i in range(2)]
    torch.cuda.synchronize()
    assert all(torch.equal(x, want) for o in outs for x in o)


def test_pools_past_32_bits():
    """The last pages of a pool of more than 2^32 bytes."""
    tk = binding()
    N, D, pages = 8, 128, 2 ** 32 // (8 * 32768) + 40
    cfg = tk.make_paged_config(1, 8, N, D, pages, 1, torch.bfloat16)
    cache = tk.PagedKVCache(cfg)
    T = 500
    g = gen(9)
    k, v, q = (torch.randn(T, 1, N, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(3))
    small = tk.PagedKVCache(tk.make_paged_config(1, 8, N, D, 8, 1, torch.bfloat16))
    t = torch.arange(T, device="cuda")
    res = []
    for c, table in ((small, ints([list(range(8))])), (cache, ints([list(range(pages - 8, pages))]))):
        c.write_slots(k, v, (table[0, t // PAGE].long() * PAGE + t % PAGE).to(torch.int32))
        res.append(c.prompt_attn(q, table, ints([0]), rows=ints([T]), start=ints([0]), return_lse=True))
    assert torch.equal(res[0][0], res[1][0]) and torch.equal(res[0][1], res[1][1])


def test_a_packed_step_end_to_end():
    """plan -> rope -> write by slots -> prompt attention -> one-token attention of the next step, twice over, in a graph, against
    dense attention in 64 bits over the rotated rows."""
    tk = binding()
    B, N_q, N_kv, D, num, width, room = 5, 8, 2, 64, 60, 12, 700
    cache = tk.PagedKVCache(tk.make_paged_config(1, N_q, N_kv, D, num, B, torch.bfloat16))
    rope = tk.Rope(D, torch.bfloat16, theta=500000.0, scaling=tk.ROPE_BANDS, factor=8.0, trained=8192.0)
    freq, m = ko.rope_frequencies(D, 500000.0, "bands", factor=8.0, trained=8192.0)
    table, lens = torch.full((B, width), -1, dtype=torch.int32, device="cuda"), torch.zeros(B, dtype=torch.int32, device="cuda")
    free, count = torch.arange(num, dtype=torch.int32, device="cuda"), ints([num])
    change, plan = torch.zeros(B, dtype=torch.int32, device="cuda"), tk.PagePlan(B, room)
    q, k, v = (torch.zeros(room, 1, n, D, dtype=torch.bfloat16, device="cuda") for n in (N_q, N_kv, N_kv))
    out = torch.zeros_like(q)

    def step():
        cache.plan(change, lens, table, free, count, in_place=True, out=plan)
        rope.apply(q, k, plan.token_pos)
        cache.write_slots(k, v, plan.slots)
        cache.prompt_attn(q, table, plan.pos, rows=plan.rows, start=plan.start, out=out)

    step()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        step()
    keys, vals, g = [[] for _ in range(B)], [[] for _ in range(B)], gen(4)
    for wanted in ([100, 0, 64, 1, 300], [1, 200, 1, 1, -40], [1, 1, -64, 65, 1]):
        total = sum(max(w, 0) for w in wanted)
        raw = [torch.randn(room, 1, n, D, generator=g, device="cuda").to(torch.bfloat16) for n in (N_q, N_kv, N_kv)]
        for x, y in zip((q, k, v), raw):
            x.copy_(y)
        change.copy_(ints(wanted))
        out.fill_(7)
        graph.replay()
        assert plan.rows.tolist() == [max(w, 0) for w in wanted] and int(plan.start[B]) == total and cache.device_error() == 0
        assert torch.equal(q[total:], raw[0][total:]) and (out[total:] == 7).all()
        pos = plan.token_pos.tolist()
        at = 0
        for b, w in enumerate(wanted):
            if w < 0:
                keys[b], vals[b] = keys[b][:max(0, len(keys[b]) + w)], vals[b][:max(0, len(vals[b]) + w)]
            for s in range(max(w, 0)):
                i = at + s
                assert pos[i] == len(keys[b])
                y = ko.rope(raw[1][i, 0].double().cpu().numpy(), pos[i], freq, m, D, "halves")
                assert np.abs((y - k[i, 0].double().cpu().numpy()).astype(float)).max() <= 2.0 ** -7 * float(np.abs(y).max())
                keys[b].append(k[i, 0].double().cpu().numpy())
                vals[b].append(v[i, 0].double().cpu().numpy())
                if s % 37 == 0 or s == w - 1:
                    kk, vv = np.stack(keys[b]), np.stack(vals[b])
                    for h in range(N_kv):
                        hs = slice(4 * h, 4 * h + 4)
                        want, wl, sizes = po.attention(q[i, 0, hs].double().cpu().numpy(), kk[:, h], vv[:, h], D ** -0.5)
                        sizes["vmax"] = np.abs(vv).max()
                        tol, half, _ = bounds(sizes, len(kk), D, torch.bfloat16, wl)
                        assert (np.abs(out[i, 0, hs].double().cpu().numpy() - want) <= tol + half * (np.abs(want) + tol)).all()
            at += max(w, 0)
        assert lens.tolist() == [len(x) for x in keys]
    last = torch.randn(B, 1, N_q, D, generator=g, device="cuda").to(torch.bfloat16)
    got = cache.decode_attn(last, table, lens)
    for b in range(B):
        if keys[b]:
            want, _, _ = po.attention(last[b, 0, :4].double().cpu().numpy(), np.stack(keys[b])[:, 0], np.stack(vals[b])[:, 0], D ** -0.5)
            assert np.abs(got[b, 0, :4].double().cpu().numpy() - want).max() < 0.02


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("rows,held,N_kv,L", [
    ([5], [9000], 1, 1),                                       # one item over all CTAs
    ([4, 4, 4], [3000, 3001, 2950], 2, 1),                     # items of CTAs of their own
    ([1 + 7 * b % 90 for b in range(23)], [(311 * b) % 700 for b in range(23)], 4, 2),         # more items than CTAs
    ([3, 1] + [2] * 30, [6000, 5] + [10 * b for b in range(30)], 1, 2),                       # fewer, one of them long
], ids=["one", "alike", "many", "unlike"])
def test_ways_in_which_work_is_cut(fmt, dtype, rows, held, N_kv, L):
    p = Prompt(fmt, dtype, rows, held, D=128, N_kv=N_kv, G=4, L=L, seed=9)
    out, lse = p.call()
    p.check(out, lse, lambda b, s: s in (0, rows[b] - 1) or (s % 40 == 0 and b % 3 == 0))
    assert p.cache.device_error() == 0
    again = p.call()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])
