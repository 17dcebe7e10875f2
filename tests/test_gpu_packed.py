"""GPU tests of packed batches: plans and slots equal to the oracle's, rotary positions within bounds counted in roundings."""
import numpy as np
import pytest
import torch

from oracle import packed_oracle as ko

pytestmark = pytest.mark.gpu

PAGE = 64
FMT = {"plain": 0, "e4m3": 1, "int4": 2}


def binding():
    from paper_2407_21018_b200 import binding as tk
    return tk


def gen(seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    return g


def ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def small_cache(num_pages, B, L=1, N_kv=1, N_q=1, D=64, dtype=torch.bfloat16, fmt="plain", **kw):
    tk = binding()
    return tk.PagedKVCache(tk.make_paged_config(L, N_q, N_kv, D, num_pages, B, dtype, FMT[fmt]), **kw)


# ---------------------------------------------------------------------------
# plans
# ---------------------------------------------------------------------------
class Step:
    """Lists of a step: tables filled from a shuffled pool, the rest of the pool free."""

    def __init__(self, lens, change, width, free, max_tokens, seed=0, num_pages=None):
        r = np.random.default_rng(seed)
        need = [ko.pages_of(n) for n in lens]
        used = sum(need)
        self.num_pages = num_pages or max(1, used + free)
        order = r.permutation(used + free).tolist()
        self.table, at = [], 0
        for n in need:
            self.table.append(order[at:at + n] + [-1 - j for j in range(width - n)])
            at += n
        self.lens, self.change, self.max_tokens = list(lens), list(change), max_tokens
        self.free_pages = order[used:] + [-1] * (self.num_pages - free)
        self.free_count = free

    def want(self):
        return ko.plan(self.table, self.lens, self.change, self.free_pages, self.free_count, self.max_tokens, self.num_pages)

    def upload(self, extra_columns=0):
        wide = ints([r + [77] * extra_columns for r in self.table])
        return ints(self.change), ints(self.lens), wide[:, :len(self.table[0])], ints(self.free_pages), ints([self.free_count])


def check_plan(got, table, free_pages, want):
    assert int(got.free_count) == want["free_count"]
    for name in ("pos", "rows", "start", "seq_lens", "token_pos", "slots"):
        assert getattr(got, name).tolist() == want[name], name
    assert table.tolist() == want["table"]
    assert free_pages.tolist() == want["free_pages"]


STEPS = {
    "one": Step([0], [1], 1, 1, 1),
    "one page border": Step([64], [1], 2, 1, 5),
    "nothing asked": Step([5, 0, 64], [0, 0, 0], 3, 2, 4),
    "no free page": Step([5, 64, 0], [3, 1, 2], 3, 0, 9),
    "freed in the same call": Step([130, 64, 10], [-1000, 65, -3], 3, 0, 65),
    "more given than taken": Step([640, 1, 300], [-640, 0, -257], 12, 3, 8),
    "exactly enough": Step([64, 64, 64], [64, 64, 1], 4, 3, 129),
    "one too few": Step([64, 64, 64, 64], [64, 64, 1, 0], 4, 2, 129),
    "none needed behind a refusal": Step([64, 64, 63, 3], [640, 64, 1, 5], 12, 2, 999),
    "room for tokens": Step([1, 2, 3, 4], [5, 6, 7, 1], 4, 9, 11),
    "past the table": Step([100, 1], [29, 3], 2, 9, 50),
    "table full": Step([128, 1], [0, 127], 2, 9, 127),
    "odd sizes": Step([0, 1, 63, 64, 65, 127, 128, 129] * 5, [1, 64, 1, 1, 63, 0, -1, -65] * 5, 4, 50, 1001, seed=3),
    "long": Step([70000, 1], [66001, 3], 2200, 1100, 70001, seed=4),
}


@pytest.mark.parametrize("name", STEPS)
def test_plan(name):
    step = STEPS[name]
    cache = small_cache(step.num_pages, 64)
    change, lens, table, free_pages, count = step.upload(extra_columns=2)
    want = step.want()
    got = cache.plan(change, lens, table, free_pages, count, step.max_tokens)
    check_plan(got, table, free_pages, want)
    assert lens.tolist() == step.lens and int(count) == step.free_count         # inputs stay
    assert cache.device_error() == (16 if want["error"] else 0)
    assert (table._base[:, len(step.table[0]):] == 77).all()
    # the same again gives the same: results lie apart from the inputs
    got = cache.plan(change, lens, table, free_pages, count, out=got)
    assert got.slots.tolist() == want["slots"]


@pytest.mark.parametrize("B,hi,seed", [(1, 1, 0), (255, 300, 1), (256, 40, 2), (257, 700, 3), (1023, 200, 4), (1025, 130, 5),
                                       (4096, 90, 6)])
@pytest.mark.parametrize("share", [1.0, 0.4])
def test_plan_of_many_sequences(B, hi, seed, share):
    r = np.random.default_rng(seed)
    lens = r.integers(0, hi + 1, B).tolist()
    change = [int(-r.integers(0, hi)) if x < 0.25 else int(r.integers(0, hi)) for x in r.random(B)]
    tokens = sum(max(c, 0) for c in change)
    need = sum(max(0, ko.pages_of(n + c) - ko.pages_of(n)) for n, c in zip(lens, change))
    width = max(ko.pages_of(n + max(c, 0)) for n, c in zip(lens, change)) or 1
    step = Step(lens, change, width, int(need * share), max(1, int(tokens * min(1.0, share * 1.5))), seed)
    cache = small_cache(step.num_pages, B)
    change_d, lens_d, table, free_pages, count = step.upload()
    got = cache.plan(change_d, lens_d, table, free_pages, count, step.max_tokens)
    check_plan(got, table, free_pages, step.want())


def test_plan_in_place_over_many_steps():
    """Lengths, table and free list live on the device and are stepped in place, from a captured graph: no page is lost or
    owned twice."""
    B, width, num = 37, 6, 120
    cache = small_cache(num, B)
    tk = binding()
    state = dict(table=[[-1] * width for _ in range(B)], lens=[0] * B, free_pages=list(range(num)), count=num)
    table, lens, free_pages, count = ints(state["table"]), ints(state["lens"]), ints(state["free_pages"]), ints([num])
    change, plan = torch.zeros(B, dtype=torch.int32, device="cuda"), tk.PagePlan(B, 900)
    call = lambda: cache.plan(change, lens, table, free_pages, count, in_place=True, out=plan)  # noqa: E731
    call()
    torch.cuda.synchronize()
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        call()
    r = np.random.default_rng(8)
    for step in range(60):
        c = [int(x) for x in r.integers(-150, 120, B)]
        change.copy_(ints(c))
        graph.replay()
        want = ko.plan(state["table"], state["lens"], c, state["free_pages"], state["count"], 900, num)
        assert lens.tolist() == want["seq_lens"] and int(count) == want["free_count"], step
        assert plan.slots.tolist() == want["slots"] and table.tolist() == want["table"]
        state = dict(table=want["table"], lens=want["seq_lens"], free_pages=want["free_pages"], count=want["free_count"])
        owned = [p for row, n in zip(state["table"], state["lens"]) for p in row[:ko.pages_of(n)]] + state["free_pages"][:state["count"]]
        assert sorted(owned) == list(range(num))
    assert plan.seq_lens is lens


def test_plan_of_bad_inputs_stays_in_its_arrays():
    """Lengths past the table, a free list that claims more than there is, pages outside the pool."""
    for lens, change, count, page in (([500, 3], [1, 70], 3, 0), ([0, -9], [4, 4], 99, 0), ([0, 5], [64, 64], -5, 0), ([64, 64], [-64, 100], 2, 999)):
        step = Step([128, 64], change, 3, 3, 200, num_pages=9)
        step.lens, step.free_count = lens, count
        step.table[0][0] = step.table[0][0] if page == 0 else page
        cache = small_cache(9, 2)
        change_d, lens_d, table, free_pages, c = step.upload(extra_columns=1)
        guard = torch.full((64,), 5, dtype=torch.int32, device="cuda")
        guard[16:25] = free_pages
        got = cache.plan(change_d, lens_d, table, guard[16:25], c, 200)
        want = step.want()
        assert cache.device_error() == 16 and want["error"]
        assert (guard[:16] == 5).all() and (guard[25:] == 5).all() and (table._base[:, 3:] == 77).all()
        assert got.rows.tolist() == want["rows"] and got.slots.tolist() == want["slots"] and table.tolist() == want["table"]


# ---------------------------------------------------------------------------
# rows by slots
# ---------------------------------------------------------------------------
@pytest.mark.parametrize("fmt,dtype", [("plain", torch.bfloat16), ("plain", torch.float32), ("e4m3", torch.bfloat16), ("int4", torch.bfloat16)])
@pytest.mark.parametrize("D,N_kv,L,T", [(128, 8, 2, 300), (64, 3, 1, 65), (128, 1, 1, 1), (64, 12, 3, 130)])
def test_rows_by_slots_are_rows_by_table(fmt, dtype, D, N_kv, L, T):
    """The same bytes as the padded write leaves, and nothing else touched; rows without a slot go nowhere."""
    pages = -(-T // PAGE) + 3
    g = gen(T)
    k, v = (torch.randn(T, L + 1, N_kv, D, generator=g, device="cuda").to(dtype)[:, 1:] for _ in range(2))
    pools = [torch.full((int(binding().paged_bytes(small_cache(pages, 1, L, N_kv, N_kv, D, dtype, fmt).cfg).pages),), 255, dtype=torch.uint8,
                        device="cuda") for _ in range(2)]
    a, b = (small_cache(pages, 1, L, N_kv, N_kv, D, dtype, fmt, pages=p) for p in pools)
    table = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)[None]
    pos = 37
    a.write(k[None], v[None], table, pos=ints([pos]))
    t = torch.arange(pos, pos + T, device="cuda")
    slots = (table[0, t // PAGE] * PAGE + t % PAGE).to(torch.int32)
    b.write_slots(k, v, slots)
    assert torch.equal(pools[0], pools[1]) and b.device_error() == 0
    # permuted, some left out, some behind the pool
    pools[1].fill_(255)
    order = torch.randperm(T, generator=g, device="cuda")
    some = slots[order].clone()
    some[::3] = -1 - some[::3]
    b.write_slots(k[order], v[order], some)
    assert b.device_error() == 0
    pools[0].fill_(255)
    kept = torch.nonzero(some >= 0).squeeze(1)
    a.write_slots(k[order][kept].contiguous(), v[order][kept].contiguous(), some[kept].contiguous())
    assert torch.equal(pools[0], pools[1])
    before = pools[1].clone()
    b.write_slots(k[:1], v[:1], ints([pages * PAGE]))
    assert b.device_error() == 16 and torch.equal(before, pools[1])
    b.write_slots(k[:0], v[:0], slots[:0])


# ---------------------------------------------------------------------------
# rotary positions
# ---------------------------------------------------------------------------
def rope_tolerance(x, y, dtype, R, layout, m):
    """Error of a turned element: the angle is off by 2^-27 turns = 2 pi 2^-27 < 2^-24, sine and cosine by two units of
    2^-24 each, m's rounding, its product with them, two products and a sum by half a unit of 2^-24 each, all relative to
    m (|a| + |b|): (1 + 2 + 4 / 2 + 1) 2^-24 < 2^-21.  Then the rounding to the output's type, half a step of |y|."""
    x = np.abs(x.astype(np.float64))
    i, j = (slice(0, R // 2), slice(R // 2, R)) if layout == "halves" else (slice(0, R, 2), slice(1, R, 2))
    pair = np.zeros_like(x)
    pair[..., i] = pair[..., j] = x[..., i] + x[..., j]
    tol = float(m) * pair * 2.0 ** -21
    half = torch.finfo(dtype).eps / 2
    tol = tol + half * (np.abs(y.astype(np.float64)) + tol)
    tol[..., R:] = 0
    return tol


def check_rope(x, got, pos, on, dtype, R, layout, freq, m, transpose, what=""):
    """x, got [b, s, l, n, D] tensors; pos [b][s]; rows with on false have to be as `got` had them before (zero here)."""
    x64, g64 = x.double().cpu().numpy(), got.double().cpu().numpy()
    for b in range(x.shape[0]):
        for s in range(x.shape[1]):
            if not on[b][s]:
                assert (g64[b, s] == 0).all()
                continue
            y = ko.rope(x64[b, s], pos[b][s], freq, m, R, layout, transpose)
            err = np.abs((y - g64[b, s]).astype(np.float64))
            tol = rope_tolerance(x64[b, s], y, dtype, R, layout, m)
            assert (err <= tol).all(), f"{what} {(b, s, pos[b][s])}: {err.max():.3g}, {(err / np.maximum(tol, 1e-300)).max():.3g} of the bound"


SCALINGS = {"plain": {}, "linear": dict(factor=4.0), "ntk": dict(factor=8.0), "yarn": dict(factor=16.0, trained=4096.0),
            "bands": dict(factor=8.0, trained=8192.0)}


def make_rope(D, dtype, R, layout, scaling, theta=10000.0, **kw):
    tk = binding()
    code = {"plain": tk.ROPE_PLAIN, "linear": tk.ROPE_LINEAR, "ntk": tk.ROPE_NTK, "yarn": tk.ROPE_YARN, "bands": tk.ROPE_BANDS}[scaling]
    args = dict(SCALINGS[scaling], **kw)
    r = tk.Rope(D, dtype, rot_dim=R, layout=tk.ROPE_HALVES if layout == "halves" else tk.ROPE_PAIRS, theta=theta, scaling=code, **args)
    freq, m = ko.rope_frequencies(R, theta, scaling, **args)
    return r, freq, m


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("D,R,scaling", [(128, 128, "plain"), (64, 64, "bands"), (128, 32, "yarn"), (64, 20, "linear"), (64, 8, "ntk"),
                                         (8, 2, "plain"), (256, 256, "linear"), (96, 48, "yarn"), (72, 70, "bands")])
def test_rope(dtype, layout, D, R, scaling):
    r, freq, m = make_rope(D, dtype, R, layout, scaling)
    for j in range(R // 2):
        assert abs(r.frequency(j) - float(freq[j])) <= 2.0 ** -52 * float(freq[j])
    assert r.frequency(R // 2) == -1 and r.frequency(-1) == -1
    g = gen(D + R)
    q = torch.randn(3, 5, 2, 3, D, generator=g, device="cuda").to(dtype)
    k = torch.randn(3, 5, 2, 1, D, generator=g, device="cuda").to(dtype)
    pos = [0, 4093, 1048573]
    every = [[p + s for s in range(5)] for p in pos]
    for transpose in (False, True):
        for rows in (None, [5, 0, 3]):
            qo, ko_ = torch.zeros_like(q), torch.zeros_like(k)
            r.apply(q, k, ints(pos), rows=None if rows is None else ints(rows), q_out=qo, k_out=ko_, transpose=transpose)
            on = [[rows is None or s < rows[b] for s in range(5)] for b in range(3)]
            check_rope(q, qo, every, on, dtype, R, layout, freq, m, transpose, "q")
            check_rope(k, ko_, every, on, dtype, R, layout, freq, m, transpose, "k")
    # in place, alone, by every row's own position: the same bits
    order = [[7, 0, 2 ** 31 - 1, -1, 99999], [1, 1, 1, 1, 1], [12345678, 5, -2 ** 31, 0, 6]]
    qo = torch.zeros_like(q)
    r.apply(q, None, ints(order), q_out=qo)
    check_rope(q, qo, order, [[p >= 0 for p in x] for x in order], dtype, R, layout, freq, m, False, "own positions")
    q2 = q.clone()
    assert r.apply(q2, None, ints(order))[0] is q2
    keep = torch.tensor(order, device="cuda") < 0
    assert torch.equal(q2, torch.where(keep[:, :, None, None, None], q, qo))
    k2, q3 = k.clone(), q.clone()
    r.apply(q3, k2, ints(pos))
    q4 = q.clone()
    r.apply(None, k.clone(), ints(pos))
    r.apply(q4, None, ints(pos))
    assert torch.equal(q3, q4)
    # packed: one axis of tokens
    flat = ints([p for x in order for p in x])
    q5 = q.reshape(15, 2, 3, D).clone()
    r.apply(q5, None, flat)
    assert torch.equal(q5.reshape(q.shape), q2)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_rope_of_strided_views(layout):
    """q, k inside one tensor of projections, permuted and padded views, repeated rows, many heads and layers."""
    dtype, D, R = torch.bfloat16, 64, 64
    r, freq, m = make_rope(D, dtype, R, layout, "plain")
    qkv = torch.randn(2, 70, 1, 7 * D, generator=gen(1), device="cuda").to(dtype)
    q, k = (qkv[..., a * D:b * D].unflatten(-1, (-1, D)) for a, b in ((0, 4), (4, 5)))
    before = qkv.clone()
    pos = ints([3, 1000])
    qo, ko_ = torch.zeros(2, 70, 1, 4, D, dtype=dtype, device="cuda"), torch.zeros(2, 70, 1, 1, D, dtype=dtype, device="cuda")
    r.apply(q, k, pos, q_out=qo, k_out=ko_)
    assert torch.equal(qkv, before)
    every = [[p + s for s in range(70)] for p in (3, 1000)]
    on = [[True] * 70] * 2
    check_rope(q, qo, every, on, dtype, R, layout, freq, m, False)
    check_rope(k, ko_, every, on, dtype, R, layout, freq, m, False)
    r.apply(q, k, pos)
    assert torch.equal(q, qo) and torch.equal(k, ko_) and torch.equal(qkv[..., 5 * D:], before[..., 5 * D:])
    perm = torch.randn(3, 2, 5, 40, D, generator=g2(), device="cuda").to(dtype).permute(1, 3, 0, 2, 4)      # [b 2, s 40, l 3, n 5, d]
    out = torch.zeros(2, 40, 3, 5, D, dtype=dtype, device="cuda")
    r.apply(perm, None, pos, q_out=out)
    check_rope(perm, out, [[p + s for s in range(40)] for p in (3, 1000)], [[True] * 40] * 2, dtype, R, layout, freq, m, False)
    one = torch.randn(1, 1, 1, 2, D, generator=g2(), device="cuda").to(dtype).expand(2, 40, 3, 2, D)
    out = torch.zeros(2, 40, 3, 2, D, dtype=dtype, device="cuda")
    r.apply(one, None, pos, q_out=out)
    check_rope(one, out, [[p + s for s in range(40)] for p in (3, 1000)], [[True] * 40] * 2, dtype, R, layout, freq, m, False)


def g2():
    return gen(2)


@pytest.mark.parametrize("layout", ["halves", "pairs"])
def test_rope_gradient(layout):
    """The transposed form is the derivative: against autograd through the formula, and against differences (the map is
    linear, so a difference along any direction is exact up to rounding)."""
    R, D = 16, 24
    r, freq, m = make_rope(D, torch.float32, R, layout, "yarn")
    g = gen(5)
    x = torch.randn(2, 9, 1, 3, D, generator=g, device="cuda")
    gy = torch.randn(x.shape, generator=g, device="cuda")
    pos = ints([11, 70000])
    gx = torch.zeros_like(x)
    r.apply(gy, None, pos, q_out=gx, transpose=True)
    x64 = x.double().requires_grad_()
    at = (pos.long()[:, None] + torch.arange(9, device="cuda")).double()
    t = at[..., None] * torch.tensor([float(f) for f in freq], dtype=torch.float64, device="cuda")
    c, s = (float(m) * t.cos())[:, :, None, None], (float(m) * t.sin())[:, :, None, None]
    a, b = (x64[..., :R // 2], x64[..., R // 2:R]) if layout == "halves" else (x64[..., 0:R:2], x64[..., 1:R:2])
    u, v = a * c - b * s, b * c + a * s
    y = torch.cat((torch.cat((u, v), -1) if layout == "halves" else torch.stack((u, v), -1).flatten(-2), x64[..., R:]), -1)
    (y * gy.double()).sum().backward()
    tol = 2.0 ** -20 * float(m) * 2 * float(gy.abs().max())       # the bound above, with |a| + |b| <= 2 max; frequencies in 64 bits
    assert (gx.double() - x64.grad).abs().max() <= tol
    d = torch.randn(x.shape, generator=g, device="cuda")
    y0, y1 = torch.zeros_like(x), torch.zeros_like(x)
    r.apply(x - d, None, pos, q_out=y0)
    r.apply(x + d, None, pos, q_out=y1)
    slope = ((y1.double() - y0.double()) * gy.double()).sum() / 2
    want = (gx.double() * d.double()).sum()
    n = x.numel()
    assert (slope - want).abs() <= 2.0 ** -20 * float(m) * 6 * float(gy.abs().max()) * float((x.abs() + d.abs()).max()) * n ** 0.5 * 8


def test_rope_captured_and_on_another_stream():
    r, freq, m = make_rope(128, torch.bfloat16, 128, "halves", "plain")
    q = torch.randn(200, 1, 8, 128, generator=gen(3), device="cuda").to(torch.bfloat16)
    pos, out = ints(list(range(200))), torch.zeros_like(q)
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    r.apply(q, None, pos, q_out=out, stream=side)
    side.synchronize()
    graph, again = torch.cuda.CUDAGraph(), torch.zeros_like(q)
    with torch.cuda.graph(graph):
        r.apply(q, None, pos, q_out=again)
    graph.replay()
    assert torch.equal(out, again)
    pos.copy_(ints([5] * 200))
    graph.replay()
    assert not torch.equal(out, again) and torch.equal(out[5], again[5])


@pytest.mark.parametrize("dtype", [torch.bfloat16, torch.float32])
@pytest.mark.parametrize("layout", ["halves", "pairs"])
@pytest.mark.parametrize("D,R", [(24, 24), (56, 16), (40, 8), (88, 64)])
def test_rope_rows_of_an_odd_number_of_pieces(dtype, layout, D, R):
    """5 and 7 pieces of 16 bytes a row, in place (only those that turn) and not."""
    r, freq, m = make_rope(D, dtype, R, layout, "plain")
    x = torch.randn(2, 40, 1, 3, D, generator=gen(D), device="cuda").to(dtype)
    y, z = torch.zeros_like(x), x.clone()
    r.apply(x, None, ints([3, 70000]), q_out=y)
    check_rope(x, y, [[3 + s for s in range(40)], [70000 + s for s in range(40)]], [[True] * 40] * 2, dtype, R, layout, freq, m, False)
    r.apply(z, None, ints([3, 70000]))
    assert torch.equal(y, z)


def test_a_plan_serves_calls_in_place_and_not():
    cache, tk = small_cache(9, 2), binding()
    step = Step([10, 64], [5, 3], 3, 4, 20, num_pages=9)
    change, lens, table, free_pages, count = step.upload()
    plan = tk.PagePlan(2, 20)
    cache.plan(change, lens, table, free_pages, count, in_place=True, out=plan)
    assert plan.seq_lens is lens and lens.tolist() == [15, 67] and plan.free_count is count
    before = lens.clone()
    cache.plan(change, lens, table, free_pages, count, out=plan)
    assert torch.equal(lens, before) and plan.seq_lens.tolist() == [20, 70] and plan.free_count is not count


def test_calls_that_the_binding_refuses():
    tk = binding()
    cache = small_cache(9, 2, L=2, N_kv=2, N_q=4, D=64)
    bf = torch.bfloat16
    table, two = torch.zeros(2, 3, dtype=torch.int32, device="cuda"), torch.zeros(2, dtype=torch.int32, device="cuda")
    x, slots = torch.zeros(5, 2, 2, 64, dtype=bf, device="cuda"), torch.full((5,), -1, dtype=torch.int32, device="cuda")
    q = torch.zeros(2, 5, 2, 4, 64, dtype=bf, device="cuda")
    free_pages = torch.zeros(9, dtype=torch.int32, device="cuda")
    one = free_pages[:1].clone()
    rope = tk.Rope(64, bf)
    calls = [lambda: cache.write_slots(x.float(), x, slots), lambda: cache.write_slots(x, x[:4], slots), lambda: cache.write_slots(x, x, slots[:4]),
             lambda: cache.write_slots(x, x, slots.long()), lambda: cache.write_slots(x, x, slots.cpu()), lambda: cache.write_slots(x, x, slots, layer0=1),
             lambda: cache.write_slots(x[:, :1], x[:, :1], slots), lambda: cache.write_slots(x[..., ::2], x[..., ::2], slots),
             lambda: cache.prompt_attn(q.float(), table), lambda: cache.prompt_attn(q[:, :, :1], table), lambda: cache.prompt_attn(q, table[:1]),
             lambda: cache.prompt_attn(q, table.long()), lambda: cache.prompt_attn(q, table, pos=two[:1]), lambda: cache.prompt_attn(q, table, rows=two.long()),
             lambda: cache.prompt_attn(q, table, out=q), lambda: cache.prompt_attn(q, table, out=q[:, :4]), lambda: cache.prompt_attn(q[0], table, start=two),
             lambda: cache.prompt_attn(q, table, lse=torch.zeros(2, 5, 2, 4, device="cuda", dtype=bf)), lambda: cache.prompt_attn(q, table, scratch=free_pages),
             lambda: cache.prompt_attn(q, table, scratch=torch.zeros(256, dtype=torch.uint8, device="cuda")), lambda: cache.prompt_attn(q, table, layer0=2),
             lambda: cache.plan(two, two, table, free_pages, one), lambda: cache.plan(two, two, table[:1], free_pages, one, 9),
             lambda: cache.plan(two.long(), two.clone(), table, free_pages, one, 9), lambda: cache.plan(two, two.clone(), table, free_pages[:8], one, 9),
             lambda: cache.plan(two, two.clone(), table, free_pages, one, out=tk.PagePlan(3, 9)), lambda: cache.plan(two, two, table, free_pages, one, 9, in_place=True),
             lambda: cache.plan(two, two.clone(), table, free_pages, one, 8, out=tk.PagePlan(2, 9)),
             lambda: cache.plan(two, two.clone(), table, free_pages, free_pages[:1], 9),
             lambda: rope.apply(q.float(), None, two), lambda: rope.apply(q, x, two), lambda: rope.apply(q, None, two.long()), lambda: rope.apply(q, None, two[:1]),
             lambda: rope.apply(q, None, two.cpu()), lambda: rope.apply(q, None, two, rows=two[:1]), lambda: rope.apply(q, None, two, q_out=q[:, :4]),
             lambda: rope.apply(q, None, two, q_out=q.transpose(0, 1).contiguous().transpose(0, 1)[:, :, :1].expand(q.shape))]
    for i, call in enumerate(calls):
        with pytest.raises(tk.ThinKError) as e:
            call()
        assert e.value.status in (tk.ERR_INVALID_ARG, tk.ERR_CAPACITY), i
    assert cache.device_error() == 0


@pytest.mark.parametrize("B", [257, 1000, 1024, 1025])
@pytest.mark.parametrize("share", [1.0, 0.3])
def test_plan_of_a_decode_step_of_many_sequences(B, share):
    r = np.random.default_rng(B)
    lens, change = r.integers(0, 300, B).tolist(), r.choice([1, 1, 1, -70, 0], B).tolist()
    need = sum(max(0, ko.pages_of(max(n + c, 0)) - ko.pages_of(n)) for n, c in zip(lens, change))
    step = Step(lens, change, 6, int(need * share), B)
    cache = small_cache(step.num_pages, B)
    change_d, lens_d, table, free_pages, count = step.upload()
    got = cache.plan(change_d, lens_d, table, free_pages, count, B)
    check_plan(got, table, free_pages, step.want())
