"""GPU tests of packed batches at the ends of their ranges: the longest sequences, the largest and smallest values and scales, the
batch sizes at which a launch changes its form.  Bounds as in test_gpu_prompt."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
from test_gpu_packed import check_rope, make_rope
from test_gpu_prompt import FMT, IDS, KINDS, PAGE, Prompt, binding, bounds, gen, ints

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("fmt", ["plain", "int4"])
def test_items_that_take_seconds(fmt):
    """148 items of 268 million tokens, one a block (the table names one page again and again): warps wait for longer than any wait
    without a tile may last.  Only the sum of the softmax is looked at; outputs of so many equal addends carry (n + 16) u."""
    tk = binding()
    N, D, pages = 148, 64, 1 << 22
    cache = tk.PagedKVCache(tk.make_paged_config(1, N, N, D, 1, 1, torch.bfloat16, FMT[fmt]))
    g = gen(1)
    k, v = (torch.randn(1, PAGE, 1, N, D, generator=g, device="cuda").to(torch.bfloat16) for _ in range(2))
    one = ints([[0]])
    cache.write(k, v, one)
    q = torch.randn(1, 1, 1, N, D, generator=g, device="cuda").to(torch.bfloat16)
    _, short = cache.prompt_attn(q, one, ints([PAGE - 1]), return_lse=True)
    table = torch.zeros(1, pages, dtype=torch.int32, device="cuda")
    a, b = (torch.cuda.Event(enable_timing=True) for _ in range(2))
    a.record()
    _, lse = cache.prompt_attn(q, table, ints([pages * PAGE - 1]), return_lse=True)
    b.record()
    b.synchronize()
    assert cache.device_error() == 0
    assert a.elapsed_time(b) > 1200                      # (2e9 cycles are 1.02 s at 1965 MHz)
    # the sum keeps what its additions lose, so only its own few roundings count: exp2 2^-21, log and its product 4 u |lse|
    assert (lse - short - 22 * np.log(2.0)).abs().max() <= 2 * (2.0 ** -20 + 4 * 2.0 ** -23 * float(lse.abs().max()))


PLAN_SIZES = r"""
import sys
sys.path[:0] = sys.argv[1:]
import torch
from test_gpu_packed import check_plan, small_cache, Step
for B in (3040, 3055, 3056, 3071, 3073, 3056, 4096):
    step = Step([b % 130 for b in range(B)], [(b * 7) % 5 - 1 for b in range(B)], 3, 900, 2 * B)
    cache = small_cache(step.num_pages, B)
    change, lens, table, free_pages, count = step.upload()
    check_plan(cache.plan(change, lens, table, free_pages, count, step.max_tokens), table, free_pages, step.want())
print("fine")
"""


def test_plan_around_48_kb_of_shared_memory():
    """In a process of its own: a larger call before may not be what makes one work."""
    tests = os.path.dirname(os.path.abspath(__file__))
    r = subprocess.run([sys.executable, "-c", PLAN_SIZES, tests, os.path.dirname(tests)], capture_output=True, text=True, timeout=300)
    assert r.returncode == 0 and r.stdout.split() == ["fine"], r.stdout + r.stderr


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("value", [2.0 ** 127, -1.75 * 2.0 ** 126])
@pytest.mark.parametrize("N_kv,G", [(1, 4), (160, 1)], ids=["a tile a block", "an item a block"])
def test_large_values_at_logits_above_those_before(fmt, dtype, value, N_kv, G):
    """A token in the second tile has a weight of e^4 relative to all tokens of the first, and a value next to the type's largest: its
    share is 0.3 of that value, whatever the weights are relative to on the way."""
    t, n = 90, 120

    def keys(k):
        k[:] = 0
        k[0, t] = 2.0

    def values(v):
        v[0, t, 0, :, 5] = value

    p = Prompt(fmt, dtype, [n], [0], N_kv=N_kv, G=G, D=64, k_edit=keys, v_edit=values)
    p.q.fill_(0.25)
    out, lse = p.call()
    p.check(out, lse, lambda b, s: s < 4 or s >= t - 2)
    share = out[t:, 0, :, 5].double() / value
    assert (share > 0.25).all() and (share < 0.45).all()


@pytest.mark.parametrize("D", [64, 128])
@pytest.mark.parametrize("sign", [1, -1])
def test_largest_values_in_4_bits(D, sign):
    """A group whose largest magnitude is bf16's largest number: 7 s lies above it by 2^-9 of itself.  Rows in front of the token
    are as without it, in keys and in values; rows that see the value are what the formula gives."""
    t, most = 40, sign * torch.finfo(torch.bfloat16).max

    def edit(x):
        x[0, t, 0, 0, 5] = most

    clean = Prompt("int4", torch.bfloat16, [100], [0], N_kv=1, G=4, D=D)
    want, wl = clean.call()
    for which in ("k_edit", "v_edit"):
        p = Prompt("int4", torch.bfloat16, [100], [0], N_kv=1, G=4, D=D, **{which: edit})
        out, lse = p.call()
        assert torch.equal(out[:t], want[:t]) and torch.equal(lse[:t], wl[:t]), which
        if which == "v_edit":
            assert torch.equal(lse, wl)
            p.check(out, lse, lambda b, s: s >= t - 1)


def test_4_bit_values_past_32_bits_that_a_program_stored():
    """Code 0 stands for -8, which no written row has: -8 times a scale of 1.75 * 2^125 is -1.75 * 2^128.  Rows in front of the token are
    as without it; of the others those are compared whose outputs fit their type."""
    tk = binding()
    t, G, D = 40, 4, 64
    p = Prompt("int4", torch.bfloat16, [100], [0], N_kv=1, G=G, D=D)
    want, wl = p.call()
    page = int(p.table[0, 0])
    code, scale = (tk.paged_offset(p.cfg, 0, page, 0, t, part) for part in (tk.PART_V, tk.PART_V_SCALE))
    p.pool[code + 2] = 0
    p.pool[scale:scale + 2] = torch.tensor([0x60, 0x7e], dtype=torch.uint8, device="cuda")
    p.k, p.v = p.exact_int4()
    assert float(p.v[0, t].abs().max()) == 1.75 * 2.0 ** 128
    out, lse = p.call()
    assert torch.equal(out[:t], want[:t]) and torch.equal(lse, wl)
    assert out[t:].isnan().sum() == 0
    seen = 0
    for s in range(t, 100):
        exact, el, sizes = po.attention(*(x.double().cpu().numpy() for x in (p.q[s, 0], p.k[0, :s + 1, 0, 0], p.v[0, :s + 1, 0, 0])), p.scale)
        sizes["vmax"] = float(p.v.abs().max())
        tol, half, _ = bounds(sizes, s + 1, D, torch.bfloat16, el)
        fits = (np.abs(exact) < 2.0 ** 127).all(1) & (sizes["absv"] < 2.0 ** 127).all(1)
        err = np.abs(out[s, 0].double().cpu().numpy() - exact)
        assert (err <= tol + half * (np.abs(exact) + tol))[fits].all()
        seen += int(fits.sum())
    assert seen > 100


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("scale", [1e4, 1e6, 1e8, 1e9, 1e10, 1e15, 1e25, 1e34])
def test_large_logits(fmt, dtype, scale):
    """Keys and queries of whole numbers, so that products are exact and equal ones equal: with such scales all the weight is on the
    tokens with a row's largest product, in equal shares.  Only roundings of the weights' quotient and of the output are left.
    fp32 caches scale the queries first, which rounds them: equal products of 64 channels come to differ by up to 64 * 2^-24 of
    sums of some 10^2 * scale * 1.44, above 1 for every scale here.  There the general bounds hold, which allow that."""
    g = gen(3)

    def keys(k):
        k.copy_(torch.randint(-7, 8, k.shape, generator=g, device="cuda"))
        k[..., ::32] = 7                       # (4-bit groups then have a scale of 1)

    p = Prompt(fmt, dtype, [150, 4], [30, 4000], N_kv=1, G=4, D=64, k_edit=keys, scale=scale)
    p.q.copy_(torch.randint(-3, 4, p.q.shape, generator=g, device="cuda"))
    out, lse = p.call()
    assert out.isfinite().all() and lse.isfinite().all()
    if dtype == torch.float32:
        with np.errstate(over="ignore"):
            p.check(out, lse, lambda b, s: s % 7 == 0)
        return
    w, half = 2.0 ** -8, torch.finfo(dtype).eps / 2
    for b in range(2):
        for s in range(p.rows[b]):
            n = p.held[b] + s + 1
            q, k, v = p.at(p.q, b)[s, 0].double(), p.k[b, :n, 0, 0].double(), p.v[b, :n, 0, 0].double()
            x = q @ k.T
            share = (x == x.max(1, keepdim=True).values).double()
            share /= share.sum(1, keepdim=True)
            want, size = share @ v, share @ v.abs()
            tol = w * size
            assert ((p.at(out, b)[s, 0].double() - want).abs() <= tol + half * (want.abs() + tol)).all(), (b, s)
            top = x.max(1).values * scale      # the logarithm of the number of such tokens, 9 at most, aside
            assert ((p.at(lse, b)[s, 0].double() - top).abs() <= 9 + 2.0 ** -20 * top.abs()).all(), (b, s)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("scale", [1e-5, 1e-30, 1e-42])
def test_small_scales(fmt, dtype, scale):
    """Some rows see nothing in pieces of their item in which others do."""
    p = Prompt(fmt, dtype, [70, 3], [30, 200], N_kv=1, G=4, D=64, scale=scale)
    out, lse = p.call()
    p.check(out, lse)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("scale", [0.0, 1.0, 2.0 ** -60])
def test_products_past_32_bits(fmt, dtype, scale):
    """A key next to the largest bf16 number: its products with queries pass fp32, its logits do not (those that do, with a scale of 1,
    are infinite in the formula in fp32 as well and not looked at)."""
    t, most = 40, 1.75 * 2.0 ** 127

    def edit(x):
        x[0, t, 0, 0, 5] = most

    p = Prompt(fmt, dtype, [100], [0], N_kv=1, G=4, D=64, k_edit=edit, scale=scale)
    p.q.clamp_(-1.75, 1.75)
    if scale == 1.0:
        p.q[..., 5] *= 0.25
    out, lse = p.call()
    assert out.isfinite().all() and lse.isfinite().all()
    p.check(out, lse, lambda b, s: s < t)
    # Behind it the bounds, relative to such a logit, are infinite.  But it is above or below all others by 2^50 and more, so a row
    # holds that token's value, or what it would hold without that token.
    q, k, v = (x.double().cpu().numpy() for x in (p.q[:, 0], p.k[0, :, 0, 0], p.v[0, :, 0, 0]))
    half = torch.finfo(dtype).eps / 2
    for s in range(t, 100):
        for g in range(4):
            x = float(q[s, g] @ k[t]) * p.scale
            assert abs(x) > 2.0 ** 50
            others = [i for i in range(s + 1) if i != t]
            if x > 0:
                want, wl, tol, ltol = v[t], x, 2.0 ** -8 * np.abs(v[t]), 2.0 ** -20 * abs(x)
            else:
                want, wl, sizes = po.attention(q[s, g:g + 1], k[others], v[others], p.scale)
                sizes["vmax"] = np.abs(v).max()
                tol, _, ltol = bounds(sizes, s + 1, 64, dtype, wl)
                want, wl, tol, ltol = want[0], wl[0], tol[0], ltol[0]
            assert (np.abs(out[s, 0, g].double().cpu().numpy() - want) <= tol + half * (np.abs(want) + tol)).all(), (s, g)
            assert abs(float(lse[s, 0, g]) - wl) <= ltol, (s, g)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("scale", [1e-46, 1e-60, 1e-300])
def test_scales_next_to_nothing(fmt, dtype, scale):
    p = Prompt(fmt, dtype, [70, 3], [30, 200], N_kv=1, G=4, D=64, scale=scale)
    out, lse = p.call()
    p.check(out, lse)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("value", [float("inf"), float("nan")])
@pytest.mark.parametrize("held", [20, 300, 9000])
def test_values_that_are_not_finite_at_weights_of_next_to_nothing(fmt, dtype, value, held):
    """The first tokens, up to 200 of them, have logits hundreds of powers of two below the others: a NaN or an infinity among them is
    in the output of all rows, whether their item is one piece or cut, and whether it shares a piece with heavier ones or not."""
    def keys(k):
        k[:] = 1.0
        k[0, :min(200, held - 8)] = -8.0

    def values(v):
        v[0, 10, 0, 0, 7] = value

    clean = Prompt(fmt, dtype, [5], [held], N_kv=1, G=4, D=64, k_edit=keys)
    p = Prompt(fmt, dtype, [5], [held], N_kv=1, G=4, D=64, k_edit=keys, v_edit=values)
    for x in (clean, p):
        x.q.abs_().add_(1.0)
    (want, wl), (out, lse) = clean.call(), p.call()
    bad = slice(0, 64) if fmt == "e4m3" else slice(0, 32) if fmt == "int4" else slice(7, 8)       # (a quantised row or group is all NaN)
    assert not out[..., bad].isfinite().any()
    keep = [c for c in range(64) if not bad.start <= c < bad.stop]
    assert torch.equal(out[..., keep], want[..., keep]) and torch.equal(lse, wl)


@pytest.mark.parametrize("S", [2 ** 31 - 64, 2 ** 31 - 1])
def test_rope_of_the_longest_axis(S):
    """34 GB of rows of 16 bytes; a block has 64 of them, so the last numbers of rows round up past 2^31."""
    r, freq, m = make_rope(8, torch.bfloat16, 8, "halves", "plain")
    x = torch.empty(1, S, 1, 1, 8, dtype=torch.bfloat16, device="cuda")
    at = [0, 1, 63, 64, 2 ** 30 - 1, 2 ** 30, S - 65, S - 64, S - 2, S - 1]
    rows = torch.randn(len(at), 1, 1, 8, generator=gen(1), device="cuda").to(torch.bfloat16)
    for i, s in enumerate(at):
        x[0, s] = rows[i]
    r.apply(x, None, ints([0]))
    got = torch.stack([x[0, s] for s in at])
    check_rope(rows[None], got[None], [at], [[True] * len(at)], torch.bfloat16, 8, "halves", freq, m, False)


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("B,most,held", [(33, 40, 300), (64, 3, 90), (65, 90, 40), (129, 20, 200), (1000, 2, 70)])
def test_batches_of_more_sequences_than_lanes(fmt, dtype, B, most, held):
    """A lane of the warp that looks for a block's place has several sequences, some without rows; first and last rows of all."""
    r = np.random.default_rng(B)
    rows = r.integers(0, most + 1, B)
    rows[r.random(B) < 0.3] = 0
    rows[[0, B - 1]] = 0, most
    rows, before = rows.tolist(), r.integers(0, held + 1, B).tolist()
    p = Prompt(fmt, dtype, rows, before, N_kv=1, G=2, D=64, packed=B % 2 == 1, seed=B)
    out, lse = p.call()
    p.check(out, lse, lambda b, s: s in (0, rows[b] - 1))
    assert p.cache.device_error() == 0
    again = p.call()
    assert torch.equal(out, again[0]) and torch.equal(lse, again[1])


@pytest.mark.parametrize("fmt,dtype", KINDS[:3], ids=IDS[:3])
def test_a_token_of_each_of_4096_sequences(fmt, dtype):
    B = 4096
    r = np.random.default_rng(2)
    before = r.integers(0, 130, B).tolist()
    p = Prompt(fmt, dtype, [1] * B, before, N_kv=1, G=1, D=64)
    out, lse = p.call()
    p.check(out, lse, lambda b, s: b % 5 == 0 or b > B - 40)
    want, wl = p.cache.decode_attn(p.q, p.table, p.pos + 1, return_lse=True)
    vmax = float(p.v.abs().max())
    assert (out.double() - want.double()).abs().max() <= vmax * (2.0 ** -7 if dtype == torch.bfloat16 else 2.0 ** -13)
    assert (lse - wl).abs().max() <= 2.0 ** -13


@pytest.mark.parametrize("fmt,dtype", KINDS, ids=IDS)
@pytest.mark.parametrize("G", [3, 4, 8])
def test_last_rows_of_every_sequence(fmt, dtype, G):
    """The last item of a sequence is not full, and the next sequence's rows follow it at once."""
    rows, held = [33, 1, 70, 2, 86, 64, 5, 257], [100, 0, 64, 500, 1, 0, 63, 10]
    p = Prompt(fmt, dtype, rows, held, N_kv=1, G=G, D=128, seed=G)
    out, lse = p.call()
    p.check(out, lse, lambda b, s: s >= rows[b] - 3)


@pytest.mark.parametrize("fmt,dtype", [KINDS[0], KINDS[2], KINDS[3]], ids=[IDS[0], IDS[2], IDS[3]])
@pytest.mark.parametrize("scale,grow", [(1e-3, 0), (1e6, 0), (1e9, 0), (1e25, 0), (1.0, 10), (100.0, 14), (1e-4, 14)])
def test_large_logits_in_pieces_of_many_tiles(fmt, dtype, scale, grow):
    """More items than blocks, six tiles each; with `grow` the keys of a tile are 2^grow times those of the tile before, so that a row's
    largest logit passes through all sizes.  Whole numbers times powers of two: products are exact, and from some size on all of the
    weight is on the largest."""
    N, n, g = 150, 384, gen(5)

    def keys(k):
        k.copy_(torch.randint(-7, 8, k.shape, generator=g, device="cuda"))
        k[..., ::32] = 7                       # (4-bit groups then have a power of two as scale)
        k *= 2.0 ** (grow * (torch.arange(k.shape[1], device="cuda") // PAGE)[None, :, None, None, None])

    p = Prompt(fmt, dtype, [8], [n - 8], N_kv=N, G=1, D=64, k_edit=keys, scale=scale)
    p.q.copy_(torch.randint(-3, 4, p.q.shape, generator=g, device="cuda"))
    out, lse = p.call()
    half = torch.finfo(dtype).eps / 2
    for s in range(8):
        m = n - 8 + s + 1
        q, k, v = p.q[s, 0].double(), p.k[0, :m, 0].double(), p.v[0, :m, 0].double()
        x = torch.einsum("hd,nhd->hn", q, k) * scale
        w = torch.softmax(x, 1)
        want, size = torch.einsum("hn,nhd->hd", w, v), torch.einsum("hn,nhd->hd", w, v.abs())
        # A logit x = scale * product carries the scale's rounding, its own and the reference's, 2^-22 |x| with room: that counts where
        # tokens other than the largest have weight.  Equal products stay equal.
        top = x.max(1, keepdim=True).values
        near = ((x > top - 40) & (x < top)).any(1)                   # others that carry weight
        err = torch.where(near, 2.0 ** -22 * (top.squeeze(1).abs() + 40), torch.zeros_like(top.squeeze(1)))
        tol = (2.0 ** -8 + 2.0 ** -13 + torch.expm1(2 * err))[:, None] * size
        assert ((out[s, 0].double() - want).abs() <= tol + half * (want.abs() + tol)).all(), s
        wl = torch.logsumexp(x, 1)
        assert ((lse[s, 0].double() - wl).abs() <= err + 2.0 ** -10 + 2.0 ** -20 * wl.abs() + (top.squeeze(1).abs() > 2.0 ** 26) * 9).all(), s
