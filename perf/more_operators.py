"""The operators of a packed batch over the paged key-value cache, as a user calls them and in plain form.

A serving step takes the new tokens of many sequences as one packed tensor [token, layer, head, D], sequence after
sequence.  Four operators carry it from the sequences' lengths to the attention's outputs:

    plan    lengths and wanted changes -> pages taken from and given back to a list of free ones, the page table, and for
            every packed token its position and its slot (page * 64 + place in the page)
    rope    rotary positions on queries and keys: pairs (j, j + R/2) or (2j, 2j + 1) of the first R channels turn by
            position * frequency(j); frequencies may be scaled for long contexts; the transposed form takes gradients back
    write   packed rows of keys and values go to the slots of their tokens, quantised on the way
    attn    softmax(scale * q K^T) V of every new token over its sequence's pages up to itself, and the log of its sum

The pool of pages is [layer][page][key head] blocks of 64 key rows | 64 value rows | key scales | value scales, rows of D
elements as they are ("plain"), as e4m3 bytes with a power-of-two exponent byte a row ("e4m3"), or as 4-bit codes, two
channels a byte, with a bf16 scale per 32 channels ("int4").
"""
import math
import random

import torch

own = False

PAGE = 64
GROUP = 32          # channels that share a scale in "int4"


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _plan(name, B, lo, hi, grow_lo, grow_hi, end=0.0, spare=1.0, lens=1):
    """lo..hi: tokens held; grow_lo..grow_hi: tokens wanted; end: share of sequences that give all their pages back;
    spare: free pages as a share of those wanted (below 1 some sequences get none)."""
    return _named(name, dict(op="plan", B=B, lo=lo, hi=hi, grow_lo=grow_lo, grow_hi=grow_hi, end=end, spare=spare, lens=lens))


def _rope(name, B, S, lens, N_q, N_kv, D, R, layout, scaling, dtype, L=1, far=8192, back=False):
    """S: rows of each sequence (packed = their positions given one by one where B is 1); far: largest position."""
    return _named(name, dict(op="rope", B=B, S=S, L=L, N_q=N_q, N_kv=N_kv, D=D, R=R, layout=layout, scaling=scaling,
                             dtype=dtype, far=far, back=back, lens=lens))


def _write(name, fmt, dtype, T, L, N_kv, D, lens=1):
    return _named(name, dict(op="write", format=fmt, dtype=dtype, T=T, L=L, N_kv=N_kv, D=D, lens=lens))


def _attn(name, fmt, dtype, B, L, N_q, N_kv, D, rows_lo, rows_hi, held_lo, held_hi, packed=True, lens=1):
    """rows: new tokens of a sequence; held: tokens it had before."""
    return _named(name, dict(op="attn", format=fmt, dtype=dtype, B=B, L=L, N_q=N_q, N_kv=N_kv, D=D, rows_lo=rows_lo,
                             rows_hi=rows_hi, held_lo=held_lo, held_hi=held_hi, packed=packed, lens=lens))


def _named(name, c):
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # a decode step of 64 sequences: one token each, a new page now and then; latency counts
        _plan("plan step", 64, 1, 8000, 1, 1),
        # continuous batching: a third of 192 sequences ends, the others take prompts, and pages run short
        _plan("plan ragged", 192, 0, 2000, 1, 2000, end=0.3, spare=0.8),
        # a few fp32 rows of the small test geometry, neighbouring channels paired: latency of the smallest call
        _rope("rope f32 rows", 3, 5, 1, 4, 4, 64, 64, "pairs", "none", "f32"),
        # an 8192-token prompt on the LLaMA-3-8B shape, frequencies scaled by bands of wavelengths, long positions
        _rope("rope bf16 prompt", 1, 8192, 2, 32, 8, 128, 128, "halves", "bands", "bf16", far=131072),
        # the gradient's way back through a partial rotation of four layers on the D = 64 shape
        _rope("rope bf16 part back", 7, 1500, 3, 12, 12, 64, 32, "pairs", "yarn", "bf16", L=4, far=32768, back=True),
        # a decode step of a batch of 64 goes to 8-bit pages of 32 layers
        _write("write e4m3 step", "e4m3", "bf16", 64, 32, 8, 128),
        # the prompts of a ragged batch, four layers, unquantised
        _write("write bf16 packed", "plain", "bf16", 20011, 4, 12, 64),
        # a prompt of 8192 tokens from its beginning, LLaMA-3-8B shape: the largest matrix work
        _attn("attn bf16 prompt", "plain", "bf16", 1, 1, 32, 8, 128, 8192, 8192, 0, 0),
        # many ragged sequences in one packed step, prompts and single tokens side by side, 8-bit pages
        _attn("attn e4m3 ragged", "e4m3", "bf16", 48, 1, 32, 8, 128, 1, 1500, 0, 4000),
        # the next 512 tokens of a long prompt over 4-bit pages
        _attn("attn int4 chunk", "int4", "bf16", 1, 2, 32, 8, 128, 512, 512, 32256, 32256, packed=False),
        # 8 guessed tokens are checked against a very long context: few rows, many bytes
        _attn("attn bf16 few rows", "plain", "bf16", 2, 1, 32, 8, 128, 8, 8, 131064, 131064, packed=False),
        # two short fp32 prompts of the small test geometry
        _attn("attn f32 short", "plain", "f32", 2, 1, 4, 4, 64, 100, 512, 0, 30),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    op = rng.choice(("plan", "rope", "write", "attn", "attn", "attn"))
    seed = rng.randrange(1, 1 << 20)
    if op == "plan":
        B = _log_int(rng, 1, 1024)
        hi = _log_int(rng, 1, 8000)
        grow = _log_int(rng, 1, max(1, min(4000, 200000 // B)))
        return _plan(None, B, rng.choice((0, hi // 2, hi)), hi, rng.choice((0, 1, grow)), grow, rng.choice((0.0, 0.2, 0.6)),
                     rng.choice((1.0, 1.0, 0.7, 0.3)), seed)
    N_kv, G = rng.choice((1, 2, 4, 8, 8, 12, 32)), rng.choice((1, 1, 2, 3, 4, 4, 7, 8))
    D = rng.choice((64, 128, 128))
    if op == "rope":
        while True:
            B, S, L = _log_int(rng, 1, 64), _log_int(rng, 1, 8192), rng.choice((1, 1, 2, 4))
            if B * S * L * N_kv * (G + 1) * D <= 8192 * 40 * 128:
                break
        R = rng.choice((D, D, D // 2, D // 4, 20))
        return _rope(None, B, S, seed, N_kv * G, N_kv, D, R, rng.choice(("halves", "pairs")),
                     rng.choice(("none", "linear", "ntk", "yarn", "bands")), rng.choice(("bf16", "bf16", "f32")), L,
                     _log_int(rng, 100, 1000000), rng.random() < 0.3)
    if op == "write":
        while True:
            T, L, fmt = _log_int(rng, 1, 30000), rng.choice((1, 2, 4, 32)), rng.choice(("plain", "e4m3"))
            if T * L * N_kv * D <= 20011 * 4 * 12 * 64:
                break
        return _write(None, fmt, "f32" if fmt == "plain" and rng.random() < 0.3 else "bf16", T, L, N_kv, D, seed)
    while True:
        fmt = rng.choice(("plain", "e4m3", "int4"))
        dtype = "f32" if fmt == "plain" and rng.random() < 0.25 else "bf16"
        B, L = _log_int(rng, 1, 64), rng.choice((1, 1, 1, 2))
        hi, held = _log_int(rng, 1, 8192), _log_int(rng, 1, 131072)
        lo, hlo = rng.choice((1, hi // 3 + 1, hi)), rng.choice((0, held // 2, held))
        c = _attn(None, fmt, dtype, B, L, N_kv * G, N_kv, D, lo, hi, hlo, held, rng.random() < 0.5, seed)
        if B * L * hi * (hi / 2 + held) * N_kv * G * D <= (8192 * 4096 * 32 * 128) // (8 if dtype == "f32" else 1) and \
                B * L * (hi + held) * N_kv * D <= 262144 * 8 * 128:
            return c


def _span(r, lo, hi, n):
    """n numbers lo..hi, spread over their logarithm where that is wide; the largest is among them."""
    wide = hi > 10 * max(lo, 1)
    x = [min(hi, max(lo, int(math.exp(r.uniform(math.log(max(lo, 1)), math.log(hi + 0.5)))))) if wide else r.randint(lo, hi)
         for _ in range(n)]
    x[r.randrange(n)] = hi
    return x


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _elem(case):
    return 2 if case["dtype"] == "bf16" else 4


def _row_bytes(case):
    return case["D"] * {"e4m3": 2, "int4": 1}[case["format"]] // 2 if case["format"] != "plain" else case["D"] * _elem(case)


def _scale_bytes(case):
    return {"plain": 0, "e4m3": 1, "int4": 2 * (case["D"] // GROUP)}[case["format"]]


def _plan_lists(case):
    r = random.Random(case["lens"])
    held = _span(r, case["lo"], case["hi"], case["B"])
    want = _span(r, case["grow_lo"], case["grow_hi"], case["B"])
    want = [-h - 5 if r.random() < case["end"] else w for h, w in zip(held, want)]
    for i in range(0, case["B"], 7):                                  # some only take back their last tokens
        if case["end"] and want[i] >= 0:
            want[i] = -(held[i] // 3)
    return held, want


def _attn_lists(case):
    r = random.Random(case["lens"])
    return _span(r, case["rows_lo"], case["rows_hi"], case["B"]), _span(r, case["held_lo"], case["held_hi"], case["B"])


def _rope_lists(case):
    """Rows of each sequence and the position of its first."""
    r = random.Random(case["lens"])
    rows = [r.randint((case["S"] + 1) // 2, case["S"]) for _ in range(case["B"])]
    rows[r.randrange(case["B"])] = case["S"]
    return rows, [r.randint(0, max(0, case["far"] - n)) for n in rows]


def work(case):
    op = case["op"]
    if op == "plan":
        held, want = _plan_lists(case)
        tokens = sum(max(w, 0) for w in want)
        pages = sum(abs(-(-max(h + w, 0) // PAGE) - -(-h // PAGE)) for h, w in zip(held, want))
        return {"bytes": 4 * (2 * tokens + 2 * pages + 7 * case["B"]), "flops": 4 * tokens}
    if op == "rope":
        n = sum(_rope_lists(case)[0]) * case["L"] * (case["N_q"] + case["N_kv"])
        return {"bytes": 2 * n * case["D"] * _elem(case), "flops": 3 * n * case["R"]}
    if op == "write":
        n = case["T"] * case["L"] * case["N_kv"]
        return {"bytes": 2 * n * (case["D"] * _elem(case) + _row_bytes(case) + _scale_bytes(case)) + 4 * case["T"], "flops": 2 * n * case["D"]}
    rows, held = _attn_lists(case)
    D, L, N_q = case["D"], case["L"], case["N_q"]
    pairs = sum(n * h + n * (n + 1) // 2 for n, h in zip(rows, held))
    kv = sum(n + h for n, h in zip(rows, held)) * L * case["N_kv"] * 2 * (_row_bytes(case) + _scale_bytes(case))
    return {"bytes": kv + sum(rows) * L * N_q * (2 * D * _elem(case) + 4), "flops": 4 * D * L * N_q * pairs}


# ---------------------------------------------------------------------------
# rows in their stored form, in plain operations
# ---------------------------------------------------------------------------
def _pow2(k):
    """2^k as float32, for -126 <= k <= 127."""
    return ((k + 127) << 23).to(torch.int32).view(torch.float32)


def _encode(x, fmt):
    """Rows [..., D] to their stored bytes: (codes [..., row bytes], scales [..., scale bytes])."""
    if fmt == "plain":
        return x.contiguous().view(torch.uint8), None
    x = x.float()
    if fmt == "e4m3":
        m, e = torch.frexp(x.abs().amax(-1))
        k = (e - 9 + (m > 0.875).to(torch.int32)).clamp_(min=-126)    # 448 = 0.875 * 2^9
        k = torch.where(m > 0, k, torch.full_like(k, -126))
        codes = (x / _pow2(k).unsqueeze(-1)).to(torch.float8_e4m3fn)
        return codes.view(torch.uint8), (k + 127).to(torch.uint8).unsqueeze(-1)
    g = x.unflatten(-1, (-1, GROUP))
    s = (g.abs().amax(-1).double() / 7).to(torch.bfloat16)
    d = s.double().unsqueeze(-1)
    n = torch.where(d > 0, g.double() / torch.where(d > 0, d, torch.ones_like(d)), torch.zeros_like(d))
    n = (n.round_().clamp_(-7, 7) + 8).to(torch.uint8).flatten(-2)
    return n[..., 0::2] | (n[..., 1::2] << 4), s.contiguous().view(torch.uint8)


def _decode(codes, scales, case):
    """The values that stored rows stand for, in 32 bits (exactly)."""
    if case["format"] == "plain":
        return codes.contiguous().view(_dtype(case)).float()
    if case["format"] == "e4m3":
        return codes.view(torch.float8_e4m3fn).float() * _pow2(scales.to(torch.int32) - 127)
    n = torch.stack((codes & 15, codes >> 4), -1).flatten(-2).float() - 8
    s = scales.contiguous().view(torch.bfloat16).float()
    return (n.unflatten(-1, (-1, GROUP)) * s.unsqueeze(-1)).flatten(-2)


def _parts(pool, case):
    """The pool's four parts as views: key rows, value rows [layer, page, head, 64, row], their scales (None if none)."""
    a, b = PAGE * _row_bytes(case), PAGE * _scale_bytes(case)
    cut = lambda o, n: pool[..., o:o + n].unflatten(-1, (PAGE, n // PAGE)) if n else None  # noqa: E731
    return cut(0, a), cut(a, a), cut(2 * a, b), cut(2 * a + b, b)


# ---------------------------------------------------------------------------
# frequencies
# ---------------------------------------------------------------------------
THETA, FACTOR, TRAINED = 500000.0, 8.0, 8192     # base, context extension, tokens of the unscaled context


def _frequencies(case):
    """Radians per token of the R/2 pairs (python floats), and the factor on the rotated channels."""
    R, kind = case["R"], case["scaling"]
    theta = THETA * FACTOR ** (R / (R - 2)) if kind == "ntk" else THETA
    f = [theta ** (-2.0 * j / R) for j in range(R // 2)]
    if kind == "linear":
        return [x / FACTOR for x in f], 1.0
    if kind == "yarn":        # pairs that turn often keep their frequency, slow ones are stretched, a ramp in between
        where = lambda turns: R * math.log(TRAINED / (turns * 2 * math.pi)) / (2 * math.log(THETA))  # noqa: E731
        low, high = max(math.floor(where(32.0)), 0), min(math.ceil(where(1.0)), R - 1)
        ramp = [min(1.0, max(0.0, (j - low) / max(high - low, 0.001))) for j in range(R // 2)]
        return [x / FACTOR * r + x * (1 - r) for x, r in zip(f, ramp)], 0.1 * math.log(FACTOR) + 1.0
    if kind == "bands":       # by the turns a pair makes over the unscaled context: below 1 stretched, above 4 kept
        turns = [TRAINED * x / (2 * math.pi) for x in f]
        keep = [min(1.0, max(0.0, (t - 1.0) / (4.0 - 1.0))) for t in turns]
        return [x / FACTOR * (1 - k) + x * k for x, k in zip(f, keep)], 1.0
    return f, 1.0


# ---------------------------------------------------------------------------
# inputs
# ---------------------------------------------------------------------------
def _normal(shape, g, dtype, factor=None):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if factor is not None:
        x *= factor
    return x.to(dtype)


def _outliers(N, D, g):
    """A few key channels are much larger than the rest, as they are in trained models."""
    factor = torch.ones(N, D, device="cuda")
    factor[:, torch.randperm(D, generator=g, device="cuda")[:4]] = 8.0
    return factor


def _ints(x):
    return torch.tensor(x, dtype=torch.int32, device="cuda")


def _cache(case, pages, pool, max_batch):
    from paper_2407_21018_b200 import binding as tk
    fmt = {"plain": tk.PAGE_PLAIN, "e4m3": tk.PAGE_E4M3, "int4": tk.PAGE_INT4}[case.get("format", "plain")]
    dtype = _dtype(case) if "dtype" in case else torch.bfloat16
    cfg = tk.make_paged_config(case.get("L", 1), case.get("N_q", case.get("N_kv", 1)), case.get("N_kv", 1), case.get("D", 64),
                               pages, max_batch, dtype, fmt)
    return tk.PagedKVCache(cfg, pages=pool)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    state = {"case": case}
    return {"plan": _prepare_plan, "rope": _prepare_rope, "write": _prepare_write, "attn": _prepare_attn}[case["op"]](case, state, g)


def _prepare_plan(case, state, g):
    held, want = _plan_lists(case)
    mix = torch.randperm(case["B"], generator=g, device="cuda").tolist()   # which sequence has which length
    held, want = [held[i] for i in mix], [want[i] for i in mix]
    used = sum(-(-h // PAGE) for h in held)
    need = sum(max(0, -(-(h + w) // PAGE) - -(-h // PAGE)) for h, w in zip(held, want) if w > 0)
    free = max(1, int(need * case["spare"]) + (4 if case["spare"] >= 1 else 0))
    order = torch.randperm(used + free, generator=g, device="cuda").to(torch.int32)
    width = max(-(-(h + max(w, 0)) // PAGE) for h, w in zip(held, want)) + 1
    table = torch.full((case["B"], width), -1, dtype=torch.int32, device="cuda")
    at = 0
    for b, h in enumerate(held):
        k = -(-h // PAGE)
        table[b, :k] = order[at:at + k]
        at += k
    free_pages = torch.full((used + free,), -1, dtype=torch.int32, device="cuda")
    free_pages[:free] = order[used:]
    state.update(table=table, seq_lens=_ints(held), change=_ints(want), free_pages=free_pages, free_count=_ints([free]),
                 max_tokens=max(1, sum(max(w, 0) for w in want)))
    if own:
        from paper_2407_21018_b200 import binding as tk
        state["cache"] = _cache(case, used + free, None, case["B"])
        state["plan"] = tk.PagePlan(case["B"], state["max_tokens"])       # where every step's results go
    return state


def _prepare_rope(case, state, g):
    rows, first = _rope_lists(case)
    B, S, L, dt = case["B"], case["S"], case["L"], _dtype(case)
    state["q"] = _normal((B, S, L, case["N_q"], case["D"]), g, dt)
    state["k"] = _normal((B, S, L, case["N_kv"], case["D"]), g, dt, _outliers(case["N_kv"], case["D"], g))
    state["q_out"], state["k_out"] = torch.zeros_like(state["q"]), torch.zeros_like(state["k"])
    shift = torch.randint(0, max(1, min(first) + 1), (1,), generator=g, device="cuda", dtype=torch.int32)
    state["pos"], state["rows"] = _ints(first) - shift, _ints(rows)
    if B == 1:                                                        # a packed batch: each token's own position
        state["pos"] = (state["pos"] + torch.arange(S, device="cuda", dtype=torch.int32)).unsqueeze(0)
    if own:
        from paper_2407_21018_b200 import binding as tk
        kind = {"none": tk.ROPE_PLAIN, "linear": tk.ROPE_LINEAR, "ntk": tk.ROPE_NTK, "yarn": tk.ROPE_YARN, "bands": tk.ROPE_BANDS}
        state["rope"] = tk.Rope(case["D"], dt, rot_dim=case["R"], layout=tk.ROPE_HALVES if case["layout"] == "halves" else tk.ROPE_PAIRS,
                                theta=THETA, scaling=kind[case["scaling"]], factor=FACTOR, trained=TRAINED)
    return state


def _prepare_write(case, state, g):
    T, L, N, D, dt = case["T"], case["L"], case["N_kv"], case["D"], _dtype(case)
    pages = -(-T // PAGE) + 2
    block = 2 * PAGE * (_row_bytes(case) + _scale_bytes(case))
    state["pool"] = torch.full((L, pages, N, block), 255, dtype=torch.uint8, device="cuda")   # NaN patterns
    # runs of slots in shuffled pages; a few tokens have none
    page = torch.randperm(pages, generator=g, device="cuda")[:-(-T // PAGE)]
    slots = (page[:, None] * PAGE + torch.arange(PAGE, device="cuda")).reshape(-1)[:T].to(torch.int32)
    if T > 8:
        slots[torch.randperm(T, generator=g, device="cuda")[:T // 50 + 1]] = -1
    state["slots"] = slots
    state["k"], state["v"] = _normal((T, L, N, D), g, dt, _outliers(N, D, g)), _normal((T, L, N, D), g, dt)
    if own:
        state["cache"] = _cache(case, pages, state["pool"], 1)
    return state


def _prepare_attn(case, state, g):
    rows, held = _attn_lists(case)
    B, L, N, D, dt = case["B"], case["L"], case["N_kv"], case["D"], _dtype(case)
    extent = [n + h for n, h in zip(rows, held)]
    width = max(-(-n // PAGE) for n in extent)
    used = sum(-(-n // PAGE) for n in extent)
    pages = used + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")
    block = 2 * PAGE * (_row_bytes(case) + _scale_bytes(case))
    pool = torch.full((L, pages, N, block), 255, dtype=torch.uint8, device="cuda")            # NaN patterns
    factor = _outliers(N, D, g)
    at = 0
    for b, n in enumerate(extent):
        k = -(-n // PAGE)
        table[b, :k] = order[at:at + k]
        at += k
        t = torch.arange(n, device="cuda")
        p, slot = table[b, t // PAGE].long(), t % PAGE
        for l in range(L):
            parts = [None if x is None else x[l] for x in _parts(pool, case)]
            for f, codes, scales in ((factor, parts[0], parts[2]), (None, parts[1], parts[3])):
                c, z = _encode(_normal((n, N, D), g, dt, f), case["format"])
                codes[p, :, slot] = c
                if z is not None:
                    scales[p, :, slot] = z
    state.update(table=table, pool=pool, rows=_ints(rows), pos=_ints(held), lists=(rows, held))
    first = [sum(rows[:b]) for b in range(B)]
    if case["packed"]:
        state["start"], shape = _ints(first), (sum(rows), L, case["N_q"], D)
    else:
        state["start"], shape = None, (B, max(rows), L, case["N_q"], D)
    state["q"] = _normal(shape, g, dt)
    if own:
        state["cache"] = _cache(case, pages, pool, B)
    else:
        state["out"] = torch.zeros_like(state["q"])
        state["lse"] = torch.zeros(shape[:-1], dtype=torch.float32, device="cuda")
    return state


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _plain_plan(state):
    table, held, want, free = state["table"], state["seq_lens"].long(), state["change"].long(), state["free_count"].long()
    dev, width, room = table.device, table.shape[1], state["max_tokens"]
    pages = lambda n: (n + PAGE - 1) // PAGE  # noqa: E731
    shrunk = torch.where(want < 0, (held + want).clamp(min=0), held)
    back = pages(held) - pages(shrunk)                                # pages given back
    fits = pages(held + want.clamp(min=0)) <= width
    ask = torch.where((want > 0) & fits, want, torch.zeros_like(want))
    need = pages(held + ask) - pages(held)
    have = free + back.sum()
    ok = ((need == 0) | (need.cumsum(0) <= have)) & ((ask == 0) | (ask.cumsum(0) <= room))
    rows = torch.where(ok, ask, torch.zeros_like(ask))
    need = torch.where(ok, need, torch.zeros_like(need))
    taken, given = need.sum(), back.sum()
    # the pages given back stand behind the free ones; new pages are taken from the end
    col = torch.arange(width, device=dev)
    lose = (col >= pages(shrunk)[:, None]) & (col < pages(held)[:, None])
    stack = torch.cat((state["free_pages"][:int(free)], table[lose]))
    gain = (col >= pages(held)[:, None]) & (col < (pages(held) + need)[:, None])
    n = int(taken)
    table[gain] = stack[stack.numel() - n:].flip(0)
    left = stack.numel() - n
    keep = min(int(free), left)
    state["free_pages"][keep:left] = stack[keep:left]
    start = torch.zeros(rows.numel() + 1, dtype=torch.long, device=dev)
    start[1:] = rows.cumsum(0)
    seq = torch.repeat_interleave(torch.arange(rows.numel(), device=dev), rows)
    token = held[seq] + torch.arange(seq.numel(), device=dev) - start[seq]
    token_pos = torch.full((room,), -1, dtype=torch.int32, device=dev)
    slots = torch.full((room,), -1, dtype=torch.int32, device=dev)
    token_pos[:seq.numel()] = token.to(torch.int32)
    slots[:seq.numel()] = (table[seq, token // PAGE].long() * PAGE + token % PAGE).to(torch.int32)
    i32 = lambda x: x.to(torch.int32)  # noqa: E731
    return {"pos": i32(shrunk), "rows": i32(rows), "start": i32(start), "token_pos": token_pos, "slots": slots,
            "seq_lens": i32(shrunk + rows), "free_count": i32(have - taken), "table": table, "free_pages": state["free_pages"]}


def _positions(state):
    """Position of every row [b, s], and which rows there are."""
    case = state["case"]
    s = torch.arange(case["S"], device="cuda")
    p = state["pos"].long()
    return (p if p.dim() == 2 else p[:, None] + s), s[None, :] < state["rows"][:, None]


def _plain_rope(state):
    case = state["case"]
    R = case["R"]
    f, m = _frequencies(case)
    at, there = _positions(state)
    angle = at.double()[..., None] * torch.tensor(f, dtype=torch.float64, device="cuda")
    c = (angle.cos() * m).float()[:, :, None, None]
    s = (angle.sin() * m).float()[:, :, None, None]
    if case["back"]:
        s = -s
    out = {}
    for name in ("q", "k"):
        x, to = state[name], state[name + "_out"]
        y = x.float()
        a, b = (y[..., :R // 2], y[..., R // 2:R]) if case["layout"] == "halves" else (y[..., 0:R:2], y[..., 1:R:2])
        u, v = a * c - b * s, b * c + a * s
        r = torch.cat((u, v), -1) if case["layout"] == "halves" else torch.stack((u, v), -1).flatten(-2)
        y = torch.cat((r, y[..., R:]), -1).to(x.dtype)
        to.copy_(torch.where(there[:, :, None, None, None], y, to))
        out[name] = to
    return out


def _held(state):
    """The pool's contents as values (rows as they are, e4m3 codes with their power-of-two scales)."""
    case, parts = state["case"], _parts(state["pool"], state["case"])
    if case["format"] == "plain":
        return {"pool": state["pool"].view(_dtype(case))}
    return {"k": parts[0].view(torch.float8_e4m3fn), "v": parts[1].view(torch.float8_e4m3fn),
            "k_scale": parts[2].view(torch.float8_e8m0fnu), "v_scale": parts[3].view(torch.float8_e8m0fnu)}


def _plain_write(state):
    case, slots = state["case"], state["slots"].long()
    there = torch.nonzero(slots >= 0).squeeze(1)
    page, slot = slots[there] // PAGE, slots[there] % PAGE
    parts = _parts(state["pool"], case)
    for x, codes, scales in ((state["k"], parts[0], parts[2]), (state["v"], parts[1], parts[3])):
        c, z = _encode(x[there], case["format"])                      # [row, l, n, bytes]
        codes[:, page, :, slot] = c
        if z is not None:
            scales[:, page, :, slot] = z
    return _held(state)


def _rows_of(state, b):
    """Where sequence b's rows stand in q: an index for its first axis or axes."""
    rows, _ = state["lists"]
    if state["case"]["packed"]:
        o = sum(rows[:b])
        return slice(o, o + rows[b])
    return (b, slice(0, rows[b]))


def _plain_attn(state):
    case, q = state["case"], state["q"]
    N, D = case["N_kv"], case["D"]
    parts = _parts(state["pool"], case)
    for b, (n, h) in enumerate(zip(*state["lists"])):
        page = state["table"][b, :-(-(n + h) // PAGE)].long()

        def rows(codes, scales, l):                                   # [n, token, d]
            x = _decode(codes[l][page], None if scales is None else scales[l][page], case)
            return x.permute(1, 0, 2, 3).flatten(1, 2)[:, :n + h]

        for l in range(case["L"]):
            k, v = rows(parts[0], parts[2], l), rows(parts[1], parts[3], l)
            at = _rows_of(state, b)
            ql = q[at][:, l].float().unflatten(1, (N, -1)) / math.sqrt(D)                      # [s, n, g, d]
            step = max(1, (1 << 28) // (case["N_q"] * (n + h)))
            for s in range(0, n, step):
                e = min(n, s + step)
                top = h + e                                           # nothing behind the last row's own token
                x = torch.einsum("sngd,ntd->nsgt", ql[s:e], k[:, :top])
                later = torch.arange(top, device=q.device)[None, :] > torch.arange(h + s, h + e, device=q.device)[:, None]
                x = x.masked_fill(later[None, :, None, :], -math.inf)
                m = x.amax(-1, keepdim=True)
                p = torch.exp(x - m)
                z = p.sum(-1, keepdim=True)
                o = torch.einsum("nsgt,ntd->sngd", p, v[:, :top]) / z.permute(1, 0, 2, 3)
                state["out"][at][s:e, l] = o.flatten(1, 2).to(q.dtype)
                state["lse"][at][s:e, l] = (m + z.log()).squeeze(-1).permute(1, 0, 2).flatten(1, 2)
    return {"out": state["out"], "lse": state["lse"]}


def run(state):
    case = state["case"]
    op = case["op"]
    if not own:
        return {"plan": _plain_plan, "rope": _plain_rope, "write": _plain_write, "attn": _plain_attn}[op](state)
    if op == "plan":
        r = state["cache"].plan(state["change"], state["seq_lens"], state["table"], state["free_pages"], state["free_count"],
                                out=state["plan"])
        return {"pos": r.pos, "rows": r.rows, "start": r.start, "token_pos": r.token_pos, "slots": r.slots, "seq_lens": r.seq_lens,
                "free_count": r.free_count, "table": state["table"], "free_pages": state["free_pages"]}
    if op == "rope":
        state["rope"].apply(state["q"], state["k"], state["pos"], rows=state["rows"], q_out=state["q_out"], k_out=state["k_out"],
                            transpose=case["back"])
        return {"q": state["q_out"], "k": state["k_out"]}
    if op == "write":
        state["cache"].write_slots(state["k"], state["v"], state["slots"])
        return _held(state)
    if "out" not in state:                                            # rows that no sequence has stay as they are
        state["out"] = torch.zeros_like(state["q"])
        state["lse"] = torch.zeros(state["q"].shape[:-1], dtype=torch.float32, device="cuda")
    out, lse = state["cache"].prompt_attn(state["q"], state["table"], state["pos"], rows=state["rows"], start=state["start"],
                                          out=state["out"], lse=state["lse"])
    return {"out": out, "lse": lse}


# ---------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------
def _two64(k):
    """2^k in 64 bits, exactly (pow() on the device rounds)."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _e4m3_64(x):
    """Rows x [..., D] as (codes' values, the row's scale) in 64 bits."""
    x = x.double()
    top = x.abs().amax(-1, keepdim=True)
    # smallest power of two, not below 2^-126, under which the largest magnitude is at most 448
    k = torch.ceil(torch.log2(torch.where(top > 0, top, torch.full_like(top, 2.0 ** -200)) / 448.0)).clamp(min=-126)
    k = torch.where(top > 448.0 * _two64(k), k + 1, k)                # log2 rounds: settle its last unit by comparing
    k = torch.where((top <= 448.0 * _two64(k - 1)) & (k > -126), k - 1, k)
    y = x * _two64(-k)
    step = _two64(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(-6, 8) - 3)      # spacing of e4m3 there
    return torch.round(y / step) * step, _two64(k)


def _stored64(raw, scale, case):
    """The values of stored rows in 64 bits, straight from their bits."""
    if case["format"] == "plain":
        return raw.contiguous().view(_dtype(case)).double()
    c = raw.to(torch.int64)
    if case["format"] == "e4m3":
        e, m = (c >> 3) & 15, c & 7
        mag = torch.where(e > 0, (8 + m).double() * _two64(e - 10), m.double() * 2.0 ** -9)
        return torch.where(c & 128 > 0, -mag, mag) * _two64(scale.to(torch.int64) - 127)
    n = torch.empty(c.shape[:-1] + (2 * c.shape[-1],), dtype=torch.float64, device=c.device)
    n[..., 0::2], n[..., 1::2] = (c % 16 - 8).double(), (c // 16 - 8).double()
    return n * scale.contiguous().view(torch.bfloat16).double().repeat_interleave(GROUP, -1)


def exact(case, seed):
    state = prepare(case, seed)
    return {"plan": _exact_plan, "rope": _exact_rope, "write": _exact_write, "attn": _exact_attn}[case["op"]](case, state)


def _exact_plan(case, state):
    """One sequence after the other, on lists."""
    table = state["table"].cpu().tolist()
    held, want = state["seq_lens"].tolist(), state["change"].tolist()
    free = int(state["free_count"])
    pool = state["free_pages"].cpu().tolist()
    stack, room, width = pool[:free], state["max_tokens"], len(table[0])
    count = lambda n: (n + PAGE - 1) // PAGE  # noqa: E731
    kept = list(held)
    for b, w in enumerate(want):
        if w < 0:
            kept[b] = max(0, held[b] + w)
            stack += table[b][count(kept[b]):count(held[b])]
    have, wanted_pages, wanted_rows = len(stack), 0, 0
    rows, start, token_pos, slots = [], [0], [-1] * room, [-1] * room
    for b, w in enumerate(want):
        ask = w if w > 0 and count(held[b] + w) <= width else 0
        need = count(held[b] + ask) - count(held[b])
        wanted_pages, wanted_rows = wanted_pages + need, wanted_rows + ask
        n = ask if (need == 0 or wanted_pages <= have) and wanted_rows <= room else 0
        for j in range(count(held[b]), count(held[b] + n)):
            table[b][j] = stack.pop()
        for i in range(n):
            t = held[b] + i
            token_pos[start[-1] + i], slots[start[-1] + i] = t, table[b][t // PAGE] * PAGE + t % PAGE
        rows.append(n)
        start.append(start[-1] + n)
    pool[min(free, len(stack)):len(stack)] = stack[min(free, len(stack)):]
    t = lambda x: torch.tensor(x, dtype=torch.int32)  # noqa: E731
    return {"pos": t(kept), "rows": t(rows), "start": t(start), "token_pos": t(token_pos), "slots": t(slots),
            "seq_lens": t([a + n for a, n in zip(kept, rows)]), "free_count": t([len(stack)]), "table": t(table), "free_pages": t(pool)}


def _exact_rope(case, state):
    f, m = _frequencies(case)
    at, _ = _positions(state)
    f = torch.tensor(f, dtype=torch.float64, device="cuda")
    out = {}
    for name in ("q", "k"):
        x = state[name].double()
        y = torch.zeros_like(x)
        for b, n in enumerate(state["rows"].tolist()):
            z = x[b, :n].clone()
            turn = torch.polar(torch.full((n, f.numel()), m, dtype=torch.float64, device="cuda"), at[b, :n, None].double() * f)
            turn = (turn.conj() if case["back"] else turn)[:, None, None, :]
            h = case["R"] // 2
            i, j = (torch.arange(h), torch.arange(h) + h) if case["layout"] == "halves" else (2 * torch.arange(h), 2 * torch.arange(h) + 1)
            w = torch.complex(x[b, :n][..., i.cuda()], x[b, :n][..., j.cuda()]) * turn
            z[..., i.cuda()], z[..., j.cuda()] = w.real, w.imag
            y[b, :n] = z
        out[name] = y
    return out


def _exact_write(case, state):
    slots = state["slots"].tolist()
    i = torch.tensor([n for n, s in enumerate(slots) if s >= 0], dtype=torch.long, device="cuda")
    page = torch.tensor([s // PAGE for s in slots if s >= 0], dtype=torch.long, device="cuda")
    slot = torch.tensor([s % PAGE for s in slots if s >= 0], dtype=torch.long, device="cuda")
    D = case["D"]
    if case["format"] == "plain":
        held = state["pool"].view(_dtype(case)).double()
        for part, x in enumerate(("k", "v")):
            held[..., part * PAGE * D:(part + 1) * PAGE * D].unflatten(-1, (PAGE, D))[:, page, :, slot] = state[x][i].double()
        return {"pool": held}
    held = {x: y.float().double() for x, y in _held(state).items()}
    for x in ("k", "v"):
        c, z = _e4m3_64(state[x][i])
        held[x][:, page, :, slot] = c
        held[x + "_scale"][:, page, :, slot] = z
    return held


def _exact_attn(case, state):
    L, N, D, pool = case["L"], case["N_kv"], case["D"], state["pool"]
    row, sc = PAGE * _row_bytes(case), PAGE * _scale_bytes(case)
    table = state["table"].cpu()
    q = state["q"].double()
    out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
    lse = torch.zeros(q.shape[:-1], dtype=torch.float64, device=q.device)

    def stored(b, l, part, h, n):
        """The first n tokens of sequence b in layer l and key head h as [token, D]; part 0: keys, 1: values."""
        blocks = pool[l, table[b, :-(-n // PAGE)].long().to(pool.device), h]                   # [page, block]
        raw = blocks[:, part * row:(part + 1) * row].reshape(blocks.shape[0] * PAGE, -1)[:n]
        z = blocks[:, 2 * row + part * sc:2 * row + (part + 1) * sc].reshape(blocks.shape[0] * PAGE, -1)[:n] if sc else None
        return _stored64(raw, z, case)

    for b, (n, held) in enumerate(zip(*state["lists"])):
        at = _rows_of(state, b)
        for l in range(L):
            for h in range(N):
                k, v = stored(b, l, 0, h, n + held), stored(b, l, 1, h, n + held)
                heads = slice(h * (case["N_q"] // N), (h + 1) * (case["N_q"] // N))
                for s in range(0, n, 1024):
                    e = min(n, s + 1024)
                    t = held + e
                    x = (q[at][s:e, l, heads].permute(1, 0, 2) @ k[:t].T) / D ** 0.5           # [g, s, t]
                    x += torch.full((e - s, t), -math.inf, dtype=torch.float64, device=q.device).triu(held + s + 1)
                    out[at][s:e, l, heads] = (torch.softmax(x, -1) @ v[:t]).permute(1, 0, 2)
                    lse[at][s:e, l, heads] = torch.logsumexp(x, -1).T
    return {"out": out, "lse": lse}
