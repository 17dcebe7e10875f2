"""The operators of the paged key-value cache, as a user calls them and in plain form.

A pool holds pages of 64 tokens.  The block of one (layer, page, key head) is, in this order,

    64 key rows | 64 value rows | scales of the 64 key rows | scales of the 64 value rows

with rows of D elements stored as they are ("plain"), as e4m3 bytes with one power-of-two exponent byte a row
("e4m3"), or as 4-bit codes, two channels a byte, with one bf16 scale per 32 channels ("int4").  A page table
[sequence, page of the sequence] says which page of the pool holds which tokens; the positions behind a
sequence's last token hold whatever was there before.  Three operators work on it:

    write   rows of keys and values go to their pages, quantised on the way
    read    rows come back from their pages, dequantised
    attn    softmax(scale * q K^T) V of one new token a sequence over its pages, and the log of its softmax sum

and "cycle" is a write followed by a read of the same rows, which is how 4-bit codes are looked at: as the
values they stand for.
"""
import math
import random

import torch

own = False

PAGE = 64
GROUP = 32          # channels that share a scale in "int4"
INT4_TOP = 7.0
E4M3_TOP = 448.0


# ---------------------------------------------------------------------------
# cases
# ---------------------------------------------------------------------------
def _case(name, op, fmt, dtype, B, L, N_q, N_kv, D, lo, hi, pos=0, lens=1):
    """lo..hi: lengths of the sequences, drawn with the seed `lens`; pos: position of the first row that is written
    or read (0 for a prompt)."""
    c = dict(op=op, format=fmt, dtype=dtype, B=B, L=L, N_q=N_q, N_kv=N_kv, D=D, lo=lo, hi=hi, pos=pos, lens=lens)
    if name:
        c["name"] = name
    return c


def listed():
    return [
        # one layer of the fp32 test geometry with its 512-token prompt: latency of the smallest call
        _case("attn f32 one short", "attn", "plain", "f32", 1, 1, 4, 4, 64, 512, 512),
        # one layer of an 8192-token chat on the LLaMA-3-8B shape, 4-bit pages: few bytes, few heads, one sequence
        _case("attn int4 one 8k", "attn", "int4", "bf16", 1, 1, 32, 8, 128, 8192, 8192),
        # one layer of a ragged batch on the LLaMA-2-7B shape (no shared heads)
        _case("attn bf16 ragged mha", "attn", "plain", "bf16", 16, 1, 32, 32, 128, 2048, 4096),
        # one layer of long prompts on the Mistral-7B shape, 8-bit pages
        _case("attn e4m3 long", "attn", "e4m3", "bf16", 4, 1, 32, 8, 128, 32768, 32768),
        # continuous batching: many sequences between one token and 2000, 4-bit pages
        _case("attn int4 many ragged", "attn", "int4", "bf16", 192, 1, 32, 8, 128, 1, 2000),
        # long-context stress: two layers over 131072 tokens
        _case("attn bf16 131k", "attn", "plain", "bf16", 1, 2, 32, 8, 128, 131072, 131072),
        # one decode step of a batch of 64: one row a sequence for each of 32 layers goes to 8-bit pages
        _case("write e4m3 step", "write", "e4m3", "bf16", 64, 32, 32, 8, 128, 1, 1, pos=1021),
        # the prompts of a ragged batch, one layer, 8-bit pages
        _case("write e4m3 prompts", "write", "e4m3", "bf16", 16, 1, 32, 32, 128, 2048, 4096),
        # the same unquantised on the D = 64 shape
        _case("write bf16 prompts", "write", "plain", "bf16", 7, 4, 12, 12, 64, 300, 5000),
        # a prompt comes back from 8-bit pages, four layers at a time, to be pruned
        _case("read e4m3 prompt", "read", "e4m3", "bf16", 1, 4, 32, 8, 128, 8192, 8192),
        # a few fp32 rows from the middle of short sequences
        _case("read f32 rows", "read", "plain", "f32", 5, 2, 4, 4, 64, 1, 150, pos=45),
        # prompts written to and read from 4-bit pages
        _case("cycle int4 prompts", "cycle", "int4", "bf16", 3, 2, 32, 8, 128, 1500, 8192),
    ]


def _log_int(rng, lo, hi):
    return min(hi, max(lo, int(round(math.exp(rng.uniform(math.log(lo), math.log(hi + 0.49)))))))


def draw(rng):
    while True:
        op = rng.choice(("attn", "attn", "attn", "write", "read", "cycle"))
        fmt = "int4" if op == "cycle" else rng.choice(("plain", "e4m3", "int4")) if op == "attn" else rng.choice(("plain", "e4m3"))
        dtype = "f32" if fmt == "plain" and rng.random() < 0.25 else "bf16"
        D = rng.choice((64, 128, 128))
        N_kv = rng.choice((1, 2, 4, 8, 8, 12, 32))
        G = rng.choice((1, 1, 2, 3, 4, 4, 7, 8))
        B = _log_int(rng, 1, 192)
        L = rng.choice((1, 1, 1, 2, 4))
        hi = _log_int(rng, 1, 131072)
        lo = hi if rng.random() < 0.3 else _log_int(rng, 1, hi)
        pos = 0 if op == "attn" or rng.random() < 0.5 else _log_int(rng, 1, 4096)
        c = _case(None, op, fmt, dtype, B, L, N_kv * G, N_kv, D, lo, hi, pos, rng.randrange(1, 1 << 20))
        # the padded extent bounds what the plain form holds
        rows = B * (hi + pos) * L * N_kv * D * (2 if dtype == "f32" else 1)
        most = 131072 * 2 * 8 * 128 if op == "attn" else 4096 * 16 * 32 * 128
        if rows <= most:
            return c


def _lens(case):
    r = random.Random(case["lens"])
    n = [r.randint(case["lo"], case["hi"]) for _ in range(case["B"])]
    n[r.randrange(case["B"])] = case["hi"]
    return n


def _dtype(case):
    return torch.bfloat16 if case["dtype"] == "bf16" else torch.float32


def _row_bytes(case):
    return case["D"] * {"e4m3": 2, "int4": 1}[case["format"]] // 2 if case["format"] != "plain" else case["D"] * (2 if case["dtype"] == "bf16" else 4)


def _scale_bytes(case):
    return {"plain": 0, "e4m3": 1, "int4": 2 * (case["D"] // GROUP)}[case["format"]]


def work(case):
    n, D, L, N = sum(_lens(case)), case["D"], case["L"], case["N_kv"]
    e = 2 if case["dtype"] == "bf16" else 4
    held = 2 * (_row_bytes(case) + _scale_bytes(case)) * n * L * N
    rows = 2 * D * e * n * L * N
    pages = sum(-(-(x + case["pos"]) // PAGE) - case["pos"] // PAGE for x in _lens(case))
    tables = 4 * (pages + 2 * case["B"])
    if case["op"] == "attn":
        per = case["B"] * L * case["N_q"]
        return {"bytes": held + 2 * per * D * e + 4 * per + tables, "flops": 4 * D * n * L * case["N_q"]}
    if case["op"] == "cycle":                         # the pool is written and read, the rows come in and go out
        return {"bytes": 2 * (held + rows) + tables, "flops": 4 * D * n * L * N}
    return {"bytes": held + rows + tables, "flops": 2 * D * n * L * N}


# ---------------------------------------------------------------------------
# the stored form, in plain operations
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
    s = (g.abs().amax(-1).double() / INT4_TOP).to(torch.bfloat16)
    d = s.double().unsqueeze(-1)
    n = torch.where(d > 0, g.double() / torch.where(d > 0, d, torch.ones_like(d)), torch.zeros_like(d))
    n = (n.round_().clamp_(-INT4_TOP, INT4_TOP) + 8).to(torch.uint8).flatten(-2)
    return n[..., 0::2] | (n[..., 1::2] << 4), s.contiguous().view(torch.uint8)


def _decode(codes, scales, case):
    """The values that stored rows stand for, in 32 bits."""
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
# inputs
# ---------------------------------------------------------------------------
def _fill(state, k, v):
    """Writes rows [b, s, l, n, d] of each sequence (s < rows[b], at position pos + s) into the pool, with plain indexing."""
    case, pool = state["case"], state["pool"]
    b, s = state["where"]
    at = s + case["pos"]
    page, slot = state["table"][b, at // PAGE].long(), at % PAGE
    parts = _parts(pool, case)
    for x, codes, scales in ((k, parts[0], parts[2]), (v, parts[1], parts[3])):
        c, z = _encode(x[b, s], case["format"])                       # [row, l, n, bytes]
        codes[:, page, :, slot] = c
        if z is not None:
            scales[:, page, :, slot] = z


def _normal(shape, g, dtype, factor=None):
    x = torch.randn(shape, generator=g, device="cuda", dtype=torch.float32)
    if factor is not None:
        x *= factor
    return x.to(dtype)


def prepare(case, seed):
    g = torch.Generator(device="cuda")
    g.manual_seed(seed)
    B, L, N, D, dt = case["B"], case["L"], case["N_kv"], case["D"], _dtype(case)
    lens = _lens(case)
    extent = [n + case["pos"] for n in lens]
    width = max(-(-n // PAGE) for n in extent)
    used = sum(-(-n // PAGE) for n in extent)
    pages = used + 3
    order = torch.randperm(pages, generator=g, device="cuda").to(torch.int32)
    table = torch.full((B, width), -1, dtype=torch.int32, device="cuda")   # entries behind a sequence's end: no page
    at = 0
    for b, n in enumerate(extent):
        k = -(-n // PAGE)
        table[b, :k] = order[at:at + k]
        at += k
    block = 2 * PAGE * (_row_bytes(case) + _scale_bytes(case))
    rows = torch.tensor(lens, dtype=torch.int32, device="cuda")
    # what was never written holds NaN patterns
    pool = torch.full((L, pages, N, block), 255, dtype=torch.uint8, device="cuda")
    state = {"case": case, "table": table, "rows": rows, "pos": torch.full_like(rows, case["pos"]), "pool": pool}
    # a few key channels are much larger than the rest, as they are in trained models
    factor = torch.ones(N, D, device="cuda")
    factor[:, torch.randperm(D, generator=g, device="cuda")[:4]] = 8.0
    longest = max(lens)
    valid = torch.arange(longest, device="cuda")[None, :] < rows[:, None]
    state["where"] = where = torch.nonzero(valid, as_tuple=True)
    if case["op"] == "attn":
        for l in range(L):
            p, slot = table[where[0], where[1] // PAGE].long(), where[1] % PAGE
            parts = [None if x is None else x[l] for x in _parts(pool, case)]
            for f, codes, scales in ((factor, parts[0], parts[2]), (None, parts[1], parts[3])):
                c, z = _encode(_normal((where[0].numel(), N, D), g, dt, f), case["format"])
                codes[p, :, slot] = c
                if z is not None:
                    scales[p, :, slot] = z
        state["q"] = _normal((B, L, case["N_q"], D), g, dt)
    else:
        k, v = _normal((B, longest, L, N, D), g, dt, factor), _normal((B, longest, L, N, D), g, dt)
        if case["op"] == "read":
            _fill(state, k, v)
        else:
            state["k"], state["v"] = k, v
        if case["op"] != "write":
            state["k_out"], state["v_out"] = torch.zeros_like(k), torch.zeros_like(v)
    if own:
        from paper_2407_21018_b200 import binding as tk
        fmt = {"plain": tk.PAGE_PLAIN, "e4m3": tk.PAGE_E4M3, "int4": tk.PAGE_INT4}[case["format"]]
        cfg = tk.make_paged_config(L, case["N_q"], N, D, pages, B, dt, fmt)
        state["cache"] = tk.PagedKVCache(cfg, pages=pool)
    return state


# ---------------------------------------------------------------------------
# one pass
# ---------------------------------------------------------------------------
def _held(state):
    """The pool's contents as values (rows as they are, e4m3 codes with their power-of-two scales)."""
    case, parts = state["case"], _parts(state["pool"], state["case"])
    if case["format"] == "plain":
        return {"pool": state["pool"].view(_dtype(case))}
    return {"k": parts[0].view(torch.float8_e4m3fn), "v": parts[1].view(torch.float8_e4m3fn),
            "k_scale": parts[2].view(torch.float8_e8m0fnu), "v_scale": parts[3].view(torch.float8_e8m0fnu)}


def _plain_read(state):
    case = state["case"]
    b, s = state["where"]
    at = s + case["pos"]
    page, slot = state["table"][b, at // PAGE].long(), at % PAGE
    parts = _parts(state["pool"], case)
    out = {}
    for name, codes, scales in (("k", parts[0], parts[2]), ("v", parts[1], parts[3])):
        x = _decode(codes[:, page, :, slot], None if scales is None else scales[:, page, :, slot], case)
        state[name + "_out"][b, s] = x.to(_dtype(case))
        out[name] = state[name + "_out"]
    return out


def _plain_attn(state):
    case, q = state["case"], state["q"]
    B, L, N, D = case["B"], case["L"], case["N_kv"], case["D"]
    parts = _parts(state["pool"], case)
    page = state["table"].long().clamp(min=0)                         # [b, page of the sequence]
    T = page.shape[1] * PAGE
    valid = torch.arange(T, device=q.device)[None, :] < state["rows"][:, None]

    def rows(codes, scales, l):                                       # [b, n, token, d], zero where there is none
        x = _decode(codes[l][page], None if scales is None else scales[l][page], case)
        x = x.permute(0, 2, 1, 3, 4).flatten(2, 3)
        return torch.where(valid[:, None, :, None], x, torch.zeros((), device=x.device))

    out, lse = [], []
    for l in range(L):
        ql = q[:, l].float().unflatten(1, (N, -1)) / math.sqrt(D)     # [b, n, g, d]
        x = ql @ rows(parts[0], parts[2], l).transpose(2, 3)
        x = x.masked_fill(~valid[:, None, None, :], -math.inf)
        m = x.amax(-1, keepdim=True)
        p = torch.exp(x - m)
        z = p.sum(-1, keepdim=True)
        out.append(((p @ rows(parts[1], parts[3], l)) / z).flatten(1, 2))
        lse.append((m + z.log()).squeeze(-1).flatten(1, 2))
    return {"out": torch.stack(out, 1).to(q.dtype), "lse": torch.stack(lse, 1)}


def run(state):
    case = state["case"]
    op = case["op"]
    if own:
        cache, table = state["cache"], state["table"]
        if op == "attn":
            out, lse = cache.decode_attn(state["q"], table, state["rows"], return_lse=True)
            return {"out": out, "lse": lse}
        if op != "read":
            cache.write(state["k"], state["v"], table, pos=state["pos"], rows=state["rows"])
        if op == "write":
            return _held(state)
        cache.read(state["k_out"], state["v_out"], table, pos=state["pos"], rows=state["rows"])
        return {"k": state["k_out"], "v": state["v_out"]}
    if op == "attn":
        return _plain_attn(state)
    if op != "read":
        _fill(state, state["k"], state["v"])
    return _held(state) if op == "write" else _plain_read(state)


# ---------------------------------------------------------------------------
# the same from the definitions, in 64 bits
# ---------------------------------------------------------------------------
def _two64(k):
    """2^k in 64 bits, exactly (pow() on the device rounds)."""
    return ((k.to(torch.int64) + 1023) << 52).view(torch.float64)


def _grid64(x, fmt):
    """What rows x [..., D] read back as, in 64 bits: (codes as values, scale of each value's row or group)."""
    x = x.double()
    if fmt == "e4m3":
        top = x.abs().amax(-1, keepdim=True)
        # smallest power of two, not below 2^-126, under which the largest magnitude is at most 448
        k = torch.ceil(torch.log2(torch.where(top > 0, top, torch.full_like(top, 2.0 ** -200)) / E4M3_TOP)).clamp(min=-126)
        k = torch.where(top > E4M3_TOP * _two64(k), k + 1, k)         # log2 rounds: settle its last unit by comparing
        k = torch.where((top <= E4M3_TOP * _two64(k - 1)) & (k > -126), k - 1, k)
        y = x * _two64(-k)
        step = _two64(torch.floor(torch.log2(y.abs().clamp(min=2.0 ** -6))).clamp(-6, 8) - 3)    # spacing of e4m3 there
        return torch.round(y / step) * step, _two64(k)
    g = x.reshape(x.shape[:-1] + (-1, GROUP))
    s = g.abs().amax(-1, keepdim=True) / INT4_TOP
    unit = _two64(torch.floor(torch.log2(s.clamp(min=2.0 ** -126))) - 7)     # spacing of bf16 there
    s = torch.round(s / unit) * unit
    n = torch.where(s > 0, torch.round(g / s.clamp(min=2.0 ** -140)), torch.zeros_like(g)).clamp(-INT4_TOP, INT4_TOP)
    return n.reshape(x.shape), s.expand(g.shape).reshape(x.shape)


def _stored64(raw, scale, case):
    """The values of stored rows in 64 bits, straight from their bits."""
    if case["format"] == "plain":
        return raw.contiguous().view(_dtype(case)).double()
    if case["format"] == "e4m3":
        c = raw.to(torch.int64)
        e, m = (c >> 3) & 15, c & 7
        mag = torch.where(e > 0, (8 + m).double() * _two64(e - 10), m.double() * 2.0 ** -9)
        return torch.where(c & 128 > 0, -mag, mag) * _two64(scale.to(torch.int64) - 127)
    c = raw.to(torch.int64)
    n = torch.empty(c.shape[:-1] + (2 * c.shape[-1],), dtype=torch.float64, device=c.device)
    n[..., 0::2], n[..., 1::2] = (c % 16 - 8).double(), (c // 16 - 8).double()
    return n * scale.contiguous().view(torch.bfloat16).double().repeat_interleave(GROUP, -1)


def exact(case, seed):
    state = prepare(case, seed)
    lens, D, pos = _lens(case), case["D"], case["pos"]
    table = state["table"].cpu()
    row, sc = PAGE * _row_bytes(case), PAGE * _scale_bytes(case)
    pool = state["pool"]
    L, N = case["L"], case["N_kv"]

    def stored(b, l, part, n0, n1):
        """Tokens n0..n1 of sequence b in layer l as [head, token, D]; part 0: keys, 1: values."""
        blocks = pool[l, table[b, n0 // PAGE:-(-n1 // PAGE)].long().to(pool.device)]          # [page, head, block]
        raw = blocks[:, :, part * row:(part + 1) * row].reshape(blocks.shape[0], N, PAGE, -1)
        z = blocks[:, :, 2 * row + part * sc:2 * row + (part + 1) * sc].reshape(blocks.shape[0], N, PAGE, -1) if sc else None
        join = lambda t: t.permute(1, 0, 2, 3).reshape(N, -1, t.shape[-1])[:, n0 % PAGE:n0 % PAGE + n1 - n0]  # noqa: E731
        return _stored64(join(raw), None if z is None else join(z), case)

    if case["op"] == "attn":
        q = state["q"].double()
        out = torch.zeros(q.shape, dtype=torch.float64, device=q.device)
        lse = torch.zeros(q.shape[:-1], dtype=torch.float64, device=q.device)
        for b, n in enumerate(lens):
            for l in range(L):
                k, v = stored(b, l, 0, 0, n), stored(b, l, 1, 0, n)
                x = torch.einsum("ngd,ntd->ngt", q[b, l].reshape(N, -1, D), k) / D ** 0.5
                out[b, l] = torch.einsum("ngt,ntd->ngd", torch.softmax(x, -1), v).reshape(-1, D)
                lse[b, l] = torch.logsumexp(x, -1).reshape(-1)
        return {"out": out, "lse": lse}
    if case["op"] in ("read", "cycle"):
        got = {x: torch.zeros(state[x + "_out"].shape, dtype=torch.float64, device=pool.device) for x in ("k", "v")}
        for b, n in enumerate(lens):
            for part, x in enumerate(("k", "v")):
                if case["op"] == "cycle":
                    c, z = _grid64(state[x][b, :n], case["format"])
                    got[x][b, :n] = c * z
                    continue
                for l in range(L):
                    got[x][b, :n, l] = stored(b, l, part, pos, pos + n).permute(1, 0, 2)
        return got
    # write: what was in the pool, with the new rows in their places
    if case["format"] == "plain":
        held = state["pool"].view(_dtype(case)).double()
        rows_of = [held[..., i * PAGE * D:(i + 1) * PAGE * D].unflatten(-1, (PAGE, D)) for i in (0, 1)]
    else:
        parts = _held(state)
        held = {x: parts[x].float().double() for x in parts}
    for b, n in enumerate(lens):
        at = torch.arange(pos, pos + n)
        page, slot = table[b, at // PAGE].long().to(pool.device), (at % PAGE).to(pool.device)
        for i, x in enumerate(("k", "v")):
            new = state[x][b, :n]                                     # [token, layer, head, D]
            if case["format"] == "plain":
                rows_of[i][:, page, :, slot] = new.double()
            else:
                c, z = _grid64(new, case["format"])
                held[x][:, page, :, slot] = c
                held[x + "_scale"][:, page, :, slot] = z
    return {"pool": held} if case["format"] == "plain" else held
