"""Oracle of packed batches: plans on Python lists, rotary positions and attention of many new tokens in 64 bits or more.

Independent of the CUDA path and of torch, written from the definitions in include/think.h.
"""
from __future__ import annotations

import math

import numpy as np

from . import paged_oracle as po

PAGE = 64


def pages_of(n: int) -> int:
    return -(-n // PAGE)


def plan(table, seq_lens, change, free_pages, free_count, max_tokens, num_pages):
    """One step, one sequence after the other.  Lists (table: list of rows); returns a dict of new lists and `error`, whether
    the call has to set bit 16 of the error word."""
    table, pool = [list(r) for r in table], list(free_pages)
    width = len(table[0])
    error = not 0 <= free_count <= num_pages
    free = min(max(free_count, 0), num_pages)
    stack = pool[:free]
    held = [min(max(n, 0), PAGE * width) for n in seq_lens]
    error |= any(n > PAGE * width for n in seq_lens)
    kept = [max(0, h + c) if c < 0 else h for h, c in zip(held, change)]
    for b, row in enumerate(table):
        stack += row[pages_of(kept[b]):pages_of(held[b])]
    have, want_pages, want_rows = len(stack), 0, 0
    out = dict(pos=kept, rows=[], start=[0], token_pos=[-1] * max_tokens, slots=[-1] * max_tokens)
    for b, c in enumerate(change):
        ask = c if c > 0 and held[b] + c <= PAGE * width else 0
        error |= c > 0 and ask == 0
        need = pages_of(held[b] + ask) - pages_of(held[b])
        want_pages, want_rows = want_pages + need, want_rows + ask
        n = ask if (need == 0 or want_pages <= have) and want_rows <= max_tokens else 0
        for j in range(pages_of(held[b]), pages_of(held[b] + n)):
            table[b][j] = stack.pop()
            error |= not 0 <= table[b][j] < num_pages
        at = out["start"][-1]
        for i in range(n):
            t = held[b] + i
            page = table[b][t // PAGE]
            out["token_pos"][at + i] = t
            if 0 <= page < num_pages:
                out["slots"][at + i] = page * PAGE + t % PAGE
            else:
                error = True
        out["rows"].append(n)
        out["start"].append(at + n)
    keep = min(free, len(stack))
    for x in range(keep, len(stack)):
        error |= not 0 <= stack[x] < num_pages
    pool[keep:len(stack)] = stack[keep:]
    out.update(table=table, free_pages=pool, free_count=len(stack), seq_lens=[k + n for k, n in zip(kept, out["rows"])],
               error=error)
    return out


def rope_frequencies(R, theta, scaling="plain", factor=1.0, trained=0.0, slow=0.0, fast=0.0, attention_factor=0.0):
    """(radians per token of the R / 2 pairs, factor m), in extended precision where the platform has it."""
    L = np.longdouble
    pi2 = 8 * np.arctan(L(1))
    theta = L(theta)
    if scaling == "ntk":
        theta = theta * L(factor) ** (L(R) / (R - 2))
    m = L(attention_factor) or (L("0.1") * np.log(L(factor)) + 1 if scaling == "yarn" else L(1))
    out = []
    for j in range(R // 2):
        f = theta ** (L(-2 * j) / R)
        if scaling == "linear":
            f = f / L(factor)
        elif scaling == "yarn":
            at = lambda turns: R * np.log(L(trained) / (L(turns) * pi2)) / (2 * np.log(theta))  # noqa: E731
            low, high = max(math.floor(at(fast or 32)), 0), min(math.ceil(at(slow or 1)), R - 1)
            r = min(L(1), max(L(0), (L(j) - low) / max(L(high - low), L("0.001"))))
            f = f * (1 - r) + f / L(factor) * r
        elif scaling == "bands":
            lo, hi = L(slow or 1), L(fast or 4)
            r = min(L(1), max(L(0), (hi - f * L(trained) / pi2) / (hi - lo)))
            f = f * (1 - r) + f / L(factor) * r
        out.append(f)
    return np.array(out), m


def rope(x, pos, freq, m, R, layout, transpose=False):
    """x [..., D] of one token at position pos, in extended precision."""
    x = np.asarray(x, dtype=np.longdouble)
    y = x.copy()
    t = np.longdouble(pos) * freq
    c, s = m * np.cos(t), m * np.sin(t) * (-1 if transpose else 1)
    i, j = (slice(0, R // 2), slice(R // 2, R)) if layout == "halves" else (slice(0, R, 2), slice(1, R, 2))
    y[..., i], y[..., j] = x[..., i] * c - x[..., j] * s, x[..., j] * c + x[..., i] * s
    return y


def prompt_attention(q, k, v, pos, scale):
    """q [s, G, D] of one key head, row i at position pos + i; k, v [n, D].  Row i sees tokens 0 .. pos + i.  Returns
    (out [s, G, D], lse [s, G], list of the sizes of paged_oracle.attention)."""
    out, lse, sizes = np.zeros(q.shape), np.zeros(q.shape[:2]), []
    for i in range(q.shape[0]):
        n = max(0, min(k.shape[0], pos + i + 1))
        out[i], lse[i], z = po.attention(q[i], k[:n], v[:n], scale)
        sizes.append(z)
    return out, lse, sizes
