"""GPU tests of packed batches at the ends of their ranges: the longest sequences, the largest and smallest values and scales, the
batch sizes at which a launch changes its form.  Bounds as in test_gpu_prompt."""
import os
import subprocess
import sys

import numpy as np
import pytest
import torch

from oracle import paged_oracle as po
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
for B in (3040, 3055, 3056, 3071, 3072, 3056, 4096):
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
def test_large_values_at_logits_above_those_before(fmt, dtype, value):
    """A token in the second tile has a weight of e^4 relative to all tokens of the first, and a value next to the type's largest: its
    share is 0.3 of that value, whatever the weights are relative to on the way."""
    t, n = 90, 120

    def keys(k):
        k[:] = 0
        k[0, t] = 2.0

    def values(v):
        v[0, t, 0, 0, 5] = value

    p = Prompt(fmt, dtype, [n], [0], N_kv=1, G=4, D=64, k_edit=keys, v_edit=values)
    p.q.fill_(0.25)
    out, lse = p.call()
    p.check(out, lse, lambda b, s: s < 4 or s >= t - 2)
    share = out[t:, 0, :, 5].double() / value
    assert (share > 0.25).all() and (share < 0.45).all()
