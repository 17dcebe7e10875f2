"""Pins of the paged-cache oracle on hand values and on torch's own e4m3 and bf16 casts."""
import numpy as np
import torch

from oracle import paged_oracle as po


def test_e4m3_table_against_torch():
    want = torch.arange(256, dtype=torch.uint8).view(torch.float8_e4m3fn).double().numpy()
    assert np.array_equal(po.E4M3, want, equal_nan=True)


def test_rounding_against_torch_casts():
    g = np.random.default_rng(1)
    y = np.concatenate([g.uniform(-448, 448, 4000), g.normal(size=4000) * 0.01, po.E4M3[np.isfinite(po.E4M3)],
                        (po._POS[1:] + po._POS[:-1]) / 2, -(po._POS[1:] + po._POS[:-1]) / 2]).astype(np.float32)
    got = po.E4M3[po.round_e4m3(y.astype(np.float64))]
    assert np.array_equal(got, torch.from_numpy(y).to(torch.float8_e4m3fn).double().numpy())
    got = po.round_bf16(y.astype(np.float64))
    assert np.array_equal(got, torch.from_numpy(y).to(torch.bfloat16).double().numpy())


def test_hand_values():
    x = np.zeros(64)
    x[0], x[1], x[2] = 448.0, -1.0, 0.3
    c, s = po.encode_row(x, "e4m3")
    assert s[0] == 127 and po.E4M3[c[0]] == 448 and po.E4M3[c[1]] == -1 and po.E4M3[c[2]] == 0.3125
    c, s = po.encode_row(x * 2, "e4m3")               # one step up: the same codes, the next power of two
    assert s[0] == 128 and po.E4M3[c[0]] == 448
    c, s = po.encode_row(np.where(np.arange(64) == 0, 449.0, x), "e4m3")
    assert s[0] == 128
    x = np.zeros(64)
    x[:4] = 7.0, -3.5, 0.5, 1.5                       # scale 1: ties go to even codes
    c, s = po.encode_row(x, "int4")
    assert list(po.decode_row(c, s, "int4")[:4]) == [7, -4, 0, 2]
    assert c[0] == (15 | 4 << 4)
    assert s.view(np.uint16)[1] == 0                  # an empty group


def test_attention_hand_value():
    q = np.array([[1.0, 0.0]])
    k = np.array([[0.0, 5.0], [np.log(3.0), 0.0]])
    v = np.array([[1.0, 0.0], [0.0, 1.0]])
    out, lse, _ = po.attention(q, k, v, 1.0)
    assert np.allclose(out, [[0.25, 0.75]]) and np.allclose(lse, np.log(4.0))
    out, lse, _ = po.attention(q, k[:0], v[:0], 1.0)
    assert (out == 0).all() and np.isneginf(lse).all()
