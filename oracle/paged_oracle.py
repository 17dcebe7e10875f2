"""fp64 oracle of the paged key-value cache: stored formats from their definitions, attention over them.

Independent of the CUDA path and of torch: numpy only, loops over sequences, heads and tokens where that keeps the
definition visible.  bf16 values are given as exactly representable float64 numbers.
"""
from __future__ import annotations

import numpy as np

PAGE = 64
GROUP = 32
FORMATS = ("plain", "e4m3", "int4")


def e4m3_values() -> np.ndarray:
    """The 256 values of the byte codes (sign, 4 exponent bits with bias 7, 3 mantissa bits; 0x7f and 0xff are NaN)."""
    out = np.zeros(256)
    for c in range(256):
        e, m = (c >> 3) & 15, c & 7
        mag = (1 + m / 8) * 2.0 ** (e - 7) if e else m / 8 * 2.0 ** -6
        if e == 15 and m == 7:
            mag = np.nan
        out[c] = -mag if c & 128 else mag
    return out


E4M3 = e4m3_values()
_POS = E4M3[:127]                                     # 0 .. 448 ascending


def round_e4m3(y: np.ndarray) -> np.ndarray:
    """Codes of |y| <= 448 rounded to nearest, ties to the even code (neighbouring codes differ in their last bit)."""
    a = np.abs(y)
    hi = np.clip(np.searchsorted(_POS, a, side="left"), 1, 126)
    lo = hi - 1
    dl, dh = a - _POS[lo], _POS[hi] - a
    code = np.where(dl < dh, lo, np.where(dh < dl, hi, np.where(lo % 2 == 0, lo, hi)))
    code = np.where(a == 0, 0, code)
    return (code + np.where(np.signbit(y), 128, 0)).astype(np.uint8)


def round_bf16(x: np.ndarray) -> np.ndarray:
    """float64 -> nearest bf16 value (ties to even), as float64; magnitudes below the largest bf16."""
    x = np.asarray(x, dtype=np.float64)
    e = np.floor(np.log2(np.maximum(np.abs(x), 2.0 ** -126)))
    e = np.where(np.abs(x) < 2.0 ** e, e - 1, e)      # log2 may round up to the next integer
    unit = 2.0 ** (np.maximum(e, -126) - 7)
    return np.round(x / unit) * unit


def bf16_bits(x: np.ndarray) -> np.ndarray:
    """Bit patterns of values that are exactly bf16."""
    return (np.asarray(x, dtype=np.float32).view(np.uint32) >> 16).astype(np.uint16)


def encode_row(x: np.ndarray, fmt: str):
    """One row of D values -> (code bytes, scale bytes) of the quantised formats."""
    D = x.shape[0]
    if fmt == "e4m3":
        if not np.isfinite(x).all():
            return np.full(D, 127, np.uint8), np.array([127], np.uint8)
        top, k = np.abs(x).max(), -126
        while top > 448.0 * 2.0 ** k:
            k += 1
        return round_e4m3(x / 2.0 ** k), np.array([k + 127], np.uint8)
    codes, scales = np.zeros(D // 2, np.uint8), np.zeros(D // GROUP, np.uint16)
    for g in range(D // GROUP):
        y = x[g * GROUP:(g + 1) * GROUP]
        n = np.zeros(GROUP, dtype=np.int64)
        if np.isfinite(y).all():
            s = float(round_bf16(np.abs(y).max() / 7.0))
            scales[g] = bf16_bits(s)
            if s > 0:
                n = np.clip(np.round(y / s), -7, 7).astype(np.int64)
        else:
            scales[g] = 0x7fc0
        c = n + 8
        codes[g * GROUP // 2:(g + 1) * GROUP // 2] = c[0::2] | (c[1::2] << 4)
    return codes, scales.view(np.uint8)


def decode_row(codes: np.ndarray, scales: np.ndarray, fmt: str) -> np.ndarray:
    """Values in 64 bits of one stored row of a quantised format."""
    if fmt == "e4m3":
        return E4M3[codes] * (np.nan if scales[0] == 255 else 2.0 ** (int(scales[0]) - 127))
    n = np.empty(2 * codes.shape[0])
    n[0::2], n[1::2] = (codes & 15).astype(np.int64) - 8, (codes >> 4).astype(np.int64) - 8
    s = (np.ascontiguousarray(scales).view(np.uint16).astype(np.uint32) << 16).view(np.float32).astype(np.float64)
    return n * np.repeat(s, GROUP)


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, scale: float):
    """One key head: q [G, D], k and v [n, D].  Returns (out [G, D], lse [G], sizes), where sizes holds the magnitudes
    that the error bounds of the tests are made of (maxima over the tokens t, weights w):
      absv [G, D]   sum of w |v|                 qk     max over t of sum |scale q_i k_i|
      top           max over t of w max|v|       q_max  max over t of |scale| max|q| sum |k_i|"""
    G, D = q.shape
    if k.shape[0] == 0:
        z = np.zeros(G)
        return np.zeros((G, D)), np.full(G, -np.inf), dict(absv=np.zeros((G, D)), top=z, qk=z, q_max=z)
    x = scale * (q @ k.T)
    m = x.max(axis=1, keepdims=True)
    p = np.exp(x - m)
    z = p.sum(axis=1, keepdims=True)
    w = p / z
    aq, ak, vm, s = np.abs(q), np.abs(k), np.abs(v).max(axis=1), abs(scale)
    sizes = dict(absv=w @ np.abs(v), top=(w * vm).max(axis=1), qk=s * (aq @ ak.T).max(axis=1),
                 q_max=s * aq.max(axis=1) * ak.sum(axis=1).max())
    return w @ v, (m + np.log(z))[:, 0], sizes
