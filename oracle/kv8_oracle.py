"""CPU oracle of the 8-bit KV cache, the head norms and the capped scores, fp64, from the format's definition in
include/arb.h.  Test infrastructure; the product path never imports it."""
from __future__ import annotations

import numpy as np

from . import arb_oracle as O

MIN_E = -100
TOO_LARGE = 2.0 ** 120


def e4m3_values() -> np.ndarray:
    """The value of every e4m3 byte: sign, 4 exponent bits (bias 7), 3 mantissa bits; 0x7f and 0xff are NaN."""
    b = np.arange(256)
    e, m = (b >> 3) & 15, b & 7
    v = np.where(e == 0, m * 2.0 ** -9, (8 + m) * 2.0 ** (np.maximum(e, 1) - 10.0))
    v[(b & 127) == 127] = np.nan
    return np.where(b & 128, -v, v)


def e4m3_round(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value of |x| <= 448, ties to the even mantissa: multiples of 2^(exponent - 3), of 2^-9 below 2^-6."""
    x = np.asarray(x, np.float64)
    _, k = np.frexp(np.abs(x))                     # |x| in [2^(k-1), 2^k)
    step = np.exp2(np.maximum(k - 1, -6) - 3.0)
    return np.rint(x / step) * step


def scale_exponent(row_max: np.ndarray) -> np.ndarray:
    """Least e >= -100 with row_max <= 448 * 2^e."""
    m, k = np.frexp(np.asarray(row_max, np.float64))           # row_max = m 2^k, m in [0.5, 1); 448 = 0.875 * 2^9
    e = np.where(m <= 0.875, k - 9, k - 8)
    return np.maximum(np.where(m == 0, MIN_E, e), MIN_E)


def quantize(k: np.ndarray, v: np.ndarray):
    """Rows [..., hd] of keys and values of the same positions -> (k elements, v elements, k exponents, v exponents)."""
    k, v = np.asarray(k, np.float64), np.asarray(v, np.float64)
    fine = lambda x: np.isfinite(x).all(-1) & (np.abs(np.nan_to_num(x)).max(-1) < TOO_LARGE)
    ok = fine(k) & fine(v)
    out = []
    for x, bad in ((k, np.nan), (v, 0.0)):
        x = np.where(ok[..., None], x, 0.0)
        e = scale_exponent(np.abs(x).max(-1))
        el = e4m3_round(x * np.exp2(-e.astype(np.float64))[..., None])
        out.append((np.where(ok[..., None], el, bad), np.where(ok, e, 0)))
    return out[0][0], out[1][0], out[0][1], out[1][1]


def head_norm(u: np.ndarray, g, eps: float) -> np.ndarray:
    return u if g is None else O.rmsnorm(u, g, eps)


def capped(x: np.ndarray, cap: float) -> np.ndarray:
    return x if cap == 0 else cap * np.tanh(x / cap)


def append_attention(q, k, v, limits, cap: float):
    """One sequence and kv head: q [R, hd] rows that see keys 0..limits[r]; k, v fp64 [n, hd].  -> (out, sum of p |v|)."""
    logits = capped(q @ k.T / np.sqrt(float(q.shape[1])), cap)
    p = O.softmax(np.where(np.arange(k.shape[0])[None] <= np.asarray(limits)[:, None], logits, -np.inf))
    return p @ v, p @ np.abs(v)
