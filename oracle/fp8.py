"""The 8-bit KV cache's rounding and attention over it (TEST INFRASTRUCTURE ONLY).

Positions lie in blocks of 64; a committed whole block of one kv head is held as
e4m3 codes times one power of two, everything past it as it was stored (bf16):

  scale = 2^e, e the smallest integer with max|x| <= 448 * 2^e over the block's
  finite entries, and at least -100 (so a zero block has 2^-100);
  code = the e4m3 value nearest x / scale, ties to even; NaN and infinities
  become NaN.

e4m3: sign, 4 exponent bits (bias 7), 3 mantissa bits, subnormals below 2^-6,
largest 448, no infinities.  All arithmetic is float64.
"""
from __future__ import annotations

import numpy as np

BLOCK = 64
E4M3_MAX = 448.0
MIN_EXP = -100


def e4m3_values() -> np.ndarray:
    """The 127 non-negative finite e4m3 values, by their codes 0 .. 126."""
    out = []
    for code in range(127):
        e, m = code >> 3, code & 7
        out.append(m / 8 * 2.0 ** -6 if e == 0 else (1 + m / 8) * 2.0 ** (e - 7))
    return np.array(out)


def round_e4m3(x: np.ndarray) -> np.ndarray:
    """Nearest e4m3 value of each entry, ties to the even code (a table search)."""
    x = np.asarray(x, np.float64)
    table = e4m3_values()
    a = np.minimum(np.abs(np.nan_to_num(x, nan=0.0, posinf=0.0, neginf=0.0)), E4M3_MAX)
    hi = np.minimum(np.searchsorted(table, a), 126)
    lo = np.maximum(hi - 1, 0)
    up, down = table[hi] - a, a - table[lo]
    pick = np.where(up < down, hi, np.where(down < up, lo, np.where(hi % 2 == 0, hi, lo)))
    out = np.copysign(table[pick], x)
    return np.where(np.isfinite(x), out, np.nan)


def block_scale(x: np.ndarray) -> float:
    """2^e of one block of one kv head (searched, no logarithm)."""
    finite = np.abs(np.asarray(x, np.float64)[np.isfinite(x)])
    amax = float(finite.max()) if finite.size else 0.0
    e = MIN_EXP
    while amax > E4M3_MAX * 2.0 ** e:
        e += 1
    return 2.0 ** e


def stored(x: np.ndarray, sealed: int) -> np.ndarray:
    """What a cache holds for rows x [n, G, hd] whose first `sealed` (whole blocks) are quantized."""
    x = np.asarray(x, np.float64)
    out = x.copy()
    for p in range(0, sealed, BLOCK):
        for g in range(x.shape[1]):
            blk = x[p:p + BLOCK, g]
            s = block_scale(blk)
            out[p:p + BLOCK, g] = round_e4m3(blk / s) * s
    return out


def attention(q: np.ndarray, k: np.ndarray, v: np.ndarray, pos0: int) -> np.ndarray:
    """q [n, H, hd] at positions pos0 .. pos0+n-1 over keys and values [m, G, hd]."""
    n, H, hd = q.shape
    G = k.shape[1]
    out = np.zeros((n, H, hd))
    for i in range(n):
        m = pos0 + i + 1
        for h in range(H):
            g = h // (H // G)
            s = k[:m, g] @ q[i, h] / np.sqrt(hd)
            e = np.exp(s - s.max())
            out[i, h] = (e[:, None] * v[:m, g]).sum(0) / e.sum()
    return out
