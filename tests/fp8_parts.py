"""Inputs over which attention's sums have next to no terms, so that what is left of
its error is the roundings that a call makes, and their bound.

The kernels hold queries (times log2(e) / sqrt(hd)) and probabilities as sums of
parts of 16 bits.  A rounding to bf16 is off by at most 2^-8 of the value, to
fp16 by 2^-11.  A float32 has 24 significant bits: three bf16 parts hold it
whole (two leave up to 2^-17 of it, one 2^-8); two fp16 parts leave up to 2^-23
(one 2^-11).  Sums of random terms hide that: their float32 bound is
3 hd 2^-23.  Here two keys alone have weight, x = exp(s2 - s1) : 1, and each has
one dimension, so a score is one product and o = x / (1 + x) with values 1 and 0:

  "scores"         s1 and s2 of 40 to 60 from different dimensions of the query, 2 apart at most
  "probabilities"  s1 = 0, s2 in (-2, 0)

All other keys are 180 or more below and weigh nothing (e^-180 < 2^-149).  Roundings,
relative to |s| for a score: the query's product 2^-24; its parts 2^-23; the
sum of the parts' products 2 * 2^-23 (nearest or truncated); the product with
the key's scale 2^-24: 3.5 * 2^-23 for each score.  In the exponent, with 2^15 p held and the
maximum taken off: 15 + |s| log2(e) rounded to 2^-24, twice a key, times ln 2.
Of each p: exp2, 2^-22; its parts, 2^-23.  Of o: sums of two, the division and the last
product, 8 * 2^-24.  So

  |dx| / x <= 3.5 2^-23 (|s1| + |s2|) + 4 ln 2 (15 + 1.45 |s|) 2^-24 + 2 (2^-22 + 2^-23)
  |do| <= o (1 - o) |dx| / x + o 2^-21

(the common factor log2(e) / sqrt(hd), 3 roundings, adds 3 2^-24 |s1 - s2| to |dx| / x).
"""
import numpy as np

A, B = 37, 45  # the two keys, in one chunk of 32: their probabilities have one maximum


def inputs(kind, hd, H, n, keys, seed):
    """q [n, H, hd]; k, v [keys, hd] (bf16 values); s1, s2 [n, H] in 64 bits."""
    rng = np.random.default_rng(seed)
    q = np.zeros((n, H, hd))
    k = np.zeros((keys, hd))
    v = np.full((keys, hd), 1.0)
    k[:, 2] = -8.0  # (q[2] / sqrt(hd) = 30 or more: 240 below 0)
    k[[A, B]] = 0
    if kind == "scores":
        q[..., 0] = rng.uniform(40, 58, (n, H))
        q[..., 1] = q[..., 0] + rng.uniform(-2, 2, (n, H))
        k[A, 0], k[B, 1] = 1.0, 1.0
    else:
        q[..., 1] = rng.uniform(0.05, 2, (n, H))
        k[B, 1] = -1.0
    q[..., 2] = 30.0
    v[A] = 0.0
    q = (q * np.sqrt(hd)).astype(np.float32)
    s = lambda key: (q.astype(np.float64) @ k[key]) / np.sqrt(hd)  # noqa: E731
    return q, k, v, s(A), s(B)


def reference(s1, s2):
    return 1.0 / (1.0 + np.exp(s1 - s2))


def bound(s1, s2):
    o, big = reference(s1, s2), np.maximum(np.abs(s1), np.abs(s2))
    dx = 3.5 * 2.0 ** -23 * (np.abs(s1) + np.abs(s2)) + 4 * np.log(2) * (15 + 1.45 * big) * 2.0 ** -24
    dx += 2 * (2.0 ** -22 + 2.0 ** -23) + 3 * 2.0 ** -24 * np.abs(s1 - s2)
    return o * (1 - o) * dx + o * 2.0 ** -21
