"""Sampling rules (TEST INFRASTRUCTURE ONLY): temperature, min-p, top-k and
top-p on one row of logits, in that order, with the integer masses that fix
every border.

With m = max l, e_j = exp((l_j - m) / T) (float64) and W_j = floor(e_j 2^43):
tokens with l_j > -inf and e_j >= min_p are candidates, ordered by falling l_j,
the lower index first on ties; top_k keeps the first k; top_p keeps the shortest
prefix of those with mass >= max(1, ceil(top_p * mass of the k)).  Probabilities
are fl32(e_j 2^43 / mass of the kept); temperature 0 is the argmax alone.
"""
from __future__ import annotations

import math

import numpy as np

from .sampling import NonFiniteError, argmax_first, sample_fixed_point

TWO43 = 2 ** 43


def kept(l, T=1.0, top_k=0, top_p=1.0, min_p=0.0):
    """(indices kept, in order; their float64 e_j; their integer mass)."""
    l = np.asarray(l, np.float64)
    if np.isnan(l).any() or (l == np.inf).any() or not np.isfinite(l).any():
        raise NonFiniteError("logits")
    if not T >= 0 or math.isnan(top_p) or math.isnan(min_p):
        raise NonFiniteError("rules")
    if T == 0:
        return np.array([argmax_first(l)]), np.ones(1), TWO43
    m = l.max()
    with np.errstate(divide="ignore", over="ignore"):
        e = np.where(l > -np.inf, np.exp(np.where(l > -np.inf, l - m, 0.0) / T), 0.0)
    order = [j for j in sorted(range(len(l)), key=lambda j: (-l[j], j)) if l[j] > -np.inf and e[j] >= min(min_p, 1.0)]
    if top_k > 0:
        order = order[:top_k]
    W = [int(math.floor(float(e[j]) * TWO43)) for j in order]
    n = len(order)
    if top_p < 1:
        need = max(1, math.ceil(max(0.0, float(top_p)) * float(sum(W))))
        run, n = 0, 0
        while run < need:
            run += W[n]
            n += 1
    return np.array(order[:n]), e[order[:n]], sum(W[:n])


def probabilities(l, **rules) -> np.ndarray:
    idx, e, mass = kept(l, **rules)
    p = np.zeros(len(l), np.float32)
    p[idx] = (e * float(TWO43) / float(mass)).astype(np.float32)
    return p


def sample(l, word: int, **rules) -> int:
    return sample_fixed_point(probabilities(l, **rules), word)
