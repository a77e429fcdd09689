"""Norm and position rotation of a row's heads (TEST INFRASTRUCTURE ONLY).

  y = gain * x / sqrt(mean(x^2) + eps)        over a head's entries (optional)
  (y_a, y_b) -> (y_a cos t - y_b sin t, y_b cos t + y_a sin t),  t = position * freq_j
for the pairs j < rotary_dim / 2 of dims (j, j + rotary_dim / 2), or (2j, 2j + 1) if
interleaved.  All arithmetic is float64.
"""
from __future__ import annotations

import numpy as np


def freqs(rotary_dim: int, base: float) -> np.ndarray:
    return base ** (-2.0 * np.arange(rotary_dim // 2) / rotary_dim)


def pairs(rotary_dim: int, interleaved: bool):
    j = np.arange(rotary_dim // 2)
    return (2 * j, 2 * j + 1) if interleaved else (j, j + rotary_dim // 2)


def norm(x: np.ndarray, gain, eps: float) -> np.ndarray:
    x = np.asarray(x, np.float64)
    if gain is None:
        return x.copy()
    with np.errstate(invalid="ignore", divide="ignore"):
        return np.asarray(gain, np.float64) * x / np.sqrt((x * x).mean(-1, keepdims=True) + eps)


def rotate(y: np.ndarray, positions: np.ndarray, freq: np.ndarray, interleaved: bool) -> np.ndarray:
    """y [batch, n, heads, head_dim], positions [batch, n]."""
    out = np.array(y, np.float64)
    a, b = pairs(2 * len(freq), interleaved)
    t = np.asarray(positions, np.float64)[:, :, None, None] * freq
    ya, yb = out[..., a], out[..., b]
    out[..., a], out[..., b] = ya * np.cos(t) - yb * np.sin(t), yb * np.cos(t) + ya * np.sin(t)
    return out


def apply(x, positions, freq, interleaved=False, gain=None, eps=0.0) -> np.ndarray:
    return rotate(norm(x, gain, eps), positions, np.asarray(freq, np.float64), interleaved)
