"""Oracle: rotary positions and their frequencies (test infrastructure only).

Plain float64 NumPy from the definition: pair i of a head at position p is the complex number x1 + i x2, multiplied by
g e^(i p f_i) (inverse: g e^(-i p f_i)).

Pins: tests/test_oracle_rotary.py.
"""

from __future__ import annotations

import numpy as np


def frequencies(r: int, base: float, scaling=None, factor: float = 1.0, original_len: int = 0, beta_fast: float = 32.0,
                beta_slow: float = 1.0):
    """(f [r / 2], g)."""
    f = np.array([base ** (-2.0 * i / r) for i in range(r // 2)])
    if scaling == "linear":
        return f / factor, 1.0
    if scaling == "ntk":
        return frequencies(r, base * factor ** (r / (r - 2)))
    if scaling == "yarn":
        keep = np.array([(original_len * v / (2 * np.pi) - beta_slow) / (beta_fast - beta_slow) for v in f])
        keep = np.minimum(np.maximum(keep, 0.0), 1.0)
        return (1 - keep) * f / factor + keep * f, 0.1 * np.log(factor) + 1.0
    return f, 1.0


def pair_channels(r: int, layout: str):
    """(first, second) channel of each pair."""
    i = np.arange(r // 2)
    return (i, i + r // 2) if layout == "half" else (2 * i, 2 * i + 1)


def rotary(x: np.ndarray, positions: np.ndarray, f: np.ndarray, layout: str, g: float = 1.0, inverse: bool = False):
    """x [rows, H, d] turned by positions [rows], in float64."""
    y = x.astype(np.float64)
    a, b = pair_channels(2 * len(f), layout)
    angle = positions.astype(np.float64)[:, None] * f[None]
    w = g * np.exp((-1j if inverse else 1j) * angle)[:, None]
    z = (y[..., a] + 1j * y[..., b]) * w
    y[..., a], y[..., b] = z.real, z.imag
    return y
