"""Rotary encoding in its published forms (oracle; test infrastructure only): float64 numpy, pairs as
complex numbers.

``frequencies`` gives the angles per position of a head's rotated pairs and the factor of the rotated
channels: plain theta^(-2i/r); positions divided by the factor ("linear"); a larger base ("ntk"); or a
ramp between the plain and the divided frequencies over the pairs that turn between ``fast`` and
``slow`` times within the ``trained`` rows ("yarn").
"""
from __future__ import annotations

import math
from typing import Tuple

import numpy as np


def frequencies(r: int, theta: float, scaling: str = "plain", factor: float = 1.0, trained: int = 1, fast: float = 32.0,
                slow: float = 1.0) -> Tuple[np.ndarray, float]:
    if scaling == "ntk":
        theta = theta * factor ** (r / (r - 2))
    f = np.array([math.exp(-2.0 * i / r * math.log(theta)) for i in range(r // 2)])
    if scaling == "linear":
        return f / factor, 1.0
    if scaling != "yarn":
        return f, 1.0

    def pair(turns):   # theta^(-2 i / r) trained = 2 pi turns
        return r / 2 * math.log(trained / (2 * math.pi * turns), theta)
    lo, hi = max(math.floor(pair(fast)), 0), min(math.ceil(pair(slow)), r - 1)
    w = np.clip((np.arange(r // 2) - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
    return f * (1 - w) + f / factor * w, 0.1 * math.log(factor) + 1.0


def rotate(x: np.ndarray, pos, freq: np.ndarray, m: float = 1.0, pairs: bool = False, back: bool = False) -> np.ndarray:
    """x [rows][heads][D]; the first 2 len(freq) channels turn.  ``pairs``: (2i, 2i + 1), otherwise
    (i, i + r/2).  ``back``: the transposed map (the gradient)."""
    y = np.array(x, np.float64)
    half = len(freq)
    turn = m * np.exp((-1j if back else 1j) * np.asarray(pos, np.float64)[:, None] * freq)[:, None, :]
    a, b = (slice(0, 2 * half, 2), slice(1, 2 * half, 2)) if pairs else (slice(0, half), slice(half, 2 * half))
    z = (y[..., a] + 1j * y[..., b]) * turn
    y[..., a], y[..., b] = z.real, z.imag
    return y
