"""Rotary positions in float64 (test infrastructure): complex rotations, pair by pair."""

import math

import numpy as np


def frequencies(base, dims, scaling="plain", factor=1.0, low=1.0, high=4.0, original_len=8192):
    out = []
    for i in range(dims // 2):
        f = base ** (-2.0 * i / dims)
        own = 1.0
        if scaling == "linear":
            own = 0.0
        elif scaling == "rotations":
            own = (original_len * f / (2 * math.pi) - low) / (high - low)
        elif scaling == "channels":
            def pair(turns):
                return (dims * math.log(original_len / (2 * math.pi * turns)) /
                        (2 * math.log(base)))
            i1 = max(math.floor(pair(high)), 0)
            i0 = min(math.ceil(pair(low)), dims - 1)
            own = 1.0 - (i - i1) / max(i0 - i1, 0.001)
        own = min(1.0, max(0.0, own))
        out.append(f if scaling == "plain" else f * (own + (1 - own) / factor))
    return np.array(out)


def rotate(x, positions, freqs, adjacent=False, magnitude=1.0):
    """Rows x [..., d] at `positions` (broadcast to x's rows)."""
    x = np.array(x, dtype=np.float64)
    half = len(freqs)
    angle = np.asarray(positions, np.float64)[..., None] * freqs
    z = magnitude * np.exp(1j * np.remainder(angle, 2 * math.pi))
    a = slice(0, 2 * half, 2) if adjacent else slice(0, half)
    b = slice(1, 2 * half, 2) if adjacent else slice(half, 2 * half)
    turned = (x[..., a] + 1j * x[..., b]) * z
    x[..., a], x[..., b] = turned.real, turned.imag
    return x
