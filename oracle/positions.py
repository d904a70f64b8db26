"""Rotary positions in 64 bits: every pair (x, y) of a row at position p becomes m (x cos a - y sin a, x sin a + y cos a), a = p f."""
import math

import numpy as np


def frequencies(rot, base=10000.0, scaling="none", factor=1.0, original_length=0, beta_fast=32.0, beta_slow=1.0):
    """(radians per position of pair i, factor on the rotated values), one pair at a time."""
    out = []
    for i in range(rot // 2):
        if scaling == "ntk":
            f = (base * factor ** (rot / (rot - 2))) ** (-2.0 * i / rot)
        else:
            f = base ** (-2.0 * i / rot)
        if scaling == "linear":
            f /= factor
        if scaling == "yarn":
            turns = original_length * f / (2 * math.pi)
            if turns <= beta_slow:
                f /= factor
            elif turns < beta_fast:
                keep = (turns - beta_slow) / (beta_fast - beta_slow)
                f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return np.array(out), (0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0)


def pairs(rot, interleaved):
    """Columns of the first and of the second member of each pair."""
    i = np.arange(rot // 2)
    return (2 * i, 2 * i + 1) if interleaved else (i, i + rot // 2)


def rotate(x, positions, freq, interleaved, magnitude=1.0, inverse=False):
    """x [B,H,N,d], positions [B,N]."""
    x = np.asarray(x, dtype=np.float64)
    a = np.asarray(positions, dtype=np.float64)[:, None, :, None] * freq * (-1.0 if inverse else 1.0)
    u, v = pairs(2 * len(freq), interleaved)
    y = x.copy()
    y[..., u] = magnitude * (x[..., u] * np.cos(a) - x[..., v] * np.sin(a))
    y[..., v] = magnitude * (x[..., u] * np.sin(a) + x[..., v] * np.cos(a))
    return y
