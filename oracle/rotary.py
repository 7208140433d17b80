"""Oracle: rotary positions, pair by pair, in float64.

TEST INFRASTRUCTURE ONLY -- never imported by the product path.
"""
import math

import numpy as np


def rotary_angles(dim, base=10000.0, scaling="none", factor=1.0, original_len=0, fast=32.0, slow=1.0):
    """theta_j of every pair, and the magnitude m."""
    if scaling == "ntk":
        base = base * factor ** (dim / (dim - 2))
    theta = np.array([base ** (-2.0 * j / dim) for j in range(dim // 2)])
    if scaling == "linear":
        theta = theta / factor
    if scaling == "yarn":
        for j, t in enumerate(theta):
            g = min(1.0, max(0.0, (original_len * t / (2 * math.pi) - slow) / (fast - slow)))
            theta[j] = (1 - g) * t / factor + g * t
    return theta, 0.1 * math.log(factor) + 1.0 if scaling == "yarn" else 1.0


def rotate(x, pos, theta, m, layout):
    """x [..., Dh] of one position each: pos broadcasts against x[..., 0]."""
    y = np.array(x, dtype=np.float64)
    half = len(theta)
    for j, t in enumerate(theta):
        p, q = (j, j + half) if layout == "half" else (2 * j, 2 * j + 1)
        a = np.asarray(pos, dtype=np.float64) * t
        y[..., p] = m * (x[..., p] * np.cos(a) - x[..., q] * np.sin(a))
        y[..., q] = m * (x[..., q] * np.cos(a) + x[..., p] * np.sin(a))
    return y
