"""Rotary positions and head norms in float64.

Pair j of the first `dim` dimensions of a head, (j, j + dim / 2) or, interleaved, (2 j, 2 j + 1), turns by position
times freq[j] radians.
"""
from __future__ import annotations

import math

import numpy as np


def frequencies(dim, theta, kind=None, factor=1.0, context=0.0, low=1.0, high=4.0):
    """(freq [dim / 2], factor of cosine and sine)."""
    freq, scale = [], 1.0
    for j in range(dim // 2):
        if kind == "base":
            freq.append((theta * factor ** (dim / (dim - 2))) ** (-2 * j / dim))
            continue
        f = theta ** (-2 * j / dim)
        if kind == "linear":
            f /= factor
        elif kind == "by_rotations":
            turns = context * f / (2 * math.pi)
            if turns <= low:
                f /= factor
            elif turns < high:
                f *= 1 / factor + (1 - 1 / factor) * (turns - low) / (high - low)
        elif kind == "by_index":
            # the pair that makes r turns: context theta^(-2j/dim) = 2 pi r
            first, last = (dim / 2 * math.log(context / (2 * math.pi * r)) / math.log(theta) for r in (high, low))
            first, last = max(math.floor(first), 0), min(math.ceil(last), dim - 1)
            scaled = min(max((j - first) / max(last - first, 1e-3), 0.0), 1.0)
            f *= scaled / factor + 1 - scaled
            scale = 1 + math.log(factor) / 10
        freq.append(f)
    return np.array(freq), scale


def norm(x, gain, eps):
    """x [..., D] over its root mean square, times gain."""
    return x / np.sqrt((x * x).mean(-1, keepdims=True) + eps) * gain


def rotate(x, pos, freq, scale=1.0, interleaved=False):
    """x [H][D] at one position."""
    half = len(freq)
    first = np.arange(half) * 2 if interleaved else np.arange(half)
    second = first + 1 if interleaved else first + half
    angle = pos * np.asarray(freq, np.float64)
    c, s = np.cos(angle) * scale, np.sin(angle) * scale
    y = np.array(x, np.float64)
    y[..., first] = x[..., first] * c - x[..., second] * s
    y[..., second] = x[..., second] * c + x[..., first] * s
    return y
