"""Rotary positions in fp64, from the definition: pairs as complex numbers, turned one axis at a time."""
from __future__ import annotations

import math

import numpy as np


def frequencies(pairs, base=10000.0, scaling="none", factor=1.0, original_len=4096.0, beta_fast=32.0, beta_slow=1.0):
    """(radians a position per pair, factor of the rotated values)."""
    if scaling == "ntk":
        base = base * factor ** (pairs / (pairs - 1))
    out = []
    for i in range(pairs):
        f = math.exp(-i / pairs * math.log(base))
        if scaling == "linear":
            f /= factor
        if scaling == "yarn":
            turns = original_len / (2 * math.pi / f)
            keep = min(1.0, max(0.0, (turns - beta_slow) / (beta_fast - beta_slow)))
            f = keep * f + (1 - keep) * f / factor
        out.append(f)
    return np.array(out), (1 + 0.1 * math.log(factor) if scaling == "yarn" else 1.0)


def rotate(x, inv_freq, positions=None, layout="half", axis_pairs=None, scale=1.0, backward=False):
    """x fp64 [B][H][N][d]; positions int [axes][B][N]."""
    x = np.asarray(x, dtype=np.float64)
    b, _, n, _ = x.shape
    p = len(inv_freq)
    axis_pairs = [p] if axis_pairs is None else axis_pairs
    if positions is None:
        positions = np.broadcast_to(np.arange(n), (1, b, n))
    axis = np.repeat(np.arange(len(axis_pairs)), axis_pairs)
    angle = np.asarray(positions, dtype=np.float64)[axis].transpose(1, 2, 0) * inv_freq   # [B][N][P]
    z = scale * np.exp((-1j if backward else 1j) * angle)[:, None]
    first = slice(0, 2 * p, 2) if layout == "interleaved" else slice(0, p)
    second = slice(1, 2 * p, 2) if layout == "interleaved" else slice(p, 2 * p)
    w = (x[..., first] + 1j * x[..., second]) * z
    out = x.copy()
    out[..., first], out[..., second] = w.real, w.imag
    return out
