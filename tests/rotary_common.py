"""Rotary positions in plain form and 64 bits (CPU)."""

import torch


def frequencies(R, base=10000.0):
    return base ** (-torch.arange(0, R, 2, dtype=torch.float64) / R)


def turned(x, positions, freq, layout="half", scale=1.0, transpose=False):
    """x [n][heads][d] turned, in float64."""
    R = 2 * len(freq)
    a = positions.double()[:, None] * freq
    c, s = scale * a.cos()[:, None], scale * a.sin()[:, None] * (-1.0 if transpose else 1.0)
    y = x.double().clone()
    first = slice(0, R // 2) if layout == "half" else slice(0, R, 2)
    second = slice(R // 2, R) if layout == "half" else slice(1, R, 2)
    u, v = x.double()[..., first], x.double()[..., second]
    y[..., first], y[..., second] = u * c - v * s, v * c + u * s
    return y


def bound(x, want, dtype, scale=1.0):
    """How far a turned value may be off: products and cosines in 64 bits (a few 2^-53 of the pair), a rounding to float
    (2^-24) and for bfloat16 another one (2^-8)."""
    pair = x.double().abs().amax(-1, keepdim=True) * 2 * scale
    return pair * 2.0 ** -49 + want.abs() * (2.0 ** -24 + (2.0 ** -8 * 1.001 if dtype == torch.bfloat16 else 0.0)) + 1e-44
