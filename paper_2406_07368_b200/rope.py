"""Frequency tables for la_norm_rope: which angle per position each rotated pair of a head turns by, and the scalings by
which a model trained on short contexts is taken to long ones.  Host arithmetic in 64 bits; the rotation is the kernel's.
"""
from __future__ import annotations

import math

import torch


def inv_freq(rot: int, base: float = 10000.0, scaling: str = "none", factor: float = 1.0, trained_len: int = 0,
             fast: float = 32.0, slow: float = 1.0, device=None) -> tuple[torch.Tensor, float]:
    """(inv_freq [rot / 2] float64, mscale) for la_norm_rope.

    f_m = base^(-2m / rot), and, for contexts `factor` times as long as the trained ones:
      "none"    as it is
      "linear"  f_m / factor: positions are squeezed into the trained range
      "base"    the base raised by factor^(rot / (rot - 2)): the slowest pair turns `factor` times more slowly, the fastest
                as before
      "parts"   a pair that turns at least `fast` times over trained_len positions stays, one that turns at most `slow`
                times is squeezed, linearly between them in the number of turns; mscale = 1 + 0.1 ln(factor)
    """
    if rot < 2 or rot % 2:
        raise ValueError(f"rot must be even and at least 2, got {rot}")
    if not base > 0 or not factor >= 1:
        raise ValueError("base must be positive and factor at least 1")
    if scaling not in ("none", "linear", "base", "parts"):
        raise ValueError(f"unknown scaling {scaling!r}")
    m = torch.arange(rot // 2, dtype=torch.float64)
    mscale = 1.0
    if scaling == "base":
        if rot < 4:
            raise ValueError("scaling the base needs two pairs at least")
        base = base * factor ** (rot / (rot - 2))
    f = float(base) ** (-2.0 * m / rot)
    if scaling == "linear":
        f = f / factor
    elif scaling == "parts":
        if trained_len < 1 or not fast > slow:
            raise ValueError("scaling by parts needs trained_len and fast > slow")
        keep = ((trained_len * f / (2.0 * math.pi) - slow) / (fast - slow)).clamp(0.0, 1.0)
        f = f * keep + f / factor * (1.0 - keep)
        mscale = 1.0 + 0.1 * math.log(factor)
    return f.to(device) if device is not None else f, mscale
