"""Tables of angles for the key-value cache's rotary positions."""
from __future__ import annotations

import math

import torch

from .binding import LqError


def lq_rotary_table(positions: int, dim: int, base: float = 10000.0, stretch: float = 1.0, trained: int = 0, slow: float = 1.0,
                    fast: float = 32.0, amplitude: float = 1.0, device="cuda") -> torch.Tensor:
    """[positions][dim] fp32: amplitude * cos of the dim / 2 angles, then amplitude * sin.  The angle of pair i at position p is
    p * f_i, f_i = base ** (-2 i / dim), formed in 64 bits (at position 10^6 a 32-bit product is off by 0.06 rad).

    stretch > 1 fits a model to contexts that many times longer.  With trained = 0 every position is divided by it.  With the
    number of positions that the model was trained on, pairs that turn often over them (fast times or more) keep their angles, those that turn
    less than `slow` times are divided, and between the two a linear share of both is taken."""
    if positions < 1 or dim < 2 or dim % 2:
        raise LqError(f"expected positions >= 1 and an even dim >= 2, got {positions} and {dim}")
    if not (base > 0 and stretch >= 1 and trained >= 0 and fast > slow >= 0 and math.isfinite(amplitude)):
        raise LqError("expected base > 0, stretch >= 1, trained >= 0, fast > slow >= 0 and a finite amplitude")
    f = float(base) ** (-torch.arange(0, dim, 2, dtype=torch.float64) / dim)
    keep = ((trained * f / (2 * math.pi) - slow) / (fast - slow)).clamp(0, 1) if trained else torch.zeros_like(f)
    f = (f * (keep + (1 - keep) / stretch)).to(device)
    a = torch.arange(positions, dtype=torch.float64, device=device)[:, None] * f
    return (torch.cat([a.cos(), a.sin()], dim=1) * amplitude).float()
