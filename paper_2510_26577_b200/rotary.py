"""Frequencies for cast_append_kv: the angle per position of every rotating pair, in 64 bits, as models that keep or stretch
their context define them.

With d rotating dims and base b, pair i turns by theta_i = b^(-2i/d) radians per position; wavelength 2 pi / theta_i. To read
`factor` times the positions that a model was trained on:

  linear   every theta_i / factor
  ntk      the base grows so that the slowest pair turns `factor` times as slowly: b factor^(d / (d - 2))
  yarn     pairs with more than beta_fast turns in the trained context keep theta_i, those with fewer than beta_slow take
           theta_i / factor, between them a ramp over the pair's index; what is rotated is scaled by 0.1 ln(factor) + 1
  llama3   pairs with wavelength below context / high_freq_factor keep theta_i, above context / low_freq_factor take theta_i / factor,
           between them a ramp over context / wavelength

Host code, run once per model: the result is an input of the calls.
"""
from __future__ import annotations

import math
from typing import Tuple

import torch


def inverse_frequencies(rot_dim: int, base: float = 10000.0, *, scaling: str = "none", factor: float = 1.0, context: int = 0,
                        beta_fast: float = 32.0, beta_slow: float = 1.0, low_freq_factor: float = 1.0, high_freq_factor: float = 4.0,
                        device="cuda") -> Tuple[torch.Tensor, float]:
    """(inv_freq [rot_dim / 2] fp64, magnitude) for cast_append_kv. `context`: positions that the model was trained on
    (yarn and llama3 need it)."""
    if rot_dim < 2 or rot_dim % 2 or not base > 0 or not factor > 0:
        raise ValueError(f"rot_dim {rot_dim}, base {base}, factor {factor}")
    if scaling == "yarn" and not (base > 1 and beta_fast > 0 and beta_slow > 0):
        raise ValueError(f"yarn: base {base}, beta_fast {beta_fast}, beta_slow {beta_slow}")
    if scaling in ("yarn", "llama3") and context < 1:
        raise ValueError(f"{scaling} needs the context that the model was trained on")
    if scaling == "ntk":
        if rot_dim < 4:
            raise ValueError("ntk needs two pairs at least")
        base = base * factor ** (rot_dim / (rot_dim - 2))
    theta = torch.tensor([base ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)], dtype=torch.float64)
    magnitude = 1.0
    if scaling == "linear":
        theta = theta / factor
    elif scaling == "yarn":
        def pair_of(turns):  # index (not whole) of the pair that turns so often in the context
            return rot_dim * math.log(context / (turns * 2 * math.pi)) / (2 * math.log(base))
        lo = max(math.floor(pair_of(beta_fast)), 0)
        hi = min(math.ceil(pair_of(beta_slow)), rot_dim - 1)
        slow = ((torch.arange(rot_dim // 2, dtype=torch.float64) - lo) / max(hi - lo, 0.001)).clamp(0, 1)
        theta = theta / factor * slow + theta * (1 - slow)
        magnitude = 0.1 * math.log(factor) + 1.0 if factor > 1 else 1.0
    elif scaling == "llama3":
        if not high_freq_factor > low_freq_factor:
            raise ValueError(f"high_freq_factor {high_freq_factor} must exceed low_freq_factor {low_freq_factor}")
        keep = ((context * theta / (2 * math.pi) - low_freq_factor) / (high_freq_factor - low_freq_factor)).clamp(0, 1)
        theta = theta / factor * (1 - keep) + theta * keep
    elif scaling not in ("none", "ntk"):
        raise ValueError(f"scaling {scaling!r}")
    return theta.to(device), magnitude
