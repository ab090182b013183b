"""Tables for the position rotation that the append applies on its way into the cache (host-side set-up, once per
model: the library reads a table's rows, whatever frequencies they were made with)."""
from __future__ import annotations

import math

import torch


def rope_table(num_positions: int, rotary_dim: int = 64, theta: float = 10000.0, factor: float = 1.0,
               original_positions: int = 4096, beta_fast: float = 32.0, beta_slow: float = 1.0,
               device="cpu", truncate: bool = True) -> torch.Tensor:
    """float32 [num_positions][rotary_dim]: the cosines of a position's rotary_dim / 2 angles, then their sines.

    Frequencies theta^(-2 i / rotary_dim).  factor > 1 stretches the context from ``original_positions`` the way
    long-context models are trained for (interpolation by frequency, Peng et al., "YaRN", 2023): a frequency that
    turns more than beta_fast times over the original context stays, one that turns less than beta_slow times is
    divided by the factor, those between are blended linearly in i, and cosines and sines carry the factor
    0.1 ln(factor) + 1.  The two ends of the blend are rounded outwards to whole i (truncate=True, the method's first
    implementation and most models since) or taken as they are (truncate=False: the gpt-oss family, with theta 150000,
    factor 32 and 4096 original positions); a model needs the table it was trained with, the two differ by up to 76 %
    there.  Angles are formed in 64 bits: at position 100000 a float32 angle is off by up to 4e-3."""
    if rotary_dim <= 0 or rotary_dim % 2 or num_positions < 1 or factor < 1.0:
        raise ValueError("rotary_dim must be even and positive, num_positions at least 1, factor at least 1")
    if factor > 1.0 and (theta <= 1.0 or original_positions < 1 or not 0.0 < beta_slow <= beta_fast):
        raise ValueError("a stretched table needs theta above 1, original_positions at least 1 and 0 < beta_slow <= beta_fast")
    i = torch.arange(rotary_dim // 2, dtype=torch.float64, device=device)
    freq = theta ** (-2.0 * i / rotary_dim)
    gain = 1.0
    if factor > 1.0:
        def turns_at(turns):     # the i whose frequency makes `turns` turns over the original context
            return rotary_dim * math.log(original_positions / (turns * 2.0 * math.pi)) / (2.0 * math.log(theta))
        lo, hi = turns_at(beta_fast), turns_at(beta_slow)
        if truncate:
            lo, hi = math.floor(lo), math.ceil(hi)
        lo, hi = max(lo, 0), min(hi, rotary_dim - 1)
        slow = torch.clamp((i - lo) / max(hi - lo, 1e-3), 0.0, 1.0)
        freq = freq * (1.0 - slow) + freq / factor * slow
        gain = 0.1 * math.log(factor) + 1.0
    angle = torch.arange(num_positions, dtype=torch.float64, device=device)[:, None] * freq[None, :]
    return torch.cat([angle.cos() * gain, angle.sin() * gain], dim=1).to(torch.float32).contiguous()
