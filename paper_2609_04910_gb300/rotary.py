"""Frequencies of rotary positions, as ``gauss_sum_rotary`` takes them.

Pair i of R rotated channels turns by f_i = base^(-2i/R) radians per position.
Contexts longer than those a network was trained on stretch the frequencies:

- ``linear``: f_i / factor (positions interpolated);
- ``ntk``: base x factor^(R / (R - 2)), so that the slowest pair is stretched
  by the factor and the fastest not at all;
- ``yarn``: pairs up to the one that turns ``fast`` times over the original
  context keep f_i, pairs from the one that turns ``slow`` times on get
  f_i / factor, and the rotated channels are multiplied by 0.1 ln(factor) + 1,
  as in arXiv 2309.00071.  Between the two, f_i is blended linearly in the
  pair's index i, from the first bound rounded down to the second rounded up:
  the form that trained networks use.  (That paper states the blend linear in
  the number of turns, which gives other frequencies in the band.)

The table holds turns per position as 64-bit fractions of a turn, so that
position x frequency modulo 2^64 is the angle with no loss at any position.
"""
from __future__ import annotations

import math

SCALINGS = ("none", "linear", "ntk", "yarn")


def angular_frequencies(rotary_dim, base=10000.0, scaling="none", factor=1.0,
                        original_length=None, fast=32.0, slow=1.0):
    """(radians per position of each pair, scale of the rotated channels)."""
    R = int(rotary_dim)
    if R < 0 or R % 2:
        raise ValueError("rotary_dim must be even and >= 0")
    if scaling not in SCALINGS:
        raise ValueError(f"scaling must be one of {SCALINGS}")
    if not (math.isfinite(base) and base > 1.0):
        raise ValueError("base must be finite and > 1")
    if not (math.isfinite(factor) and factor >= 1.0):
        raise ValueError("factor must be finite and >= 1")
    if scaling == "ntk":
        base = base * factor ** (R / max(1.0, R - 2.0))
    freqs = [base ** (-2.0 * i / R) for i in range(R // 2)]
    if scaling == "linear":
        freqs = [f / factor for f in freqs]
    if scaling != "yarn":
        return freqs, 1.0
    if original_length is None or not original_length > 0:
        raise ValueError("yarn scaling needs the original context length")
    if not fast > slow > 0:
        raise ValueError("yarn scaling needs fast > slow > 0")

    def pair_of(turns):
        """The (fractional) pair that turns so many times over the original context."""
        return R * math.log(original_length / (turns * 2.0 * math.pi)) / (2.0 * math.log(base))

    low = max(0.0, math.floor(pair_of(fast)))
    high = min(R - 1.0, math.ceil(pair_of(slow)))
    if high <= low:
        high = low + 0.001
    for i, f in enumerate(freqs):
        ramp = min(1.0, max(0.0, (i - low) / (high - low)))
        freqs[i] = f * (1.0 - ramp) + f / factor * ramp
    return freqs, 0.1 * math.log(factor) + 1.0


def fixed_point(freqs):
    """Radians per position as signed 64-bit fractions of a turn."""
    table = []
    for f in freqs:
        t = int(round(f / (2.0 * math.pi) * 2.0 ** 64)) % (1 << 64)
        table.append(t - (1 << 64) if t >= 1 << 63 else t)
    return table


def rotary_frequencies(rotary_dim, base=10000.0, scaling="none", factor=1.0,
                       original_length=None, fast=32.0, slow=1.0, device="cuda"):
    """(int64 (R/2,) tensor for ``gauss_sum_rotary``, its ``scale`` argument)."""
    import torch
    freqs, scale = angular_frequencies(rotary_dim, base, scaling, factor, original_length, fast,
                                       slow)
    return torch.tensor(fixed_point(freqs), dtype=torch.int64, device=device), scale
