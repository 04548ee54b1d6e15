"""Frequencies of the rotary embedding for spade_verify_rope, plain or stretched for long contexts.

Pair j of `dims` turning dims turns by theta^(-2j/dims) radians per position.  A model trained on
`context` positions is run on `factor` times as many by turning slower:
  "linear": every pair by 1 / factor (positions are interpolated);
  "ntk":    theta times factor^(dims / (dims - 2)): the slowest pair by 1 / factor, the fastest as it was;
  "bands":  by the turns r = context * frequency / (2 pi) that a pair makes over the trained context: as it
            was from r = high on, by 1 / factor up to r = low, linear in r between.  The defaults, low 1 and high 4,
            are those of the Llama-3.1 family, whose turned dims have no factor; others go up to high = 32, with the
            factor of attention_scale.
Set-up code in torch; nothing here is on a verify step's path.
"""
from __future__ import annotations

import math

import torch


def inv_freq(theta, dims, kind=None, factor=1.0, context=None, low=1.0, high=4.0, device="cuda"):
    """float64 [dims / 2] radians per position."""
    if dims < 2 or dims % 2 or not theta > 1:
        raise ValueError(f"dims must be even and theta > 1, got {dims} and {theta}")
    if kind not in (None, "linear", "ntk", "bands"):
        raise ValueError(f"unknown scaling {kind!r}")
    if kind is not None and not (factor >= 1 and math.isfinite(factor)):
        raise ValueError(f"factor must be finite and >= 1, got {factor}")
    if kind == "ntk":
        if dims < 4:
            raise ValueError("ntk needs at least 4 dims")
        theta = theta * factor ** (dims / (dims - 2))
    freq = float(theta) ** (-torch.arange(dims // 2, dtype=torch.float64) * 2 / dims)
    if kind == "linear":
        freq = freq / factor
    elif kind == "bands":
        if context is None or not 0 <= low < high:
            raise ValueError("bands needs the trained context and 0 <= low < high")
        keep = ((context * freq / (2 * math.pi) - low) / (high - low)).clamp(0, 1)
        freq = freq * keep + freq / factor * (1 - keep)
    return freq.to(device)


def attention_scale(factor):
    """0.1 ln(factor) + 1: the factor of the turned dims (mscale of spade_verify_rope) of models that were stretched with
    one.  It scales the scores by its square, so it is for a model whose configuration says so, and for no other."""
    return 0.1 * math.log(factor) + 1.0
