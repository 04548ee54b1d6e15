"""Tensors of the verify step in 4 bits: weights packed once, an empty paged cache, the rotation's table.

The formats are those of include/spade.h: value = scale * (code - zero), (scale, zero) pairs of
float16 per group, eight codes to a word whose 4-bit fields hold numbers 0, 2, 4, 6, 1, 3, 5, 7.
Set-up code in torch; nothing here is on a verify step's path.
"""
from __future__ import annotations

import torch

KV_GROUP = 64        # dims of a head per (scale, zero) pair of the cache
MAX_SCALE = 4364.0   # 15 steps of it stay within float16


def pack_codes(codes):
    """Codes [..., n] in 0 .. 15 (n a multiple of 8) as bytes [..., n / 2]."""
    fields = codes.to(torch.uint8).reshape(codes.shape[:-1] + (-1, 4, 2)).transpose(-1, -2)
    fields = fields.reshape(codes.shape[:-1] + (codes.shape[-1] // 2, 2))
    return (fields[..., 0] | (fields[..., 1] << 4)).contiguous()


def unpack_codes(packed):
    """Bytes [..., n / 2] as codes [..., n]."""
    fields = torch.stack((packed & 15, packed >> 4), -1)
    n = 2 * packed.shape[-1]
    return fields.reshape(packed.shape[:-1] + (n // 8, 2, 4)).transpose(-1, -2).reshape(packed.shape[:-1] + (n,))


def quantize(x, group):
    """Numbers x [..., n] as (codes [..., n / 2] uint8, params [..., n / group, 2] float16): the rule by which
    the cache is written, and how spade_linear_w4's weights can be made (group 32, 64 or 128)."""
    g = x.float().reshape(x.shape[:-1] + (x.shape[-1] // group, group))
    finite = g.isfinite().all(-1)
    lo, hi = g.amin(-1).clamp(max=0), g.amax(-1).clamp(min=0)
    scale = ((hi - lo) * (1 / 15)).clamp(max=MAX_SCALE).to(torch.float16).float()
    real = finite & (scale > 0)
    step = torch.where(real, scale, torch.ones_like(scale))
    zero = torch.where(real, torch.round(-lo / step).clamp(0, 15), torch.zeros_like(scale))
    codes = (torch.round(g / step[..., None]) + zero[..., None]).clamp(0, 15)
    codes = torch.where(real[..., None], codes, torch.zeros_like(codes)).reshape(x.shape)
    scale = torch.where(finite, scale, torch.full_like(scale, float("nan")))
    return pack_codes(codes), torch.stack((scale, zero), -1).to(torch.float16)


def dequantize(codes, params):
    """The values (float32 [..., n]) that codes [..., n / 2] and params [..., n / group, 2] stand for."""
    c = unpack_codes(codes).float()
    p = params.float()[..., None]
    g = c.reshape(c.shape[:-1] + (params.shape[-2], c.shape[-1] // params.shape[-2]))
    return (p[..., 0, :] * (g - p[..., 1, :])).reshape(c.shape)


def kv4_pools(num_pages, Hkv, page_size, D, device="cuda"):
    """An empty 4-bit cache: (k_codes, k_params, v_codes, v_params)."""
    def codes():
        return torch.zeros((num_pages, Hkv, page_size, D // 2), dtype=torch.uint8, device=device)

    def params():
        return torch.zeros((num_pages, Hkv, page_size, D // KV_GROUP, 2), dtype=torch.float16, device=device)

    return codes(), params(), codes(), params()


def rope_table(theta, D, max_pos, device="cuda"):
    """(cos, sin) of pos * theta^(-2j/D), float32 [max_pos, D / 2, 2], from angles in float64."""
    freq = float(theta) ** (-torch.arange(D // 2, dtype=torch.float64) * 2 / D)
    angle = torch.arange(max_pos, dtype=torch.float64)[:, None] * freq
    return torch.stack((angle.cos(), angle.sin()), -1).to(torch.float32).to(device)
