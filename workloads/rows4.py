"""4-bit rows with group scales, the form boa.matvec_4bit multiplies.

Offline, like the product-quantisation codes: per row and group of `group`
consecutive values, scale = (max - min) / 15 and offset = min, codes the
nearest of the 16 values scale * q + offset.
"""
from __future__ import annotations

import torch


def quantize(rows, group: int = 32, dtype=torch.float32):
    """(codes, scales, offsets) of float rows (N, K): codes uint8 (N, K / 2),
    value 2j in the low nibble of byte j; scales and offsets (N, K / group) of
    `dtype`. K must be a multiple of group, and even."""
    N, K = rows.shape
    if K % group or K % 2:
        raise ValueError("K must be even and a multiple of group")
    w = rows.float().reshape(N, K // group, group)
    lo, hi = w.amin(2), w.amax(2)
    scales = ((hi - lo) / 15).to(dtype)
    offsets = lo.to(dtype)
    step = scales.float().clamp(min=torch.finfo(torch.float32).tiny)
    q = ((w - offsets.float()[:, :, None]) / step[:, :, None]).round_().clamp_(0, 15).to(torch.uint8).reshape(N, K)
    return q[:, 0::2] | (q[:, 1::2] << 4), scales, offsets


def dequantize(codes, scales, offsets):
    """The rows that the codes stand for, in float32."""
    N, G = scales.shape
    q = torch.stack((codes & 15, codes >> 4), dim=2).reshape(N, G, -1).float()
    return (scales.float()[:, :, None] * q + offsets.float()[:, :, None]).reshape(N, -1)
