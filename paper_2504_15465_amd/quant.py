"""Weights in 4 bits: quantisation and the layout that GEMM_Q4 reads.

A weight row [K] is cut into groups of ``group`` consecutive k; a code q = 0 .. 15 of a group stands for
scale * (q - zero), with a scale and a zero point in bf16.  Plain torch, once per weight matrix.
"""
from __future__ import annotations

import torch


def quantize_q4(w: torch.Tensor, group: int, symmetric: bool = False):
    """[N, K] weights -> codes uint8 [N, K], scales bf16 [N, ceil(K / group)], zeros likewise (None if symmetric: zero 8).

    Codes are the nearest ones for the scale and zero point as bf16 holds them."""
    n, k = w.shape
    groups = -(-k // group)
    x = torch.nn.functional.pad(w.float(), (0, groups * group - k)).reshape(n, groups, group)
    live = (torch.arange(groups * group, device=w.device) < k).reshape(1, groups, group)
    if symmetric:
        scale = x.abs().amax(2) / 7.0
        zero = torch.full_like(scale, 8.0)
    else:
        lo = torch.where(live, x, torch.inf).amin(2)
        scale = ((torch.where(live, x, -torch.inf).amax(2) - lo) / 15.0).bfloat16()
        # weights that are equal, or less apart than bf16 can say: one step away from zero, so that code and zero point reproduce them
        for other in (lo.abs().bfloat16(), torch.ones_like(scale)):
            scale = torch.where(scale > 0, scale, other)
        zero = (-lo / scale.float()).bfloat16().float()
    scale = scale.bfloat16()
    s = scale.float()
    q = torch.where(s[:, :, None] > 0, x / s[:, :, None], 0.0) + zero[:, :, None]
    q = q.round().clamp(0, 15).to(torch.uint8).reshape(n, groups * group)[:, :k].contiguous()
    return q, scale, None if symmetric else zero.bfloat16()


def pack_q4(codes: torch.Tensor) -> torch.Tensor:
    """Codes [N, K] -> bytes [ceil(N/16), ceil(K/128), 4, 16, 16] (16 rows and 128 k together, in the order of the products' operands)."""
    n, k = codes.shape
    nt, kc = -(-n // 16), -(-k // 128)
    x = torch.nn.functional.pad(codes, (0, kc * 128 - k, 0, nt * 16 - n))
    # k = 32 t + 8 p + 4 h + j  ->  piece p, dword t, byte j, half h
    x = x.reshape(nt, 16, kc, 4, 4, 2, 4).permute(0, 2, 4, 1, 3, 6, 5)      # nt, kc, p, row, t, j, h
    return (x[..., 0] | (x[..., 1] << 4)).reshape(nt, kc, 4, 16, 16).contiguous()


def unpack_q4(packed: torch.Tensor, n: int, k: int) -> torch.Tensor:
    """The inverse of ``pack_q4``."""
    nt, kc = packed.shape[:2]
    x = packed.reshape(nt, kc, 4, 16, 4, 4)
    x = torch.stack([x & 15, x >> 4], 5)                                     # nt, kc, p, row, t, h, j
    return x.permute(0, 3, 1, 4, 2, 5, 6).reshape(nt * 16, kc * 128)[:n, :k].contiguous()


def pack_q4_groups(x: torch.Tensor) -> torch.Tensor:
    """Scales or zero points [N, groups] -> bf16 [ceil(N/16), groups, 16]."""
    n, groups = x.shape
    nt = -(-n // 16)
    x = torch.nn.functional.pad(x.bfloat16(), (0, 0, 0, nt * 16 - n))
    return x.reshape(nt, 16, groups).transpose(1, 2).contiguous()
