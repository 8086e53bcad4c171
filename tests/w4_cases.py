"""Inputs of the GPU tests with 4-bit weights."""
from __future__ import annotations

import numpy as np
import torch

from oracle import w4_oracle as wo


def packed(moe, q, s):
    """Row-major codes and scales (numpy, [rows, ..] or [mats, rows, ..]) -> packed device tensors."""
    dq, ds = torch.from_numpy(q).cuda(), torch.from_numpy(s).cuda()
    mats, rows, half = q.shape if q.ndim == 3 else (1, *q.shape)
    w = torch.empty_like(dq)
    ws = torch.empty(moe.moe_w4_scale_bytes(mats, rows, 2 * half), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    moe.moe_pack_weight_w4(dq, ds, w, ws, status)
    assert int(status.item()) == 0
    return w, ws


def whole(rng, *shape):
    """Codes and scales whose products with small whole numbers add up without rounding: multiples of 1/4 up to 12."""
    q = rng.integers(0, 256, (*shape[:-1], shape[-1] // 2)).astype(np.uint8)
    s = rng.integers(126, 129, (*shape[:-1], shape[-1] // 32)).astype(np.uint8)
    return q, s


def ordinary(rng, *shape):
    """Weights of the size that keeps a product's outputs at its inputs' size: any codes, scales around that."""
    q = rng.integers(0, 256, (*shape[:-1], shape[-1] // 2)).astype(np.uint8)
    middle = 125 - int(round(np.log2(shape[-1]) / 2))
    return q, rng.integers(middle - 1, middle + 2, (*shape[:-1], shape[-1] // 32)).astype(np.uint8)


def values(q, s):
    """What the weights stand for, fp64 on the device (from the oracle's table; the powers are exact)."""
    table = torch.from_numpy(wo.E2M1).cuda()
    c = torch.from_numpy(q).cuda().int()
    v = torch.stack([table[c & 15], table[c >> 4]], -1).reshape(*q.shape[:-1], -1, wo.GROUP)
    power = torch.ldexp(torch.ones(1, dtype=torch.float64, device="cuda"), torch.from_numpy(s).cuda().int() - 127)
    return (v * power[..., None]).flatten(-2)


def on_canvas(rows, cols, stride, dtype, fill=float("nan")):
    """A [rows, cols] view of a larger tensor full of `fill`, and the tensor."""
    canvas = torch.full((rows + 2, stride), fill, dtype=dtype, device="cuda")
    return canvas[1:rows + 1, :cols], canvas


def untouched(canvas, rows, cols):
    """Whether only the view's own part of the canvas has been written."""
    c = canvas.clone()
    c[1:rows + 1, :cols] = float("nan")
    return bool(torch.isnan(c.float()).all())
