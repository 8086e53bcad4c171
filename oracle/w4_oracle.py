"""4-bit weights and the norm between a layer's halves, by their definitions, in 64 bits (numpy)."""
from __future__ import annotations

import numpy as np

GROUP = 32
E2M1 = np.array([0.0, 0.5, 1.0, 1.5, 2.0, 3.0, 4.0, 6.0])
E2M1 = np.concatenate([E2M1, -E2M1])


def quantize(w):
    """fp32 [..., cols] -> (bytes of two codes [..., cols / 2], scale bytes [..., cols / 32]): a group's scale is the smallest
    2^e (-120 <= e <= 120) that leaves no magnitude above 7 * 2^e; the nearest code, ties to the even one."""
    x = np.asarray(w, np.float64).reshape(*w.shape[:-1], -1, GROUP)
    e = np.full(x.shape[:-1], -120)
    while True:
        grow = (np.abs(x).max(-1) > 7.0 * 2.0 ** e) & (e < 120)
        if not grow.any():
            break
        e = e + grow
    y = np.abs(x) / 2.0 ** e[..., None]
    off = np.abs(y[..., None] - E2M1[:8])
    best = off.min(-1, keepdims=True)
    even_first = np.array([0, 2, 4, 6, 1, 3, 5, 7])  # of two codes equally near one is even
    code = even_first[np.argmax((off == best)[..., even_first], -1)]
    code = np.where(y > 6.0, 7, code) + 8 * np.signbit(x)
    code = code.reshape(w.shape).astype(np.uint8)
    return code[..., 0::2] | code[..., 1::2] << 4, (e + 127).astype(np.uint8)


def values(q, s):
    """The weights that codes and scale bytes stand for, fp64 [..., cols]."""
    v = np.stack([E2M1[q & 15], E2M1[q >> 4]], -1).reshape(*q.shape[:-1], -1, GROUP)
    return (v * 2.0 ** (s.astype(np.float64) - 127)[..., None]).reshape(*q.shape[:-1], -1)


def pack(q, s):
    """The packed layout, byte by byte from its definition: (codes, scales) of one [rows, cols] matrix."""
    rows, half = q.shape
    cols = 2 * half
    packed = np.empty(rows * half, np.uint8)
    chunks = -(-cols // 512)
    scales = np.full(rows // 16 * chunks * 256, 127, np.uint8)
    nb = cols // 128
    for row in range(rows):
        g, r = divmod(row, 16)
        for b in range(nb):
            for kq in range(4):
                for j in range(4):
                    at = (g * nb + b) * 1024 + 256 * kq + 16 * r + 4 * j
                    first = (128 * b + 32 * j + 8 * kq) // 2
                    packed[at:at + 4] = q[row, first:first + 4]
        for i in range(cols // GROUP):
            scales[(g * chunks + i // 16) * 256 + 16 * r + i % 16] = s[row, i]
    return packed, scales


def add_norm(x, residual, weight, eps, offset=0.0):
    """(sum, norm) of fp64 rows."""
    z = x if residual is None else x + residual
    y = z / np.sqrt((z * z).mean(-1, keepdims=True) + eps)
    return z, y if weight is None else y * (weight + offset)
