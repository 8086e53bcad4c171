"""Plain numpy oracle of the attention half of a decoder layer (test infrastructure only).

Rotary positions and the e4m3 cache rows are stated in fp32, operation by
operation, as the library defines them (bit for bit comparable); attention in
fp64, with the error that the definition's own roundings may cause beside
every value.
"""
from __future__ import annotations

import numpy as np

from .moe_oracle import E4M3_MAX, bf16_to_f32, e4m3_decode, e4m3_encode

BF16_ROUNDOFF = 2.0 ** -8  # half the spacing of bf16 above 1: 7 stored bits of mantissa
TWO_BF16_ROUNDOFF = 2.0 ** -16  # a number as a rounded bf16 and the rounded rest, which is at most 2^-8 of it


def rope_frequencies(rot_dim, base, scaling="plain", factor=1.0, original_len=1.0, slow_turns=1.0, fast_turns=32.0):
    """fp64 [rot_dim / 2] angle per position of each pair."""
    g = [float(base) ** (-2.0 * i / rot_dim) for i in range(rot_dim // 2)]
    if scaling == "plain":
        return np.array(g)
    if scaling == "linear":
        return np.array(g) / factor
    out = []
    for f in g:
        turns = original_len * f / (2.0 * np.pi)
        w = min(1.0, max(0.0, (turns - slow_turns) / (fast_turns - slow_turns)))
        out.append((1.0 - w) * f / factor + w * f)
    return np.array(out)


def rope_table(n_pos, freqs, magnitude=1.0):
    """fp32 [n_pos, 2 len(freqs)]: cosines, then sines."""
    a = np.arange(n_pos, dtype=np.float64)[:, None] * freqs[None]
    return np.concatenate([np.cos(a) * magnitude, np.sin(a) * magnitude], 1).astype(np.float32)


def rotate(x, row, interleaved):
    """fp32 x [T, heads, dim] turned by table rows [T, rot]: products and sums rounded one by one."""
    y = x.astype(np.float32).copy()
    half = row.shape[1] // 2
    for i in range(half):
        lo, hi = (2 * i, 2 * i + 1) if interleaved else (i, i + half)
        c, s = row[:, i][:, None], row[:, half + i][:, None]
        a, b = x[..., lo].astype(np.float32), x[..., hi].astype(np.float32)
        y[..., lo] = a * c - b * s
        y[..., hi] = b * c + a * s
    return y


def quantize_head_rows(x):
    """fp32 [..., dim] -> e4m3 codes and one fp32 scale max|x| / 448 per row."""
    x = np.asarray(x, np.float32)
    s = (np.abs(x).max(-1) / np.float32(E4M3_MAX)).astype(np.float32)
    safe = np.where(s > 0, s, np.float32(1.0))[..., None]
    return e4m3_encode(np.where(s[..., None] > 0, x / safe, x).astype(np.float32)), s


def cached_rows(codes, scales):
    """fp32 values that codes [..., dim] with scales [...] stand for (one rounding)."""
    return e4m3_decode(codes).astype(np.float32) * scales[..., None].astype(np.float32)


def attention(q, k, v, scale, visible=None, numerators=BF16_ROUNDOFF):
    """fp64 attention of rows q [n, dim] over k, v [t, dim] and a bound on a kernel's error.

    visible: bool [n, t] (None: all).  Returns (out [n, dim], bound [n, dim]).

    The bound follows from the roundings of the definition: the softmax's
    numerators are rounded to bf16 for the product with v (unit roundoff 2^-8, 8
    significant bits, of every term; `numerators`: TWO_BF16_ROUNDOFF where they are
    two bf16 each), the result to bf16 (2^-8 of it); scores are sums of dim products
    in fp32, so a score is off by at most (dim + 8) 2^-24 of the sum of its terms'
    magnitudes, which moves its numerator by that much relatively and the
    denominator no more; 2^-18 covers the exponential, the sums' fp32 roundings
    and the joining of partial results.
    """
    q, k, v = (np.asarray(x, np.float64) for x in (q, k, v))
    n, dim = q.shape
    if k.shape[0] == 0 or n == 0:
        return np.zeros((n, v.shape[1])), np.full((n, v.shape[1]), 1e-30)
    s = scale * (q @ k.T)
    size = scale * (np.abs(q) @ np.abs(k).T)
    if visible is None:
        visible = np.ones(s.shape, bool)
    s = np.where(visible, s, -np.inf)
    top = s.max(1, keepdims=True)
    top = np.where(np.isfinite(top), top, 0.0)
    p = np.exp(s - top)
    total = p.sum(1, keepdims=True)
    p = p / np.where(total > 0, total, 1.0)
    out, terms = p @ v, p @ np.abs(v)
    seen = np.where(p > 2.0 ** -40, size, 0.0).max(1, keepdims=True)
    moved = 2.0 * (dim + 8) * 2.0 ** -24 * seen + 2.0 ** -18
    return out, (numerators + moved) * terms + BF16_ROUNDOFF * np.abs(out) + 1e-30


def packed_attention(q, k, v, cu_q, cu_k, scale, causal, want=None):
    """q [Tq, hq, dim], k, v [Tk, hkv, dim] fp values, cu_*: offsets.  (out, bound) fp64 [Tq, hq, dim]; rows outside all
    sequences are NaN.  want: only these heads."""
    hq, hkv = q.shape[1], k.shape[1]
    out = np.full(q.shape, np.nan)
    bound = np.zeros(q.shape)
    for b in range(len(cu_q) - 1):
        a, z, c, e = cu_q[b], cu_q[b + 1], cu_k[b], cu_k[b + 1]
        vis = (np.arange(e - c)[None] <= np.arange(z - a)[:, None] + (e - c) - (z - a)) if causal else None
        for h in (range(hq) if want is None else want):
            g = h // (hq // hkv)
            out[a:z, h], bound[a:z, h] = attention(q[a:z, h], k[c:e, g], v[c:e, g], scale, vis)
    return out, bound


def bf16_values(bits):
    return bf16_to_f32(np.asarray(bits).view(np.uint16)).astype(np.float64)
