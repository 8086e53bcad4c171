"""The norm between the layer's halves, and the calls with 4-bit weights.

``moe_add_norm`` adds the residual and normalises; ``moe_quant_weight_w4`` and
``moe_pack_weight_w4`` bring weights into the packed form that
``moe_linear_w4`` (projections), ``moe_expert_ffn_w4`` and
``moe_ffn_layer_w4`` (routed experts) read.  As with the attention calls, those of
a layer step check their tensors and call the library in one native function
each (csrc/binding.cpp).  Nothing is computed in Python.
"""
from __future__ import annotations

from . import _dev, _stream  # defined before the package imports this module
from ._lib import MoeDims, MOE_W4_GROUP, check as _check, lib
from .attention import _binding


def moe_add_norm(x, weight, out=None, q=None, s=None, residual=None, sum_out=None, eps: float = 1e-6,
                 weight_offset: float = 0.0, stream=None):
    """x (+ residual), bf16 or fp32 [T, H] or, each head by itself, [T, heads, H] -> its root-mean-square norm times weight
    (bf16 [H] or None) in out (bf16, x's shape), in q (e4m3 codes) and s (fp32, one per 128 values), or in both; the sum
    itself in sum_out, which has the residual's type and may be the residual."""
    _check(_binding.add_norm(x, weight, out, q, s, residual, sum_out, eps, weight_offset, stream))


def _matrices(t, name):
    if t.dim() not in (2, 3):
        raise ValueError(f"{name} must be [rows, cols] or [n_mats, rows, cols]")
    return t.shape if t.dim() == 3 else (1, *t.shape)


def _on_stream(stream, **tensors):
    import torch
    device = getattr(stream, "device_index", None)  # an object that has a handle alone is of the current device
    if device is None:
        device = torch.cuda.current_device()
    for name, t in tensors.items():
        if t is not None and t.device.index != device:
            raise ValueError(f"{name} is on another device than the call's stream")


def moe_quant_weight_w4(w, q, s, stream=None):
    """w fp32 [n_mats, rows, cols] (or [rows, cols]) -> q uint8 [.., rows, cols / 2] (two e2m1 codes a byte), s uint8
    [.., rows, cols / 32] (powers of two)."""
    import torch
    pw, pq, ps = _dev(w, 4, "w"), _dev(q, 1, "q"), _dev(s, 1, "s")
    if w.dtype != torch.float32:
        raise ValueError("w must be fp32")
    n, rows, cols = _matrices(w, "w")
    if q.numel() * 2 != w.numel() or s.numel() != n * rows * (cols // MOE_W4_GROUP):
        raise ValueError("q must have half a byte and s a byte per 32 columns for every weight")
    _on_stream(stream, w=w, q=q, s=s)
    _check(lib.moe_quant_weight_w4(pw, n, rows, cols, pq, ps, _stream(stream)))


def moe_w4_scale_bytes(n_mats: int, rows: int, cols: int) -> int:
    """Bytes of the packed scales of n_mats [rows, cols] matrices (0 for shapes that moe_pack_weight_w4 refuses)."""
    return int(lib.moe_w4_scale_bytes(n_mats, rows, cols))


def moe_pack_weight_w4(q, s, packed, packed_s, dev_status=None, stream=None):
    """q uint8 [n_mats, rows, cols / 2] (or [rows, cols / 2]), s uint8 [.., rows, cols / 32], row-major -> packed (as many
    bytes as q) and packed_s (moe_w4_scale_bytes of them)."""
    args = _dev(q, 1, "q"), _dev(s, 1, "s")
    out = _dev(packed, 1, "packed"), _dev(packed_s, 1, "packed_s"), _dev(dev_status, 4, "dev_status")
    n, rows, half = _matrices(q, "q")
    cols = 2 * half
    need = moe_w4_scale_bytes(n, rows, cols)
    if s.numel() * MOE_W4_GROUP != n * rows * cols or packed.numel() != q.numel() or (need and packed_s.numel() != need):
        raise ValueError("s must have a byte per 32 columns, packed as many bytes as q, packed_s moe_w4_scale_bytes")
    _on_stream(stream, q=q, s=s, packed=packed, packed_s=packed_s, dev_status=dev_status)
    _check(lib.moe_pack_weight_w4(*args, n, rows, cols, *out, _stream(stream)))


def moe_linear_w4_workspace(T: int, K: int, N: int) -> int:
    return int(lib.moe_linear_w4_workspace(T, K, N))


def moe_linear_w4(x, w, w_s, out, bias=None, ws=None, stream=None):
    """x bf16 [T, K] times the packed [N, K] matrix (w, w_s) -> out bf16 or fp32 [T, N]; bias bf16 [N]."""
    _check(_binding.linear_w4(x, w, w_s, out, bias, ws, stream))


def moe_expert_ffn_w4_workspace(dims: MoeDims, T: int) -> int:
    return int(lib.moe_expert_ffn_w4_workspace(dims, T))


def moe_expert_ffn_w4(dims: MoeDims, T: int, x_bf16, expert_offsets, sorted_src, w_gate, s_gate, w_up, s_up, w_down, s_down,
                      y_rows, ws, stream=None):
    """Expert FFN over the expert-sorted rows, bf16 activations and packed 4-bit weights."""
    _check(_binding.expert_ffn_w4(dims, T, x_bf16, expert_offsets, sorted_src, w_gate, s_gate, w_up, s_up, w_down, s_down,
                                  y_rows, ws, stream))


def moe_ffn_layer_w4_workspace(dims: MoeDims, T: int) -> int:
    return int(lib.moe_ffn_layer_w4_workspace(dims, T))


def moe_ffn_layer_w4(dims: MoeDims, T: int, x_bf16, topk_ids, topk_w, w_gate, s_gate, w_up, s_up, w_down, s_down, out_bf16,
                     dev_status, ws, stream=None):
    """The whole layer with packed 4-bit weights in one library call (see include/moe.h)."""
    _check(_binding.ffn_layer_w4(dims, T, x_bf16, topk_ids, topk_w, w_gate, s_gate, w_up, s_up, w_down, s_down, out_bf16,
                                 dev_status, ws, stream))
