"""The attention half of a decoder layer through the C ABI: the binding of the
rotary, cache and attention calls, and one layer's steps put together.  The
calls check their tensors and call the library in one native function each
(csrc/binding.cpp), since a decode step is bound by the host.

``KVCache`` holds a layer's paged cache; ``AttentionBuffers`` the outputs and
workspaces of one shape of call; ``run_attention`` enqueues a layer's
attention for new tokens: rotate and write the cache, then attend (prompts
over their own keys, single tokens over the cache).  Nothing is computed in
Python.
"""
from __future__ import annotations

import ctypes
import importlib

import torch

from . import _dev, _stream  # defined before the package imports this module
from ._lib import MoeAttnDims, MoeKvCache, MoeRopeCfg, MOE_ROPE_HALF, MOE_ROPE_PLAIN, check as _check, lib


class _NoBinding:
    """Stands for a binding that is not there: the rest of the package works, every call that needs it says why it does not."""

    def __init__(self, why: str):
        self.why = why

    def __getattr__(self, name):
        raise ImportError(f"_binding.so, which the attention calls, the norm and the calls with 4-bit weights need, cannot be "
                          f"loaded ({self.why}); build it with `python paper_2606_10493_amd/build.py`")


try:
    _binding = importlib.import_module("._binding", __package__)  # links libmoe.so, which is loaded by now
except ImportError as e:
    _binding = _NoBinding(str(e))


class _DeviceCache(ctypes.Structure):
    """What the binding takes: the C ABI's structure and its tensors' device."""
    _fields_ = [("cache", MoeKvCache), ("device", ctypes.c_int64)]


class KVCache:
    """A layer's paged key/value cache: e4m3 codes [n_pages, kv_heads, page_size, head_dim] (uint8) and
    fp32 scales [n_pages, kv_heads, page_size] of keys and values."""

    def __init__(self, k, v, k_scale, v_scale):
        if k.dim() != 4 or v.shape != k.shape or k_scale.shape != k.shape[:3] or v_scale.shape != k.shape[:3]:
            raise ValueError("KVCache: codes are [n_pages, kv_heads, page_size, head_dim], scales [n_pages, kv_heads, "
                             "page_size]")
        for t, name in ((k, "k"), (v, "v")):
            if t.dtype not in (torch.uint8, torch.int8, torch.float8_e4m3fn):
                raise ValueError(f"{name} must be e4m3 codes (uint8, int8 or float8_e4m3fn)")
        for t, name in ((k_scale, "k_scale"), (v_scale, "v_scale")):
            if t.dtype != torch.float32:
                raise ValueError(f"{name} must be fp32")
        if len({t.device for t in (k, v, k_scale, v_scale)}) != 1:
            raise ValueError("KVCache: the tensors are on different devices")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.kv_heads, self.page_size, self.head_dim = k.shape[1:]
        self.n_pages = k.shape[0]
        c = MoeKvCache(_dev(k, 1, "k"), _dev(v, 1, "v"), _dev(k_scale, 4, "k_scale"), _dev(v_scale, 4, "v_scale"),
                       k.shape[0], k.shape[2])
        self.on_device = _DeviceCache(c, k.device.index)
        self.c = self.on_device.cache

    @classmethod
    def empty(cls, n_pages: int, kv_heads: int, page_size: int, head_dim: int, device="cuda"):
        def codes():
            return torch.empty((n_pages, kv_heads, page_size, head_dim), dtype=torch.uint8, device=device)

        def scales():
            return torch.empty((n_pages, kv_heads, page_size), dtype=torch.float32, device=device)
        return cls(codes(), codes(), scales(), scales())

    def check(self, dims: MoeAttnDims):
        if self.kv_heads != dims.kv_heads or self.head_dim != dims.head_dim:
            raise ValueError(f"the cache has {self.kv_heads} heads of {self.head_dim}, the call {dims.kv_heads} of "
                             f"{dims.head_dim}")
        return self.on_device


def moe_rope_table(table, base: float = 10000.0, scaling: int = MOE_ROPE_PLAIN, factor: float = 1.0,
                   original_len: float = 1.0, slow_turns: float = 1.0, fast_turns: float = 32.0, magnitude: float = 1.0,
                   stream=None):
    """Fills table fp32 [n_pos, rot_dim]: cosines, then sines of every position (see include/moe.h)."""
    n_pos, rot = table.shape
    if table.dtype != torch.float32:
        raise ValueError("table must be fp32")
    if table.is_cuda and table.device.index != (torch.cuda.current_device() if stream is None else stream.device_index):
        raise ValueError("table is on another device than the call's stream")
    cfg = MoeRopeCfg(rot, scaling, base, factor, original_len, slow_turns, fast_turns, magnitude)
    _check(lib.moe_rope_table(cfg, n_pos, _dev(table, 4, "table"), _stream(stream)))


def moe_rope(dims: MoeAttnDims, q, k, positions, table, layout, q_out, k_out, dev_status=None, stream=None):
    """bf16 q [T, q_heads, head_dim] and k [T, kv_heads, head_dim] rotated into q_out and k_out (q or k None: left out)."""
    _check(_binding.rope(dims, q, k, positions, table, layout, q_out, k_out, dev_status, stream))


def moe_rope_cache(dims: MoeAttnDims, q, k, v, positions, table, layout, slots, cache: KVCache, q_out, k_out=None,
                   dev_status=None, stream=None):
    """moe_rope, and the rotated keys and the values quantized into the cache at each token's slot."""
    _check(_binding.rope_cache(dims, q, k, v, positions, table, layout, slots, cache.check(dims), q_out, k_out, dev_status,
                               stream))


def moe_cache_read(dims: MoeAttnDims, cache: KVCache, page_table, cu, k_out, v_out, dev_status=None, stream=None):
    """Sequences' first tokens (page_table int32 [B, width], cu int32 [B + 1]) as packed bf16 rows of k_out, v_out."""
    _check(_binding.cache_read(dims, cache.check(dims), page_table, cu, k_out, v_out, dev_status, stream))


def moe_attn_prefill_workspace(dims: MoeAttnDims, B: int, T_q: int, max_k: int) -> int:
    return int(lib.moe_attn_prefill_workspace(dims, B, T_q, max_k))


def moe_attn_prefill(dims: MoeAttnDims, q, k, v, cu_q, cu_k, max_k: int, scale: float, out, ws=None, causal: bool = True,
                     dev_status=None, stream=None):
    """Attention over packed prompts: q [T_q, q_heads, head_dim] over k, v [T_k, kv_heads, head_dim] -> out bf16."""
    _check(_binding.attn_prefill(dims, q, k, v, cu_q, cu_k, max_k, scale, out, ws, causal, dev_status, stream))


def moe_attn_decode_workspace(dims: MoeAttnDims, B: int, max_len: int, prefix_len: int = 0) -> int:
    return int(lib.moe_attn_decode_workspace(dims, B, max_len, prefix_len))


def moe_attn_decode(dims: MoeAttnDims, q, cache: KVCache, page_table, lens, max_len: int, scale: float, out, ws=None,
                    prefix_pages=None, prefix_len: int = 0, dev_status=None, stream=None):
    """Attention of one token per sequence, q [B, q_heads, head_dim], over the prefix's and its own cached keys."""
    _check(_binding.attn_decode(dims, q, cache.check(dims), page_table, lens, max_len, scale, out, ws, prefix_pages,
                                prefix_len, dev_status, stream))


class AttentionBuffers:
    """Outputs and workspaces of one shape of attention call: `tokens` packed tokens of `batch` prompts with at most
    `longest` keys (prompts), or `batch` single tokens over at most `longest` cached ones behind `prefix_len` shared ones
    (steps: tokens == 0)."""

    def __init__(self, dims: MoeAttnDims, batch: int, longest: int, tokens: int = 0, prefix_len: int = 0, device="cuda"):
        self.dims, self.batch, self.longest, self.prefix_len = dims, batch, longest, prefix_len
        self.prompt = tokens > 0
        n = tokens or batch
        dev = torch.device(device)
        self.dev_status = torch.zeros(1, dtype=torch.int32, device=dev)
        self.q = torch.empty((n, dims.q_heads, dims.head_dim), dtype=torch.bfloat16, device=dev)
        self.k = torch.empty((n, dims.kv_heads, dims.head_dim), dtype=torch.bfloat16, device=dev) if self.prompt else None
        self.out = torch.empty_like(self.q)
        need = (moe_attn_prefill_workspace(dims, batch, n, longest) if self.prompt else
                moe_attn_decode_workspace(dims, batch, longest, prefix_len))
        self.ws = torch.empty(max(need, 256), dtype=torch.uint8, device=dev)


def run_attention(buf: AttentionBuffers, q, k, v, positions, table, slots, cache: KVCache, scale: float, cu=None,
                  page_table=None, lens=None, prefix_pages=None, layout: int = MOE_ROPE_HALF, stream=None):
    """A layer's attention for new tokens: rotate and write the cache, then attend.  Prompts: cu int32 [batch + 1] of the
    packed tokens, which attend to their own prompt.  Steps: page_table and lens, the new tokens counted."""
    moe_rope_cache(buf.dims, q, k, v, positions, table, layout, slots, cache, buf.q, buf.k, buf.dev_status, stream)
    if buf.prompt:
        moe_attn_prefill(buf.dims, buf.q, buf.k, v, cu, cu, buf.longest, scale, buf.out, buf.ws, True, buf.dev_status,
                         stream)
    else:
        moe_attn_decode(buf.dims, buf.q, cache, page_table, lens, buf.longest, scale, buf.out, buf.ws, prefix_pages,
                        buf.prefix_len, buf.dev_status, stream)
    return buf.out
