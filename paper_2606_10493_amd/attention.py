"""The attention half of a decoder layer through the C ABI: the binding of the
rotary, cache and attention calls, and one layer's steps put together.

``KVCache`` holds a layer's paged cache; ``AttentionBuffers`` the outputs and
workspaces of one shape of call; ``run_attention`` enqueues a layer's
attention for new tokens: rotate and write the cache, then attend (prompts
over their own keys, single tokens over the cache).  Nothing is computed in
Python.
"""
from __future__ import annotations

import torch

from . import _dev, _stream  # defined before the package imports this module
from ._lib import MoeAttnDims, MoeKvCache, MoeRopeCfg, MOE_ROPE_HALF, MOE_ROPE_PLAIN, check as _check, lib


_BF16 = (torch.bfloat16, torch.int16, torch.uint16)


def _rows(t, heads, dim, name):
    """Address, token stride and tokens of bf16 rows [tokens, heads, dim] whose heads are contiguous."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in _BF16:
        raise ValueError(f"{name} has type {t.dtype}, expected bf16 or its bits")
    shape = t.shape
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"{name} has shape {tuple(shape)}, expected [tokens, {heads}, {dim}]")
    n = shape[0]
    if n == 0:
        return t.data_ptr(), heads * dim, n
    stride, head, one = t.stride()
    if one != 1 or (head != dim and heads != 1):
        raise ValueError(f"{name}: a token's heads must be contiguous")
    # the stride of a single token is arbitrary
    return t.data_ptr(), (stride if n > 1 else heads * dim), n


def _same(n, expected, name):
    if n != expected:
        raise ValueError(f"{name} has {n} entries, expected {expected}")


def _out(t, tokens, heads, dim, name):
    p = _dev(t, 2, name)
    if t.dtype not in _BF16:
        raise ValueError(f"{name} has type {t.dtype}, expected bf16 or its bits")
    if t.shape != (tokens, heads, dim):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(tokens, heads, dim)}")
    return p


def _ints(t, name):
    """Address and entries of a contiguous int32 vector."""
    return _dev(t, 4, name), t.numel()


class KVCache:
    """A layer's paged key/value cache: e4m3 codes [n_pages, kv_heads, page_size, head_dim] (uint8) and
    fp32 scales [n_pages, kv_heads, page_size] of keys and values."""

    def __init__(self, k, v, k_scale, v_scale):
        if k.dim() != 4 or v.shape != k.shape or k_scale.shape != k.shape[:3] or v_scale.shape != k.shape[:3]:
            raise ValueError("KVCache: codes are [n_pages, kv_heads, page_size, head_dim], scales [n_pages, kv_heads, "
                             "page_size]")
        self.k, self.v, self.k_scale, self.v_scale = k, v, k_scale, v_scale
        self.kv_heads, self.page_size, self.head_dim = k.shape[1:]
        self.n_pages = k.shape[0]
        self.c = MoeKvCache(_dev(k, 1, "k"), _dev(v, 1, "v"), _dev(k_scale, 4, "k_scale"), _dev(v_scale, 4, "v_scale"),
                            k.shape[0], k.shape[2])

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
        return self.c


def moe_rope_table(table, base: float = 10000.0, scaling: int = MOE_ROPE_PLAIN, factor: float = 1.0,
                   original_len: float = 1.0, slow_turns: float = 1.0, fast_turns: float = 32.0, magnitude: float = 1.0,
                   stream=None):
    """Fills table fp32 [n_pos, rot_dim]: cosines, then sines of every position (see include/moe.h)."""
    n_pos, rot = table.shape
    cfg = MoeRopeCfg(rot, scaling, base, factor, original_len, slow_turns, fast_turns, magnitude)
    _check(lib.moe_rope_table(cfg, n_pos, _dev(table, 4, "table"), _stream(stream)))


def moe_rope(dims: MoeAttnDims, q, k, positions, table, layout, q_out, k_out, dev_status=None, stream=None):
    """bf16 q [T, q_heads, head_dim] and k [T, kv_heads, head_dim] rotated into q_out and k_out (q or k None: left out)."""
    pos, T = _ints(positions, "positions")
    hq, hkv, d = dims.q_heads, dims.kv_heads, dims.head_dim
    pq = sq = pk = sk = po = ko = 0
    if q is not None:
        (pq, sq, n), po = _rows(q, hq, d, "q"), _out(q_out, T, hq, d, "q_out")
        _same(n, T, "q")
    if k is not None:
        (pk, sk, n), ko = _rows(k, hkv, d, "k"), _out(k_out, T, hkv, d, "k_out")
        _same(n, T, "k")
    n_pos, rot = table.shape
    _check(lib.moe_rope(dims, T, pq, sq, pk, sk, pos, _dev(table, 4, "table"), n_pos, rot, layout, po, ko,
                        _dev(dev_status, 4, "dev_status"), _stream(stream)))


def moe_rope_cache(dims: MoeAttnDims, q, k, v, positions, table, layout, slots, cache: KVCache, q_out, k_out=None,
                   dev_status=None, stream=None):
    """moe_rope, and the rotated keys and the values quantized into the cache at each token's slot."""
    hq, hkv, d = dims.q_heads, dims.kv_heads, dims.head_dim
    pos, T = _ints(positions, "positions")
    slot, n = _ints(slots, "slots")
    (pq, sq, nq), (pk, sk, nk), (pv, sv, nv) = _rows(q, hq, d, "q"), _rows(k, hkv, d, "k"), _rows(v, hkv, d, "v")
    if not nq == nk == nv == n == T:
        raise ValueError("q, k, v, slots and positions must have one entry per token")
    n_pos, rot = table.shape
    _check(lib.moe_rope_cache(dims, T, pq, sq, pk, sk, pv, sv, pos, _dev(table, 4, "table"), n_pos, rot, layout, slot,
                              cache.check(dims), _out(q_out, T, hq, d, "q_out"),
                              0 if k_out is None else _out(k_out, T, hkv, d, "k_out"),
                              _dev(dev_status, 4, "dev_status"), _stream(stream)))


def moe_cache_read(dims: MoeAttnDims, cache: KVCache, page_table, cu, k_out, v_out, dev_status=None, stream=None):
    """Sequences' first tokens (page_table int32 [B, width], cu int32 [B + 1]) as packed bf16 rows of k_out, v_out."""
    B, width = page_table.shape
    offsets, n = _ints(cu, "cu")
    _same(n, B + 1, "cu")
    T = k_out.shape[0]
    hkv, d = dims.kv_heads, dims.head_dim
    _check(lib.moe_cache_read(dims, cache.check(dims), _dev(page_table, 4, "page_table"), B, width, offsets, T,
                              _out(k_out, T, hkv, d, "k_out"), _out(v_out, T, hkv, d, "v_out"),
                              _dev(dev_status, 4, "dev_status"), _stream(stream)))


def moe_attn_prefill_workspace(dims: MoeAttnDims, B: int, T_q: int, max_k: int) -> int:
    return int(lib.moe_attn_prefill_workspace(dims, B, T_q, max_k))


def moe_attn_prefill(dims: MoeAttnDims, q, k, v, cu_q, cu_k, max_k: int, scale: float, out, ws=None, causal: bool = True,
                     dev_status=None, stream=None):
    """Attention over packed prompts: q [T_q, q_heads, head_dim] over k, v [T_k, kv_heads, head_dim] -> out bf16."""
    hq, hkv, d = dims.q_heads, dims.kv_heads, dims.head_dim
    (pq, sq, T), (pk, sk, nk), (pv, sv, nv) = _rows(q, hq, d, "q"), _rows(k, hkv, d, "k"), _rows(v, hkv, d, "v")
    _same(nv, nk, "v")
    (pcq, n), (pck, m) = _ints(cu_q, "cu_q"), _ints(cu_k, "cu_k")
    _same(m, n, "cu_k")
    _check(lib.moe_attn_prefill(dims, n - 1, T, nk, max_k, pq, sq, pk, sk, pv, sv, pcq, pck, scale, 1 if causal else 0,
                                _out(out, T, hq, d, "out"), _dev(dev_status, 4, "dev_status"), _dev(ws, 1, "ws"),
                                0 if ws is None else ws.numel(), _stream(stream)))


def moe_attn_decode_workspace(dims: MoeAttnDims, B: int, max_len: int, prefix_len: int = 0) -> int:
    return int(lib.moe_attn_decode_workspace(dims, B, max_len, prefix_len))


def moe_attn_decode(dims: MoeAttnDims, q, cache: KVCache, page_table, lens, max_len: int, scale: float, out, ws=None,
                    prefix_pages=None, prefix_len: int = 0, dev_status=None, stream=None):
    """Attention of one token per sequence, q [B, q_heads, head_dim], over the prefix's and its own cached keys."""
    B, width = page_table.shape
    hq, d = dims.q_heads, dims.head_dim
    pq, sq, nq = _rows(q, hq, d, "q")
    plens, n = _ints(lens, "lens")
    if not nq == n == B:
        raise ValueError("q, lens and page_table must have one entry per sequence")
    if prefix_len > 0 and (prefix_pages is None or prefix_pages.numel() * cache.page_size < prefix_len):
        raise ValueError(f"prefix_pages must hold the pages of {prefix_len} tokens")
    _check(lib.moe_attn_decode(dims, B, pq, sq, cache.check(dims), _dev(page_table, 4, "page_table"), width, plens,
                               max_len, _dev(prefix_pages, 4, "prefix_pages"), prefix_len, scale,
                               _out(out, B, hq, d, "out"), _dev(dev_status, 4, "dev_status"), _dev(ws, 1, "ws"),
                               0 if ws is None else ws.numel(), _stream(stream)))


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
