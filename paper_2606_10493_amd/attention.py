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

from ._lib import MoeAttnDims, MoeKvCache, MoeRopeCfg, MOE_ROPE_HALF, MOE_ROPE_PLAIN, check as _check, lib


def _stream(stream):
    from . import _stream as current
    return current(stream)


def _dev(t, dtype_bytes, name):
    from . import _dev as address
    return address(t, dtype_bytes, name)


def _rows(t, heads, dim, name):
    """Address and token stride of bf16 rows [tokens, heads, dim] whose heads are contiguous."""
    if not t.is_cuda:
        raise ValueError(f"{name} must be a device tensor")
    if t.dtype not in _BF16:
        raise ValueError(f"{name} has type {t.dtype}, expected bf16 or its bits")
    shape, stride = t.shape, t.stride()
    if len(shape) != 3 or shape[1] != heads or shape[2] != dim:
        raise ValueError(f"{name} has shape {tuple(shape)}, expected [tokens, {heads}, {dim}]")
    if shape[0] == 0:
        return t.data_ptr(), heads * dim
    if stride[2] != 1 or (stride[1] != dim and heads != 1):
        raise ValueError(f"{name}: a token's heads must be contiguous")
    # the stride of a single token is arbitrary
    return t.data_ptr(), (stride[0] if shape[0] > 1 else heads * dim)


def _same(t, n, name):
    if t.shape[0] != n:
        raise ValueError(f"{name} has {t.shape[0]} entries, expected {n}")


_BF16 = (torch.bfloat16, torch.int16, torch.uint16)


def _out(t, tokens, heads, dim, name):
    p = _dev(t, 2, name)
    if t.dtype not in _BF16:
        raise ValueError(f"{name} has type {t.dtype}, expected bf16 or its bits")
    if tuple(t.shape) != (tokens, heads, dim):
        raise ValueError(f"{name} has shape {tuple(t.shape)}, expected {(tokens, heads, dim)}")
    return p


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
    T = positions.shape[0]
    pq = sq = pk = sk = po = ko = 0
    if q is not None:
        (pq, sq), po = _rows(q, dims.q_heads, dims.head_dim, "q"), _out(q_out, T, dims.q_heads, dims.head_dim, "q_out")
        _same(q, T, "q")
    if k is not None:
        (pk, sk), ko = _rows(k, dims.kv_heads, dims.head_dim, "k"), _out(k_out, T, dims.kv_heads, dims.head_dim, "k_out")
        _same(k, T, "k")
    _check(lib.moe_rope(dims, T, pq, sq, pk, sk, _dev(positions, 4, "positions"), _dev(table, 4, "table"),
                        table.shape[0], table.shape[1], layout, po, ko, _dev(dev_status, 4, "dev_status"),
                        _stream(stream)))


def moe_rope_cache(dims: MoeAttnDims, q, k, v, positions, table, layout, slots, cache: KVCache, q_out, k_out=None,
                   dev_status=None, stream=None):
    """moe_rope, and the rotated keys and the values quantized into the cache at each token's slot."""
    T, hq, hkv, d = positions.shape[0], dims.q_heads, dims.kv_heads, dims.head_dim
    (pq, sq), (pk, sk), (pv, sv) = _rows(q, hq, d, "q"), _rows(k, hkv, d, "k"), _rows(v, hkv, d, "v")
    if not q.shape[0] == k.shape[0] == v.shape[0] == slots.shape[0] == T:
        raise ValueError("q, k, v, slots and positions must have one entry per token")
    po = _out(q_out, T, hq, d, "q_out")
    ko = 0 if k_out is None else _out(k_out, T, hkv, d, "k_out")
    _check(lib.moe_rope_cache(dims, T, pq, sq, pk, sk, pv, sv, _dev(positions, 4, "positions"),
                              _dev(table, 4, "table"), table.shape[0], table.shape[1], layout, _dev(slots, 4, "slots"),
                              cache.check(dims), po, ko, _dev(dev_status, 4, "dev_status"), _stream(stream)))


def moe_cache_read(dims: MoeAttnDims, cache: KVCache, page_table, cu, k_out, v_out, dev_status=None, stream=None):
    """Sequences' first tokens (page_table int32 [B, width], cu int32 [B + 1]) as packed bf16 rows of k_out, v_out."""
    B, width = page_table.shape
    _same(cu, B + 1, "cu")
    T = k_out.shape[0]
    pk = _out(k_out, T, dims.kv_heads, dims.head_dim, "k_out")
    pv = _out(v_out, T, dims.kv_heads, dims.head_dim, "v_out")
    _check(lib.moe_cache_read(dims, cache.check(dims), _dev(page_table, 4, "page_table"), B, width, _dev(cu, 4, "cu"), T,
                              pk, pv, _dev(dev_status, 4, "dev_status"), _stream(stream)))


def moe_attn_prefill_workspace(dims: MoeAttnDims, B: int, T_q: int, max_k: int) -> int:
    return int(lib.moe_attn_prefill_workspace(dims, B, T_q, max_k))


def moe_attn_prefill(dims: MoeAttnDims, q, k, v, cu_q, cu_k, max_k: int, scale: float, out, ws=None, causal: bool = True,
                     dev_status=None, stream=None):
    """Attention over packed prompts: q [T_q, q_heads, head_dim] over k, v [T_k, kv_heads, head_dim] -> out bf16."""
    hq, hkv, d = dims.q_heads, dims.kv_heads, dims.head_dim
    (pq, sq), (pk, sk), (pv, sv) = _rows(q, hq, d, "q"), _rows(k, hkv, d, "k"), _rows(v, hkv, d, "v")
    _same(v, k.shape[0], "v")
    _same(cu_k, cu_q.shape[0], "cu_k")
    T = q.shape[0]
    _check(lib.moe_attn_prefill(dims, cu_q.shape[0] - 1, T, k.shape[0], max_k, pq, sq, pk, sk, pv, sv,
                                _dev(cu_q, 4, "cu_q"), _dev(cu_k, 4, "cu_k"), scale, 1 if causal else 0,
                                _out(out, T, hq, d, "out"), _dev(dev_status, 4, "dev_status"), _dev(ws, 1, "ws"),
                                0 if ws is None else ws.numel(), _stream(stream)))


def moe_attn_decode_workspace(dims: MoeAttnDims, B: int, max_len: int, prefix_len: int = 0) -> int:
    return int(lib.moe_attn_decode_workspace(dims, B, max_len, prefix_len))


def moe_attn_decode(dims: MoeAttnDims, q, cache: KVCache, page_table, lens, max_len: int, scale: float, out, ws=None,
                    prefix_pages=None, prefix_len: int = 0, dev_status=None, stream=None):
    """Attention of one token per sequence, q [B, q_heads, head_dim], over the prefix's and its own cached keys."""
    B, width = page_table.shape
    pq, sq = _rows(q, dims.q_heads, dims.head_dim, "q")
    _same(q, B, "q")
    _same(lens, B, "lens")
    if prefix_len > 0 and (prefix_pages is None or prefix_pages.numel() * cache.page_size < prefix_len):
        raise ValueError(f"prefix_pages must hold the pages of {prefix_len} tokens")
    _check(lib.moe_attn_decode(dims, B, pq, sq, cache.check(dims), _dev(page_table, 4, "page_table"), width,
                               _dev(lens, 4, "lens"), max_len, _dev(prefix_pages, 4, "prefix_pages"), prefix_len, scale,
                               _out(out, B, dims.q_heads, dims.head_dim, "out"), _dev(dev_status, 4, "dev_status"),
                               _dev(ws, 1, "ws"), 0 if ws is None else ws.numel(), _stream(stream)))


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
