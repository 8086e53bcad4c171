"""Refusals of the rotary, cache and attention calls, through the C ABI and the binding (CPU; nothing is launched)."""
import ctypes

import pytest
import torch

import paper_2606_10493_amd as moe

P = ctypes.c_void_p
A, ODD = P(0x10000), P(0x10008)     # stand-ins for device addresses, never followed
INVALID, SHAPE, WORKSPACE = moe.MOE_ERR_INVALID_ARG, moe.MOE_ERR_UNSUPPORTED_SHAPE, moe.MOE_ERR_WORKSPACE
D = moe.MoeAttnDims(8, 2, 128)


def cache(k=0x10000, v=0x20000, ks=0x30000, vs=0x40000, pages=4, size=64):
    return moe.MoeKvCache(k, v, ks, vs, pages, size)


BAD_DIMS = [(moe.MoeAttnDims(0, 1, 64), INVALID), (moe.MoeAttnDims(4, 0, 64), INVALID), (moe.MoeAttnDims(4, -2, 64), INVALID),
            (moe.MoeAttnDims(4, 4, 0), INVALID), (moe.MoeAttnDims(5, 2, 64), SHAPE), (moe.MoeAttnDims(2, 4, 64), SHAPE),
            (moe.MoeAttnDims(4, 4, 96), SHAPE), (moe.MoeAttnDims(4, 4, 256), SHAPE), (moe.MoeAttnDims(2048, 8, 64), SHAPE)]
BAD_CACHES = [cache(k=0), cache(v=0), cache(ks=0), cache(vs=0), cache(k=0x10008), cache(vs=0x40004), cache(pages=0),
              cache(size=8), cache(size=48), cache(size=2048), cache(size=0), cache(size=-64)]


def rope(d=D, T=4, q=A, qs=1024, k=A, ks=256, pos=A, table=A, n_pos=10, rot=128, layout=0, qo=P(0x90000), ko=P(0xa0000)):
    return moe.lib.moe_rope(d, T, q, qs, k, ks, pos, table, n_pos, rot, layout, qo, ko, None, None)


def rope_cache(d=D, T=4, q=A, qs=1024, k=A, ks=256, v=A, vs=256, pos=A, table=A, n_pos=10, rot=128, layout=0, slots=A,
               c=None, qo=P(0x90000), ko=None):
    return moe.lib.moe_rope_cache(d, T, q, qs, k, ks, v, vs, pos, table, n_pos, rot, layout, slots,
                                  cache() if c is None else c, qo, ko, None, None)


def read(d=D, c=None, table=A, B=2, width=3, cu=A, T=9, k=A, v=A):
    return moe.lib.moe_cache_read(d, cache() if c is None else c, table, B, width, cu, T, k, v, None, None)


def prefill(d=D, B=2, Tq=9, Tk=9, max_k=9, q=A, qs=1024, k=A, ks=256, v=A, vs=256, cq=A, ck=A, scale=0.1, out=A, ws=None,
            n=0):
    return moe.lib.moe_attn_prefill(d, B, Tq, Tk, max_k, q, qs, k, ks, v, vs, cq, ck, scale, 1, out, None, ws, n, None)


def decode(d=D, B=2, q=A, qs=1024, c=None, table=A, width=3, lens=A, max_len=9, pages=None, prefix=0, scale=0.1, out=A,
           ws=None, n=0):
    return moe.lib.moe_attn_decode(d, B, q, qs, cache() if c is None else c, table, width, lens, max_len, pages, prefix,
                                   scale, out, None, ws, n, None)


@pytest.mark.parametrize("call", [rope, rope_cache, read, prefill, decode])
@pytest.mark.parametrize("dims,status", BAD_DIMS)
def test_dims(call, dims, status):
    assert call(d=dims) == status
    assert moe.moe_last_error().startswith("moe_")


@pytest.mark.parametrize("call", [rope_cache, read, decode])
@pytest.mark.parametrize("bad", BAD_CACHES)
def test_caches(call, bad):
    assert call(c=bad) == INVALID


def test_rope_refusals():
    for call in (rope, rope_cache):
        for bad in (dict(T=-1), dict(n_pos=0), dict(layout=2), dict(pos=None), dict(table=None), dict(table=ODD),
                    dict(qs=1016), dict(qs=1028), dict(qs=1 << 23), dict(ks=-256), dict(q=ODD), dict(k=ODD), dict(qo=ODD),
                    dict(ko=ODD), dict(qo=None), dict(qo=A, q=A, qs=2048)):
            assert call(**bad) == INVALID, bad
        for rot in (0, 8, 24, 144, -16):
            assert call(rot=rot) == SHAPE
        assert call(T=0) == moe.MOE_OK
    assert rope(q=None) == rope(ko=None) == rope(q=None, qo=None, k=None, ko=None) == INVALID
    assert rope_cache(q=None) == rope_cache(v=None) == rope_cache(slots=None) == rope_cache(v=ODD) == INVALID


def test_rope_table_refusals():
    def call(rot=64, scaling=0, base=1e4, factor=1.0, orig=1.0, slow=1.0, fast=32.0, mag=1.0, n=8, table=A):
        return moe.lib.moe_rope_table(moe.MoeRopeCfg(rot, scaling, base, factor, orig, slow, fast, mag), n, table, None)
    for rot in (0, 8, 24, 144):
        assert call(rot=rot) == SHAPE
    assert call(n=(1 << 22) + 1) == SHAPE
    inf, nan = float("inf"), float("nan")
    for bad in (dict(scaling=3), dict(scaling=-1), dict(base=1.0), dict(base=nan), dict(base=inf), dict(mag=nan), dict(n=-1),
                dict(table=None), dict(table=ODD), dict(scaling=1, factor=0.0), dict(scaling=1, factor=nan),
                dict(scaling=2, orig=0.0), dict(scaling=2, slow=-1.0), dict(scaling=2, slow=32.0), dict(scaling=2, fast=inf)):
        assert call(**bad) == INVALID, bad
    assert call(n=0, table=None) == moe.MOE_OK


def test_cache_read_refusals():
    for bad in (dict(B=-1), dict(T=-1), dict(width=-1), dict(table=None), dict(cu=None), dict(k=None), dict(v=None),
                dict(k=ODD), dict(v=ODD)):
        assert read(**bad) == INVALID, bad
    assert read(T=(1 << 26) + 1) == SHAPE
    assert read(B=0) == read(T=0) == moe.MOE_OK


def test_prefill_refusals():
    nan = float("nan")
    for bad in (dict(B=-1), dict(Tq=-1), dict(Tk=-1), dict(max_k=-1), dict(q=None), dict(k=None), dict(v=None), dict(cq=None),
                dict(ck=None), dict(out=None), dict(out=ODD), dict(q=ODD), dict(v=ODD), dict(qs=1000), dict(ks=1 << 23),
                dict(scale=0.0), dict(scale=-0.1), dict(scale=nan), dict(scale=float("inf"))):
        assert prefill(**bad) == INVALID, bad
    assert prefill(Tk=(1 << 30) + 1) == SHAPE
    assert prefill(Tq=1 << 30) == SHAPE
    assert prefill(B=0) == prefill(Tq=0) == moe.MOE_OK
    need = moe.moe_attn_prefill_workspace(D, 1, 509, 8701)
    assert need > 0
    args = dict(B=1, Tq=509, Tk=8701, max_k=8701)
    assert prefill(**args) == prefill(**args, ws=A, n=need - 1) == prefill(**args, ws=ODD, n=need) == WORKSPACE


def test_decode_refusals():
    for bad in (dict(B=-1), dict(B=65536), dict(width=-1), dict(max_len=-1), dict(max_len=(1 << 30) + 1), dict(prefix=-1),
                dict(prefix=(1 << 30) + 1, pages=A), dict(prefix=5), dict(q=None), dict(q=ODD), dict(qs=1000),
                dict(table=None), dict(lens=None), dict(out=None), dict(out=ODD), dict(scale=0.0),
                dict(scale=float("nan"))):
        assert decode(**bad) == INVALID, bad
    assert decode(B=0) == moe.MOE_OK
    assert decode(B=65535, width=1 << 24, c=cache(size=1024)) == SHAPE   # over 2^31 steps
    need = moe.moe_attn_decode_workspace(D, 2, 9000, 0)
    assert need > 0
    assert decode(max_len=9000) == decode(max_len=9000, ws=A, n=need - 1) == decode(max_len=9000, ws=ODD, n=need) == WORKSPACE


def test_workspace_queries():
    """Zero for what the calls refuse; no trouble at the ends of the ranges; a larger call never needs less."""
    big = 2 ** 31 - 1
    for d, _ in BAD_DIMS:
        assert moe.moe_attn_prefill_workspace(d, 1, 1, 1) == moe.moe_attn_decode_workspace(d, 1, 9000, 9000) == 0
    for B in (-1, 0, 65536):
        assert moe.moe_attn_decode_workspace(D, B, 9000) == 0
    assert moe.moe_attn_decode_workspace(D, 1, big) == moe.moe_attn_decode_workspace(D, 1, 1, big) == 0
    assert moe.moe_attn_decode_workspace(moe.MoeAttnDims(1024, 1, 128), 65535, 1 << 30, 1 << 30) > 0
    for args in ((1, big, big), (big, big, big), (1, 1, big)):
        assert moe.moe_attn_prefill_workspace(moe.MoeAttnDims(1024, 1, 128), *args) >= 0
    sizes = [moe.moe_attn_decode_workspace(D, b, 9000, 500) for b in (1, 2, 30, 64, 1000)]
    assert sizes == sorted(sizes)


def test_binding_refusals():
    cpu = torch.zeros((4, 8, 128), dtype=torch.bfloat16)
    with pytest.raises(ValueError, match="device tensor"):
        moe.moe_rope(D, cpu, None, torch.zeros(4, dtype=torch.int32), torch.zeros(9, 128), 0, cpu, None)
    with pytest.raises(ValueError, match="device tensor"):
        moe.KVCache(*(torch.zeros((2, 2, 16, 128), dtype=torch.uint8) for _ in "kv"),
                    *(torch.zeros((2, 2, 16)) for _ in "kv"))
    with pytest.raises(ValueError, match="codes are"):
        moe.KVCache(*(torch.zeros((2, 2, 16, 128), dtype=torch.uint8) for _ in "kv"),
                    *(torch.zeros((2, 2, 8)) for _ in "kv"))
