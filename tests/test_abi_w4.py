"""Refusals of the norm and of the calls with 4-bit weights, through the C ABI and the binding (CPU; nothing is launched)."""
import ctypes
import random

import pytest
import torch

import paper_2606_10493_amd as moe

P = ctypes.c_void_p
A, ODD = P(0x10000), P(0x10008)     # stand-ins for device addresses, never followed
INVALID, SHAPE, WORKSPACE = moe.MOE_ERR_INVALID_ARG, moe.MOE_ERR_UNSUPPORTED_SHAPE, moe.MOE_ERR_WORKSPACE
OK = moe.MOE_OK


def cfg(eps=1e-6, offset=0.0, heads=1, x=moe.MOE_BF16, stream=moe.MOE_BF16):
    return moe.MoeNormCfg(eps, offset, heads, x, stream)


def norm(x=A, xs=256, r=A, rs=256, w=A, T=3, H=256, c=None, sum_=A, ss=256, out=A, os_=256, q=A, s=A):
    return moe.lib.moe_add_norm(x, xs, r, rs, w, T, H, cfg() if c is None else c, sum_, ss, out, os_, q, s, None)


def linear(x=A, xs=256, T=3, K=256, w=A, ws_=A, N=48, bias=A, out=A, os_=48, ot=moe.MOE_BF16, ws=A, n=1 << 40):
    return moe.lib.moe_linear_w4(x, xs, T, K, w, ws_, N, bias, out, os_, ot, ws, n, None)


D = moe.MoeDims(256, 128, 8, 2)


def ffn(d=D, T=3, x=A, off=A, src=A, w=A, s=A, y=A, ws=A, n=1 << 40):
    return moe.lib.moe_expert_ffn_w4(d, T, x, off, src, w, s, w, s, w, s, y, ws, n, None)


def layer(d=D, T=3, x=A, ids=A, p=A, w=A, s=A, out=A, ws=A, n=1 << 40):
    return moe.lib.moe_ffn_layer_w4(d, T, x, ids, p, w, s, w, s, w, s, out, None, ws, n, None)


def test_norm_refusals():
    for bad in (dict(T=-1), dict(H=0), dict(H=-8), dict(c=cfg(heads=0)), dict(c=cfg(x=2)), dict(c=cfg(stream=-1)),
                dict(c=cfg(eps=0.0)), dict(c=cfg(eps=-1.0)), dict(c=cfg(eps=1e-13)), dict(c=cfg(eps=float("nan"))),
                dict(c=cfg(eps=float("inf"))), dict(c=cfg(offset=float("inf"))), dict(q=None), dict(s=None),
                dict(out=None, q=None, s=None), dict(x=None), dict(x=ODD), dict(r=ODD), dict(sum_=ODD), dict(out=ODD),
                dict(w=ODD), dict(q=P(0x10004)), dict(s=P(0x10002)), dict(xs=248), dict(xs=260), dict(rs=0), dict(ss=-256),
                dict(os_=255), dict(c=cfg(heads=2))):
        assert norm(**bad) == INVALID, bad
        assert "moe_add_norm" in moe.moe_last_error()
    for bad in (dict(H=4), dict(H=132), dict(H=64), dict(H=32776, q=None, s=None), dict(H=32768 + 128),
                dict(T=1 << 30, c=cfg(heads=4))):
        assert norm(**bad) == SHAPE, bad
    assert norm(T=0) == OK and norm(T=0, x=None) == OK


def test_weights_refusals():
    quant, pack = moe.lib.moe_quant_weight_w4, moe.lib.moe_pack_weight_w4
    for bad in ((A, -1, 16, 32, A, A), (A, 1, 0, 32, A, A), (A, 1, 16, 0, A, A), (None, 1, 16, 32, A, A),
                (A, 1, 16, 32, None, A), (A, 1, 16, 32, A, None), (ODD, 1, 16, 32, A, A), (A, 1, 16, 32, ODD, A)):
        assert quant(*bad, None) == INVALID, bad
    assert quant(A, 1, 16, 48, A, A, None) == SHAPE and quant(A, 0, 16, 32, A, A, None) == OK
    assert quant(A, 2 ** 31 - 1, 2 ** 31 - 1, 2 ** 31 - 32, A, A, None) == SHAPE
    for bad in ((A, A, -1, 16, 128, A, A), (A, A, 1, 0, 128, A, A), (A, A, 1, 16, -128, A, A), (None, A, 1, 16, 128, A, A),
                (A, None, 1, 16, 128, A, A), (A, A, 1, 16, 128, None, A), (A, A, 1, 16, 128, A, None),
                (ODD, A, 1, 16, 128, A, A), (A, P(0x10002), 1, 16, 128, A, A), (A, A, 1, 16, 128, ODD, A),
                (A, A, 1, 16, 128, A, ODD)):
        assert pack(*bad, None, None) == INVALID, bad
    assert pack(A, A, 1, 24, 128, A, A, None, None) == SHAPE and pack(A, A, 1, 16, 160, A, A, None, None) == SHAPE
    assert pack(A, A, 0, 16, 128, A, A, None, None) == OK


def test_scale_bytes():
    size = moe.moe_w4_scale_bytes
    assert size(1, 16, 128) == 256 and size(1, 16, 512) == 256 and size(1, 16, 640) == 512 and size(3, 48, 1024) == 9 * 512
    assert size(256, 7168, 2048) == 256 * 448 * 4 * 256
    assert size(0, 16, 128) == 0 and size(1, 8, 128) == 0 and size(1, 16, 96) == 0 and size(-1, 16, 128) == 0


def test_linear_refusals():
    for bad in (dict(T=-1), dict(K=0), dict(N=0), dict(N=-16), dict(ot=2), dict(x=None), dict(w=None), dict(ws_=None),
                dict(out=None), dict(x=ODD), dict(w=ODD), dict(ws_=ODD), dict(out=ODD), dict(bias=P(0x10004)), dict(xs=248),
                dict(xs=260), dict(os_=40), dict(os_=52), dict(ws=P(0x10080))):
        assert linear(**bad) == INVALID, bad
        assert "moe_linear_w4" in moe.moe_last_error()
    assert linear(K=192) == SHAPE and linear(K=64) == SHAPE and linear(N=24, os_=24) == SHAPE
    assert linear(T=0) == OK


BAD_DIMS = [(moe.MoeDims(0, 128, 8, 2), INVALID), (moe.MoeDims(256, -128, 8, 2), INVALID), (moe.MoeDims(256, 128, 0, 1), INVALID),
            (moe.MoeDims(256, 128, 1025, 2), INVALID), (moe.MoeDims(256, 128, 8, 0), INVALID), (moe.MoeDims(256, 128, 8, 9), INVALID),
            (moe.MoeDims(256, 128, 64, 33), INVALID), (moe.MoeDims(200, 128, 8, 2), SHAPE), (moe.MoeDims(256, 64, 8, 2), SHAPE)]


@pytest.mark.parametrize("call", [ffn, layer])
@pytest.mark.parametrize("dims,status", BAD_DIMS)
def test_expert_dims(call, dims, status):
    assert call(d=dims) == status


@pytest.mark.parametrize("call", [ffn, layer])
def test_expert_refusals(call):
    out = "y" if call is ffn else "out"
    for bad in (dict(T=-1), dict(x=None), dict(w=None), dict(s=None), {out: None}, dict(x=ODD), dict(w=ODD), dict(s=ODD),
                {out: ODD}, dict(ws=P(0x10080))):
        assert call(**bad) == INVALID, bad
    for name in ("off", "src") if call is ffn else ("ids", "p"):
        assert call(**{name: None}) == INVALID
    assert call(ws=None) == WORKSPACE and call(n=255) == WORKSPACE
    assert call(T=1 << 30, d=moe.MoeDims(256, 128, 8, 8)) == SHAPE
    assert call(T=0) == OK and call(T=0, x=None, ws=None) == OK


def test_workspaces_grow_with_the_call():
    rng = random.Random(7)
    for _ in range(300):
        d = moe.MoeDims(128 * rng.randint(1, 60), 128 * rng.randint(1, 20), rng.randint(8, 300), rng.randint(1, 8))
        a = rng.randint(0, 9000)
        b = a + rng.choice((0, 1, rng.randint(0, 9000)))
        assert moe.moe_ffn_layer_w4_workspace(d, a) <= moe.moe_ffn_layer_w4_workspace(d, b)
        assert moe.moe_expert_ffn_w4_workspace(d, a) <= moe.moe_expert_ffn_w4_workspace(d, b)
        k, n = d.hidden, 16 * rng.randint(1, 500)
        assert moe.moe_linear_w4_workspace(a, k, n) <= moe.moe_linear_w4_workspace(b, k, n)
    assert moe.moe_ffn_layer_w4_workspace(moe.MoeDims(100, 128, 8, 2), 4) == 0


def test_host_tensors_are_refused():
    x = torch.zeros((2, 128), dtype=torch.bfloat16)
    w = torch.zeros((16, 64), dtype=torch.uint8)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        moe.moe_add_norm(x, None, x)
    with pytest.raises(ValueError, match="x must be a device tensor"):
        moe.moe_linear_w4(x, w, w, x)
    with pytest.raises(ValueError, match="must be a device tensor"):
        moe.moe_ffn_layer_w4(D, 2, x, x, x, w, w, w, w, w, w, x, None, None)
    with pytest.raises(ValueError, match="must be a device tensor"):
        moe.moe_quant_weight_w4(x.float(), w, w)
    with pytest.raises(ValueError, match="must be a device tensor"):
        moe.moe_pack_weight_w4(w, w, w, w)
    with pytest.raises(TypeError):
        moe.moe_add_norm([1.0], None, x)


def test_buffers_take_one_kind_of_weights():
    with pytest.raises(ValueError, match="4 bits or 8"):
        moe.MoELayerBuffers(256, 128, 8, 2, 4, w4=True, w8a16=True)
    with pytest.raises(ValueError, match="themselves"):
        moe.MoELayerBuffers(256, 128, 8, 2, 4, regime=moe.MOE_REGIME_DECODE, w4=True)
