"""GPU: what a call with 4-bit weights leaves alone: other rows than those that hold NaN or infinities, the memory behind
its workspace, and another call that runs beside it.
"""
import numpy as np
import pytest
import torch

from gpu_cases import require_gpu
from test_gpu_ffn_w4 import Stack, route, weights_of
from w4_cases import ordinary, packed, values, whole

pytestmark = pytest.mark.gpu
BITS = {"nan": 0x7fc0, "largest nan": 0x7fff, "negative nan": 0xffff, "inf": 0x7f80, "-inf": 0xff80}


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def spoiled(x, kinds):
    """x with a value of each kind in rows of its own (and the rows)."""
    y, rows = x.clone(), []
    for n, kind in enumerate(kinds):
        row, col = (7 * n + 2) % x.shape[0], (n * 331 + 130) % x.shape[1]
        y.view(torch.int16)[row, col] = BITS[kind] - (1 << 16 if BITS[kind] >> 15 else 0)
        rows.append(row)
    return y, rows


@pytest.mark.parametrize("k,n", [(1024, 528), (640, 1040), (16384, 64)])
@pytest.mark.parametrize("tokens", [1, 3, 16, 17, 40, 100, 300, 700])
def test_rows_of_a_product(moe, tokens, k, n):
    rng = np.random.default_rng(tokens + k)
    q, s = ordinary(rng, n, k)
    w, ws = packed(moe, q, s)
    x = torch.from_numpy(rng.standard_normal((tokens, k)).astype(np.float32)).bfloat16().cuda()
    scratch = torch.empty(max(256, moe.moe_linear_w4_workspace(tokens, k, n)), dtype=torch.uint8, device="cuda")
    for kinds in [[kind] for kind in BITS] + [list(BITS)] if tokens >= 16 else [[kind] for kind in BITS]:
        bad, rows = spoiled(x, kinds)
        good = torch.ones(tokens, dtype=torch.bool, device="cuda")
        good[rows] = False
        ref = bad[rows].double().cpu() @ values(q, s).t().cpu()
        for dtype in (torch.float32, torch.bfloat16):
            outs = [torch.empty((tokens, n), dtype=dtype, device="cuda") for _ in range(2)]
            moe.moe_linear_w4(x, w, ws, outs[0], ws=scratch)
            moe.moe_linear_w4(bad, w, ws, outs[1], ws=scratch)
            assert torch.equal(outs[0][good], outs[1][good])
            got = outs[1][rows].cpu()
            assert torch.equal(torch.isnan(got), torch.isnan(ref)), kinds
            assert torch.equal(got[torch.isinf(ref)].double(), ref[torch.isinf(ref)])
            assert not torch.isfinite(got).any()


@pytest.mark.parametrize("tokens", [1, 4, 20, 31, 70, 300])
def test_tokens_of_a_layer(moe, tokens):
    rng = np.random.default_rng(tokens)
    h, i, e, k = 512, 384, 6, 2
    stack = Stack(moe, rng, h, i, e)
    dims = moe.MoeDims(h, i, e, k)
    x = torch.from_numpy(rng.standard_normal((tokens, h)).astype(np.float32)).bfloat16().cuda()
    ids, p = route(rng, tokens, e, k, 0.3).cuda(), weights_of(rng, tokens, k).cuda()
    ws = torch.empty(moe.moe_ffn_layer_w4_workspace(dims, tokens), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    outs = [torch.empty_like(x) for _ in range(2)]
    moe.moe_ffn_layer_w4(dims, tokens, x, ids, p, *stack.packed, outs[0], status, ws)
    for kinds in [[kind] for kind in BITS] + ([list(BITS)] if tokens > 16 else []):
        bad, rows = spoiled(x, kinds)
        good = torch.ones(tokens, dtype=torch.bool, device="cuda")
        good[rows] = False
        moe.moe_ffn_layer_w4(dims, tokens, bad, ids, p, *stack.packed, outs[1], status, ws)
        assert torch.equal(outs[0][good], outs[1][good])
        # a NaN, or both infinities, in every product's sum
        assert torch.isnan(outs[1][rows]).all(), kinds
    assert int(status.item()) == 0


@pytest.mark.parametrize("t,k,n", [(1, 16384, 512), (16, 65536, 32), (3, 8320, 1040), (17, 65536, 32), (24, 7168, 512), (64, 4096, 1536),
                                   (65, 7168, 1024), (100, 7168, 4096), (201, 4096, 6144), (500, 7168, 1024), (512, 16384, 272)])
def test_sums_stay_in_the_workspace(moe, t, k, n):
    """As much workspace as is asked for, and bytes behind it that stay; the same for the most rows of a smaller call."""
    rng = np.random.default_rng(k + t)
    q, s = whole(rng, n, k)
    w, ws = packed(moe, q, s)
    need = moe.moe_linear_w4_workspace(t, k, n)
    ref_w = values(q, s)
    for rows in (t, max(1, t - 1), (t + 1) // 2):
        x = torch.from_numpy(rng.integers(-1, 2, (rows, k)).astype(np.float32)).bfloat16().cuda()
        scratch = torch.full((need + 4096,), 255, dtype=torch.uint8, device="cuda")
        out = torch.empty((rows, n), device="cuda")
        moe.moe_linear_w4(x, w, ws, out, ws=scratch[:need] if need else None)
        assert torch.equal(out.double(), x.double() @ ref_w.t())
        assert (scratch[need:] == 255).all()


def test_calls_side_by_side(moe):
    """Two streams with a workspace each, a layer and a product in turn on both: as one after the other."""
    rng = np.random.default_rng(4)
    h, i, e, k, tokens = 1024, 512, 8, 2, 48
    stack = Stack(moe, rng, h, i, e)
    dims = moe.MoeDims(h, i, e, k)
    q, s = ordinary(rng, 1536, h)
    w, w_s = packed(moe, q, s)
    x = [torch.from_numpy(rng.standard_normal((tokens, h)).astype(np.float32)).bfloat16().cuda() for _ in range(2)]
    ids, p = [route(rng, tokens, e, k, 0.2).cuda() for _ in range(2)], weights_of(rng, tokens, k).cuda()
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def buffers():
        return (torch.empty((tokens, h), dtype=torch.bfloat16, device="cuda"),
                torch.empty((tokens, 1536), dtype=torch.bfloat16, device="cuda"),
                torch.empty(moe.moe_ffn_layer_w4_workspace(dims, tokens), dtype=torch.uint8, device="cuda"),
                torch.empty(max(256, moe.moe_linear_w4_workspace(tokens, h, 1536)), dtype=torch.uint8, device="cuda"))

    def call(n, to, stream=None):
        out, y, ws, scratch = to
        moe.moe_ffn_layer_w4(dims, tokens, x[n], ids[n], p, *stack.packed, out, status, ws, stream=stream)
        moe.moe_linear_w4(out, w, w_s, y, ws=scratch, stream=stream)
    alone, beside = [buffers() for _ in range(2)], [buffers() for _ in range(2)]
    for n in range(2):
        call(n, alone[n])
    torch.cuda.synchronize()
    streams = [torch.cuda.Stream() for _ in range(2)]
    for _ in range(20):
        for n in range(2):
            call(n, beside[n], streams[n])
    torch.cuda.synchronize()
    for n in range(2):
        assert torch.equal(alone[n][0], beside[n][0]) and torch.equal(alone[n][1], beside[n][1])
    assert int(status.item()) == 0
