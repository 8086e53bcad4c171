"""GPU: 4-bit weights quantized, packed and multiplied.

Most products are of small whole numbers and weights that are multiples of 1/4, so that fp32 holds every partial sum
and the result is known bit for bit.  With ordinary values the bound is K roundings of 2^-23 of the terms' sizes (a
matrix instruction may cut its sums instead of rounding them), and 2^-8 for an output in bf16.
"""
import numpy as np
import pytest
import torch

from gpu_cases import require_gpu
from oracle import w4_oracle as wo
from w4_cases import on_canvas, ordinary, packed, untouched, values, whole

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def test_quantizer_bit_for_bit(moe):
    rng = np.random.default_rng(1)
    w = (rng.standard_normal((6, 160, 128)) * np.exp(2 * rng.standard_normal((6, 160, 1)))).astype(np.float32)
    w[0, 0, :32] = 0.0
    w[0, 1, :8] = [0.25, 0.75, 1.25, 1.75, 2.5, 3.5, 5.0, 7.0]           # ties, at scale 1
    w[0, 1, 8:32] = 0.0
    w[0, 2, :32] = -w[0, 1, :32]
    w[0, 3, :32] = np.nextafter(w[0, 1, :32], 10, dtype=np.float32)      # above 7: the next scale
    w[0, 4, :32] = np.nextafter(w[0, 1, :32], 0, dtype=np.float32)
    w[0, 5, :32] = 2.0 ** -149
    w[0, 6, :32] = 3e38
    w[0, 7, :32] = w[0, 1, :32] * np.float32(2.0 ** -118)
    w[0, 8, :4] = [2.0 ** 123, -2.0 ** 122, 1.0, 0.0]
    q, s = wo.quantize(w)
    dq, ds = torch.empty(q.shape, dtype=torch.uint8, device="cuda"), torch.empty(s.shape, dtype=torch.uint8, device="cuda")
    moe.moe_quant_weight_w4(torch.from_numpy(w).cuda(), dq, ds)
    assert np.array_equal(ds.cpu().numpy(), s)
    assert np.array_equal(dq.cpu().numpy(), q)


@pytest.mark.parametrize("mats,rows,cols", [(1, 16, 128), (3, 48, 640), (2, 32, 1024), (1, 160, 1152)])
def test_packed_layout(moe, mats, rows, cols):
    rng = np.random.default_rng(cols)
    q = rng.integers(0, 256, (mats, rows, cols // 2)).astype(np.uint8)
    s = rng.integers(0, 253, (mats, rows, cols // 32)).astype(np.uint8)
    w, ws = packed(moe, q, s)
    ref = [wo.pack(a, b) for a, b in zip(q, s)]
    assert np.array_equal(w.cpu().numpy().reshape(-1), np.concatenate([a for a, _ in ref]))
    assert np.array_equal(ws.cpu().numpy(), np.concatenate([b for _, b in ref]))


def test_scales_out_of_range_are_reported(moe):
    q = torch.zeros((32, 64), dtype=torch.uint8, device="cuda")
    s = torch.full((32, 4), 127, dtype=torch.uint8, device="cuda")
    w, ws = torch.empty_like(q), torch.empty(moe.moe_w4_scale_bytes(1, 32, 128), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    for value, bad in ((252, 0), (0, 0), (253, moe.MOE_DEV_BAD_SCALE), (255, moe.MOE_DEV_BAD_SCALE)):
        s[17, 2] = value
        status.zero_()
        moe.moe_pack_weight_w4(q, s, w, ws, status)
        assert int(status.item()) == bad
        moe.moe_pack_weight_w4(q, s, w, ws)  # without a word to report in


def times(moe, x, w, ws, n, out_type=torch.float32, bias=None, x_stride=None, out_stride=None):
    """moe_linear_w4 of bf16 x into a view of a canvas; what lies around the view has to stay."""
    t, k = x.shape
    if x_stride:
        wide = torch.full((t, x_stride), float("nan"), dtype=torch.bfloat16, device="cuda")
        wide[:, :k] = x
        x = wide[:, :k]
    out, canvas = on_canvas(t, n, out_stride or n + 8 - n % 8, out_type)
    scratch = torch.empty(max(256, moe.moe_linear_w4_workspace(t, k, n)), dtype=torch.uint8, device="cuda")
    moe.moe_linear_w4(x, w, ws, out, bias=bias, ws=scratch)
    assert untouched(canvas, t, n)
    return out


@pytest.mark.parametrize("tokens", [1, 20, 80])
def test_every_code_and_scale_expands_exactly(moe, tokens):
    """Column c of the identity's rows reads column c of W back: every code under every scale whose weights are normal
    in bf16 (bytes 2 .. 252)."""
    q = np.zeros((256, 64), np.uint8)
    s = np.full((256, 4), 127, np.uint8)
    row = np.arange(256)
    for c in range(16):                                  # columns 0 .. 15 the codes, 32 .. 47 too
        for first in (0, 32):
            q[:, (first + c) // 2] |= c << 4 * (c % 2)
    s[:, 0] = np.clip(row, 2, 252)
    s[:, 1] = np.clip(255 - row, 2, 252)
    w, ws = packed(moe, q, s)
    ref = wo.values(q, s)
    for first in range(0, 128, tokens):
        t = min(tokens, 128 - first)
        x = torch.zeros((tokens, 128), dtype=torch.bfloat16, device="cuda")
        x[torch.arange(t), first + torch.arange(t)] = 1.0
        out = times(moe, x, w, ws, 256)
        assert np.array_equal(out[:t].double().cpu().numpy(), ref[:, first:first + t].T)


TOKENS = [1, 2, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 200, 257, 1000]
SIZES = [(128, 16), (256, 48), (384, 256), (640, 272), (1024, 1536), (1152, 240), (7168, 512), (2048, 4112), (4480, 96), (8320, 48),
         (16384, 32), (5120, 1040)]


@pytest.mark.parametrize("k,n", SIZES)
def test_whole_numbers_bit_for_bit(moe, k, n):
    rng = np.random.default_rng(k + n)
    q, s = whole(rng, n, k)
    w, ws = packed(moe, q, s)
    ref_w = values(q, s)
    bias = torch.from_numpy(rng.integers(-8, 9, n).astype(np.float32)).bfloat16().cuda()
    for i, t in enumerate(TOKENS):
        x = torch.from_numpy(rng.integers(-4, 5, (t, k)).astype(np.float32)).bfloat16().cuda()
        ref = (x.double() @ ref_w.t())
        print(f"k={k} n={n} t={t}", flush=True)
        out = times(moe, x, w, ws, n, x_stride=k + 8 * (i % 3) if i % 3 else None, out_stride=((n + 7) // 8 + i % 4) * 8)
        assert torch.equal(out.double(), ref), t
        out = times(moe, x, w, ws, n, torch.bfloat16, bias)
        assert torch.equal(out, (ref + bias.double()).float().bfloat16()), t


@pytest.mark.parametrize("k,n", [(1152, 4176), (2048, 4096), (2048, 4128), (7168, 4144), (8192, 4112), (16384, 1024), (16384, 1072)])
def test_whole_numbers_where_items_change(moe, k, n):
    """Few rows: matrices on both sides of the size where a workgroup's item has one tile of rows or two, odd ones among them."""
    test_whole_numbers_bit_for_bit(moe, k, n)


@pytest.mark.parametrize("tokens", [1, 30, 64, 100, 300])
def test_ordinary_values(moe, tokens):
    k, n = 2048, 528
    rng = np.random.default_rng(tokens)
    q, s = ordinary(rng, n, k)
    w, ws = packed(moe, q, s)
    x = torch.from_numpy((rng.standard_normal((tokens, k)) * np.exp(rng.standard_normal((tokens, k)))).astype(np.float32)).bfloat16().cuda()
    ref_w = values(q, s)
    ref, size = x.double() @ ref_w.t(), x.double().abs() @ ref_w.abs().t()
    bias = torch.from_numpy(rng.standard_normal(n).astype(np.float32)).bfloat16().cuda()
    out = times(moe, x, w, ws, n).double()
    assert ((out - ref).abs() <= k * 2.0 ** -23 * size).all()
    ref = ref + bias.double()
    out = times(moe, x, w, ws, n, torch.bfloat16, bias).double()
    assert ((out - ref).abs() <= k * 2.0 ** -23 * (size + bias.double().abs()) + 2.0 ** -8 * ref.abs()).all()


@pytest.mark.parametrize("tokens,k,n", [(1500, 384, 2064), (2100, 256, 4112), (8200, 256, 1040), (4097, 640, 2560),
                                        (8191, 384, 4096), (6200, 128, 8208), (12290, 256, 2048)])
def test_many_tokens_bit_for_bit(moe, tokens, k, n):
    rng = np.random.default_rng(tokens)
    q, s = whole(rng, n, k)
    w, ws = packed(moe, q, s)
    x = torch.from_numpy(rng.integers(-4, 5, (tokens, k)).astype(np.float32)).bfloat16().cuda()
    assert torch.equal(times(moe, x, w, ws, n, x_stride=k + 16).double(), x.double() @ values(q, s).t())


def test_long_and_wide(moe):
    """K past 2^15 with few columns, and many columns with little K."""
    for k, n, t in ((40960, 32, 3), (40960, 32, 70), (75776, 16, 2), (75776, 16, 16), (128, 70000, 2), (128, 70000, 66)):
        rng = np.random.default_rng(k)
        q, s = whole(rng, n, k)
        w, ws = packed(moe, q, s)
        x = torch.from_numpy(rng.integers(-1, 2, (t, k)).astype(np.float32)).bfloat16().cuda()
        assert torch.equal(times(moe, x, w, ws, n).double(), x.double() @ values(q, s).t())


def test_no_tokens_and_refusals(moe):
    rng = np.random.default_rng(2)
    w, ws = packed(moe, *whole(rng, 48, 256))
    x = torch.zeros((3, 256), dtype=torch.bfloat16, device="cuda")
    out = torch.zeros((3, 48), dtype=torch.bfloat16, device="cuda")
    moe.moe_linear_w4(x[:0], w, ws, out[:0])
    for bad in (dict(x=x.half()), dict(x=x.float()), dict(x=x[:2]), dict(x=x[:, :128]), dict(x=x[None]), dict(w=w[:24]),
                dict(w=w.float()), dict(w_s=ws[:256]), dict(out=out.half()), dict(out=out[:, :32]), dict(out=out.t()),
                dict(bias=out[0, :32]), dict(bias=out[0].float()), dict(bias=out[0].half())):
        with pytest.raises(ValueError):
            moe.moe_linear_w4(**(dict(x=x, w=w, w_s=ws, out=out) | bad))
    for bad in (dict(w=None), dict(w_s=None), dict(out=torch.zeros((3, 52), dtype=torch.bfloat16, device="cuda")[:, :48])):
        with pytest.raises(moe.MoEError):
            moe.moe_linear_w4(**(dict(x=x, w=w, w_s=ws, out=out) | bad))


@pytest.mark.parametrize("tokens", [1, 40, 150])
def test_other_stream_and_replayed_graphs(moe, tokens):
    """Two graphs with a workspace each, replayed in turn with eager calls between."""
    rng = np.random.default_rng(tokens)
    k, n = 1024, 272
    w, ws = packed(moe, *ordinary(rng, n, k))
    x = torch.from_numpy(rng.standard_normal((tokens, k)).astype(np.float32)).bfloat16().cuda()
    need = max(256, moe.moe_linear_w4_workspace(tokens, k, n))
    outs = [torch.empty((tokens, n), dtype=torch.bfloat16, device="cuda") for _ in range(4)]
    scratch = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(4)]
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    moe.moe_linear_w4(x, w, ws, outs[3], ws=scratch[3])
    for i, graph in enumerate(graphs):
        with torch.cuda.graph(graph):
            moe.moe_linear_w4(x, w, ws, outs[i], ws=scratch[i])
    stream = torch.cuda.Stream()
    for turn in range(3):
        x.copy_(torch.from_numpy(rng.standard_normal((tokens, k)).astype(np.float32)).bfloat16())
        stream.wait_stream(torch.cuda.current_stream())
        moe.moe_linear_w4(x, w, ws, outs[2], ws=scratch[2], stream=stream)
        for graph in graphs:
            graph.replay()
        moe.moe_linear_w4(x, w, ws, outs[3], ws=scratch[3])
        torch.cuda.synchronize()
        assert all(torch.equal(o, outs[3]) for o in outs[:3]), turn
