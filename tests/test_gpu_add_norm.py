"""GPU: moe_add_norm against its formula in 64 bits.

Tolerances count roundings: the sum is one fp32 addition (2^-24) rounded to bf16 (2^-8) where it is bf16.  The norm:
squares, their sum (at most H + 10 roundings in all, each at most 2^-24 of a sum of positive terms, halved by the
root), quotient, root, reciprocal and two products: (H / 2 + 16) 2^-24 and 2^-8 for bf16.  Scales are a maximum over 448;
codes the nearest of the quotient, which is off as much, so at most half a step (2^-4) more than that.
"""
import numpy as np
import pytest
import torch

from gpu_cases import require_gpu
from oracle import w4_oracle as wo

pytestmark = pytest.mark.gpu
EPS = 1e-6
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def f32_bound(h):
    return (h / 2 + 16) * 2.0 ** -24


def check(got, ref, rel, tiny=0.0):
    got = got.double().cpu().numpy()
    assert got.shape == ref.shape
    off = np.abs(got - ref) - rel * np.abs(ref)
    assert np.isfinite(got).all() and (off <= tiny).all(), float(off.max())


def check_codes(q, s, y):
    """q [rows, H], s [rows, H / 128] against fp64 y [rows, H]."""
    rel = f32_bound(y.shape[-1])
    y = y.reshape(y.shape[0], -1, 128)
    top = np.abs(y).max(-1)
    check(s, top / 448, rel + 2.0 ** -24)
    v = q.view(torch.float8_e4m3fn).double().cpu().numpy().reshape(y.shape)
    unit = y / np.where(top > 0, top / 448, 1.0)[..., None]
    # half a step of normal codes, or of the smallest (2^-9 apart)
    assert (np.abs(v - unit) <= np.maximum(np.abs(unit) * 2.0 ** -4, 2.0 ** -10) + 448 * 4 * rel).all()


CASES = [  # tokens, H, heads, x, stream, residual, codes
    (1, 7168, 1, "bf16", "bf16", True, True), (1, 128, 1, "bf16", "bf16", False, False), (3, 8, 1, "bf16", "f32", True, False),
    (5, 64, 7, "bf16", "bf16", False, False), (67, 128, 5, "bf16", "bf16", True, True), (9, 72, 3, "f32", "bf16", True, False),
    (33, 136, 1, "bf16", "bf16", True, False), (4, 512, 2, "f32", "f32", True, True), (2, 520, 1, "bf16", "bf16", True, False),
    (7, 640, 1, "bf16", "f32", True, True), (3, 2048, 1, "f32", "f32", True, True), (3, 2056, 1, "bf16", "bf16", True, False),
    (700, 1024, 1, "bf16", "bf16", True, True), (5000, 2176, 1, "bf16", "f32", True, True), (2, 8192, 1, "f32", "bf16", False, True),
    (3, 8200, 1, "bf16", "bf16", True, False), (2, 8320, 1, "bf16", "f32", True, True), (1, 32768, 1, "f32", "f32", True, True),
    (70001, 64, 1, "bf16", "bf16", True, False)]


@pytest.mark.parametrize("tokens,h,heads,xt,st,residual,codes", CASES)
def test_formula(moe, tokens, h, heads, xt, st, residual, codes):
    g = torch.Generator().manual_seed(tokens * 7 + h)
    shape = (tokens, heads, h) if heads > 1 else (tokens, h)
    x = (torch.randn(shape, generator=g) * 3).to(TYPES[xt])
    r = (torch.randn(shape, generator=g) * 2).to(TYPES[st]) if residual else None
    w = (1 + 0.3 * torch.randn(h, generator=g)).bfloat16()
    dx, dr = x.cuda(), r.cuda() if residual else None
    out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
    total = torch.empty(shape, dtype=TYPES[st], device="cuda") if residual else None
    q = torch.empty((tokens * heads, h), dtype=torch.uint8, device="cuda") if codes else None
    s = torch.empty((tokens * heads, h // 128), dtype=torch.float32, device="cuda") if codes else None
    moe.moe_add_norm(dx, w.cuda(), out, q, s, residual=dr, sum_out=total, eps=EPS)
    z, y = wo.add_norm(x.double().numpy(), r.double().numpy() if residual else None, w.double().numpy(), EPS)
    rel = f32_bound(h)
    # a sum that cancels is off by 2^-24 of its terms, which weigh on the row's norm no more than the row's largest
    lost = 2.0 ** -23 * np.abs(y).max()
    check(out, y, 2.0 ** -8 + rel, lost)
    if residual:
        check(total, z, (2.0 ** -8 if st == "bf16" else 0) + 2.0 ** -24, 1e-30)
    if codes:
        check_codes(q, s, y.reshape(tokens * heads, h))


def test_codes_are_those_of_the_layers_quantizer(moe):
    """A weight of ones, and rows whose root mean square is exactly 1 and eps lost beside it: y is z, bit for bit."""
    x = torch.ones((40, 256))
    g = torch.Generator().manual_seed(5)
    x[torch.rand((40, 256), generator=g) < 0.5] = -1.0
    x = x.bfloat16().cuda()
    q, s, q2, s2 = (torch.empty(n, dtype=t, device="cuda") for n, t in
                    (((40, 256), torch.uint8), ((40, 2), torch.float32), ((40, 256), torch.uint8), ((40, 2), torch.float32)))
    moe.moe_add_norm(x, None, None, q, s, eps=1e-12)
    moe.moe_quant_act(x, q2, s2)
    assert torch.equal(q, q2) and torch.equal(s, s2)


def test_strided_rows_and_untouched_surroundings(moe):
    """Query heads inside a packed projection, in place; the rest of the projection stays as it was."""
    g = torch.Generator().manual_seed(8)
    row = torch.randn((37, 10 * 64), generator=g).bfloat16()
    w = torch.randn(64, generator=g).bfloat16()
    dev = row.cuda()
    x = dev[:, 64:7 * 64].unflatten(1, (6, 64))
    moe.moe_add_norm(x, w.cuda(), x, eps=1e-5, weight_offset=1.0)
    _, y = wo.add_norm(row[:, 64:7 * 64].double().numpy().reshape(37, 6, 64), None, w.double().numpy(), 1e-5, 1.0)
    check(dev[:, 64:7 * 64].unflatten(1, (6, 64)), y, 2.0 ** -8 + f32_bound(64))
    assert torch.equal(dev[:, :64].cpu(), row[:, :64]) and torch.equal(dev[:, 7 * 64:].cpu(), row[:, 7 * 64:])


@pytest.mark.parametrize("st", ["bf16", "f32"])
def test_sum_in_place_of_the_residual(moe, st):
    g = torch.Generator().manual_seed(9)
    x, r = torch.randn((19, 384), generator=g).bfloat16(), torch.randn((19, 400), generator=g).to(TYPES[st])
    dx, dr = x.cuda(), r.cuda()
    view = dr[:, :384]
    moe.moe_add_norm(dx, None, dx, residual=view, sum_out=view)
    z, y = wo.add_norm(x.double().numpy(), r[:, :384].double().numpy(), None, 1e-6)
    check(view, z, (2.0 ** -8 if st == "bf16" else 0) + 2.0 ** -24, 1e-30)
    check(dx, y, 2.0 ** -8 + f32_bound(384), 2.0 ** -23 * np.abs(y).max())
    assert torch.equal(dr[:, 384:].cpu(), r[:, 384:])


@pytest.mark.parametrize("h", [64, 128, 512, 1024, 7168, 16384])
def test_sizes_that_fp32_squares_do_not_hold(moe, h):
    """Rows of huge, ordinary and tiny values and of zeros side by side, so that one row's range is not another's."""
    g = torch.Generator().manual_seed(h)
    x = torch.randn((8, h), generator=g)
    x = x * torch.tensor([1e38, 1.0, 1e-30, 0.0, 1e20, 1e-3, 1e37, 1e18])[:, None]
    x = x.clamp(-3e38, 3e38)
    out = torch.empty((8, h), dtype=torch.bfloat16, device="cuda")
    moe.moe_add_norm(x.cuda(), None, out, eps=1e-6)
    _, y = wo.add_norm(x.double().numpy(), None, None, 1e-6)
    check(out, y, 2.0 ** -8 + f32_bound(h), 2.0 ** -133)
    assert (out[3] == 0).all()


def test_zero_rows_of_codes_and_no_tokens(moe):
    x = torch.zeros((2, 256), dtype=torch.bfloat16, device="cuda")
    q, s = torch.full((2, 256), 9, dtype=torch.uint8, device="cuda"), torch.full((2, 2), 9.0, device="cuda")
    moe.moe_add_norm(x, None, None, q, s)
    assert not q.any() and not s.any()
    empty = torch.empty((0, 256), dtype=torch.bfloat16, device="cuda")
    moe.moe_add_norm(empty, None, empty)


def test_refusals_of_the_binding(moe):
    x = torch.zeros((4, 256), dtype=torch.bfloat16, device="cuda")
    f = x.float()
    q, s = torch.zeros((4, 256), dtype=torch.uint8, device="cuda"), torch.zeros((4, 2), device="cuda")
    for bad in (dict(out=f), dict(out=x[:3]), dict(out=x[:, :128]), dict(out=x.half()), dict(out=x, residual=x[:, :128]),
                dict(out=x, residual=f, sum_out=x), dict(out=x, sum_out=x[:2]), dict(q=q, s=s[:3]), dict(q=q[:3], s=s),
                dict(out=x.t().contiguous().t()), dict(out=x, weight=x[0, :128]), dict(out=x, weight=f[0]),
                dict(out=x, weight=x[0].half()), dict(q=q, s=s.half())):
        args = dict(weight=None) | bad
        with pytest.raises(ValueError):
            moe.moe_add_norm(x, **args)
    with pytest.raises(ValueError):
        moe.moe_add_norm(x[0], None, x[0])
    for bad in (dict(), dict(out=x, eps=0.0), dict(q=q), dict(out=x.expand(1, 4, 256)[0].as_strided((4, 256), (0, 1)))):
        with pytest.raises(moe.MoEError):
            moe.moe_add_norm(x, None, **bad)


def test_other_stream_and_replayed_graph(moe):
    g = torch.Generator().manual_seed(11)
    x = torch.randn((65, 896), generator=g).bfloat16().cuda()
    r = torch.randn((65, 896), generator=g).cuda()
    outs = [torch.empty_like(x) for _ in range(2)]
    sums = [torch.empty_like(r) for _ in range(2)]
    stream = torch.cuda.Stream()
    stream.wait_stream(torch.cuda.current_stream())
    moe.moe_add_norm(x, None, outs[0], residual=r, sum_out=sums[0], stream=stream)
    torch.cuda.current_stream().wait_stream(stream)
    graph = torch.cuda.CUDAGraph()
    with torch.cuda.graph(graph):
        moe.moe_add_norm(x, None, outs[1], residual=r, sum_out=sums[1])
    for turn in range(3):
        x.copy_(torch.randn((65, 896), generator=g).bfloat16())
        graph.replay()
        moe.moe_add_norm(x, None, outs[0], residual=r, sum_out=sums[0])
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[1]) and torch.equal(sums[0], sums[1]), turn
