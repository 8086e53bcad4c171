"""GPU: routed experts with 4-bit weights against the formula in 64 bits, the layer in one call against its steps, and a
decode step that runs from norm to norm.

Bounds: G and U are off by H roundings of 2^-23 of their terms' sizes each, which silu passes on with a slope of at most
1.1; h = silu(G) U is rounded once to bf16 (2^-8) after a few roundings in fp32 (2^-20 covers them); y adds I roundings of
2^-23 of its own terms' sizes.
"""
import importlib.util
import os

import numpy as np
import pytest
import torch

from gpu_cases import log, require_gpu
from oracle import w4_oracle as wo
from w4_cases import ordinary, packed, values

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


class Stack:
    """Experts' weights: packed on the device, and the values they stand for."""

    def __init__(self, moe, rng, h, i, e):
        self.dims = (h, i, e)
        self.packed, self.values = [], []
        for rows, cols in ((i, h), (i, h), (h, i)):
            q, s = ordinary(rng, e, rows, cols)
            self.packed += packed(moe, q, s)
            self.values.append(values(q, s))

    def rows(self, e, x):
        """(y, bound) of activation rows x [n, H] (fp64) through expert e."""
        x = x.cuda()
        wg, wu, wd = (v[e] for v in self.values)
        h, i, _ = self.dims
        g, u = x @ wg.t(), x @ wu.t()
        dg, du = (h * 2.0 ** -23 * (x.abs() @ w.abs().t()) for w in (wg, wu))
        silu = g * torch.sigmoid(g)
        mid = silu * u
        off = (2.0 ** -8 + 2.0 ** -20) * mid.abs() + 1.1 * dg * (u.abs() + du) + silu.abs() * du
        return (mid @ wd.t()).cpu(), ((off + i * 2.0 ** -23 * mid.abs()) @ wd.abs().t()).cpu()


def route(rng, tokens, experts, k, skew):
    """Expert ids [tokens, k], distinct in a token: even, or most tokens on the same experts."""
    p = np.exp(-skew * np.arange(experts))
    ids = np.stack([rng.choice(experts, k, replace=False, p=p / p.sum()) for _ in range(tokens)])
    return torch.from_numpy(ids.astype(np.int32))


def weights_of(rng, tokens, k):
    p = rng.random((tokens, k)).astype(np.float32) + 0.1
    return torch.from_numpy(p / p.sum(1, keepdims=True))


def run(moe, stack, x, ids, p, fused):
    h, i, e = stack.dims
    buf = moe.MoELayerBuffers(h, i, e, ids.shape[1], x.shape[0], w4=True, fused=fused)
    if not fused:
        buf.y_rows.fill_(float("nan"))
    out = moe.run_layer(buf, x.cuda(), ids.cuda(), p.cuda(), stack.packed)
    torch.cuda.synchronize()
    assert int(buf.dev_status.item()) == 0
    return out.view(torch.bfloat16), buf


CASES = [  # hidden, inter, experts, k, tokens, skew
    (128, 128, 1, 1, 1, 0.0), (256, 128, 8, 2, 16, 0.0), (384, 256, 5, 3, 1, 0.0), (256, 128, 8, 8, 7, 0.0),
    (512, 384, 16, 2, 33, 0.5), (256, 256, 300, 4, 17, 0.0), (640, 128, 4, 1, 64, 2.0), (256, 128, 3, 2, 63, 0.0),
    (256, 2048, 8, 8, 2, 0.0), (2048, 4096, 5, 2, 20, 0.3), (7168, 1280, 3, 1, 18, 0.5), (4096, 2176, 2, 2, 7, 0.0),
    (512, 256, 256, 8, 640, 0.0), (512, 256, 256, 8, 1920, 0.002), (512, 256, 256, 8, 2880, 0.0), (512, 256, 256, 8, 4480, 0.001),
    (512, 384, 8, 2, 250, 0.0), (512, 384, 8, 2, 400, 0.0), (256, 128, 8, 2, 65, 0.0), (512, 256, 16, 4, 100, 0.6), (384, 384, 4, 2, 130, 3.0), (256, 128, 1024, 8, 200, 0.0),
    (256, 128, 2, 1, 513, 1.5), (1280, 640, 6, 2, 257, 0.0), (256, 128, 1, 1, 1000, 0.0)]


@pytest.mark.parametrize("h,i,e,k,tokens,skew", CASES)
def test_layer(moe, h, i, e, k, tokens, skew):
    rng = np.random.default_rng(h + i + e + tokens)
    stack = Stack(moe, rng, h, i, e)
    x = torch.from_numpy(rng.standard_normal((tokens, h)).astype(np.float32)).bfloat16()
    ids, p = route(rng, tokens, e, k, skew), weights_of(rng, tokens, k)
    ref, bound = torch.zeros((tokens, h), dtype=torch.float64), torch.zeros((tokens, h), dtype=torch.float64)
    size = torch.zeros((tokens, h), dtype=torch.float64)
    for ex in ids.unique().tolist():
        t, j = (ids == ex).nonzero(as_tuple=True)
        y, off = stack.rows(ex, x[t].double())
        w = p[t, j].double()[:, None]
        ref.index_add_(0, t, y * w)
        bound.index_add_(0, t, off * w)
        size.index_add_(0, t, y.abs() * w)
    fused, _ = run(moe, stack, x, ids, p, True)
    out = fused.double().cpu()
    worst = float(((out - ref).abs() / (bound + (k + 1) * 2.0 ** -24 * size + 2.0 ** -8 * (ref.abs() + bound))).max())
    log(f"H={h} I={i} E={e} k={k} T={tokens}: {worst:.3f} of the bound")
    assert torch.isfinite(out).all() and worst <= 1.0
    steps, buf = run(moe, stack, x, ids, p, False)
    # the same sums; a slot's row is written whether or not another's is
    assert torch.isfinite(buf.y_rows).all()
    off = (steps.double().cpu() - ref).abs()
    assert (off <= bound + (k + 1) * 2.0 ** -24 * size + 2.0 ** -8 * (ref.abs() + bound)).all()


@pytest.mark.parametrize("h,i", [(128, 256), (512, 1024), (1024, 512), (640, 2176), (2048, 384), (4352, 128), (8192, 256)])
@pytest.mark.parametrize("tokens", [24, 25])
def test_layers_of_eight_rows_an_expert(moe, h, i, tokens):
    """At eight rows an expert and behind it the kernel changes; some experts have two tiles of rows, some none."""
    test_layer(moe, h, i, 12, 4, tokens, 1.5)


@pytest.mark.parametrize("tokens", [1, 5, 64, 65, 300])
def test_no_run_differs_from_another(moe, tokens):
    rng = np.random.default_rng(tokens)
    stack = Stack(moe, rng, 512, 256, 12)
    x = torch.from_numpy(rng.standard_normal((tokens, 512)).astype(np.float32)).bfloat16()
    ids, p = route(rng, tokens, 12, 4, 0.4), weights_of(rng, tokens, 4)
    first = run(moe, stack, x, ids, p, True)[0].clone()
    for _ in range(4):
        assert torch.equal(run(moe, stack, x, ids, p, True)[0], first)


@pytest.mark.parametrize("tokens", [1, 3, 40, 90])
def test_bad_ids_are_reported_and_leave_the_other_tokens(moe, tokens):
    rng = np.random.default_rng(tokens)
    h, i, e, k = 256, 128, 8, 2
    stack = Stack(moe, rng, h, i, e)
    x = torch.from_numpy(rng.standard_normal((tokens, h)).astype(np.float32)).bfloat16()
    ids, p = route(rng, tokens, e, k, 0.0), weights_of(rng, tokens, k)
    good, _ = run(moe, stack, x, ids, p, True)
    good = good.clone()
    dims = moe.MoeDims(h, i, e, k)
    ws = torch.empty(moe.moe_ffn_layer_w4_workspace(dims, tokens), dtype=torch.uint8, device="cuda")
    for bad, bit in ((e, moe.MOE_DEV_BAD_EXPERT_ID), (-1, moe.MOE_DEV_BAD_EXPERT_ID), (2 ** 31 - 1, moe.MOE_DEV_BAD_EXPERT_ID),
                     (None, moe.MOE_DEV_DUP_EXPERT_ID)):
        some = ids.clone()
        at = tokens // 2
        some[at, 1] = some[at, 0] if bad is None else bad
        ws.fill_(255)
        out = torch.zeros((tokens, h), dtype=torch.bfloat16, device="cuda")
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        moe.moe_ffn_layer_w4(dims, tokens, x.cuda(), some.cuda(), p.cuda(), *stack.packed, out, status, ws)
        assert int(status.item()) == bit
        rest = torch.arange(tokens) != at
        assert torch.equal(out[rest.cuda()], good[rest.cuda()])


@pytest.mark.parametrize("tokens", [1, 2, 70])
def test_no_id_is_an_experts(moe, tokens):
    """Every slot is bad: it is reported, and nothing outside the output is written."""
    rng = np.random.default_rng(3)
    h, i, e, k = 256, 128, 8, 2
    stack = Stack(moe, rng, h, i, e)
    dims = moe.MoeDims(h, i, e, k)
    x = torch.ones((tokens, h), dtype=torch.bfloat16, device="cuda")
    ids = torch.full((tokens, k), 2 ** 30, dtype=torch.int32, device="cuda")
    canvas = torch.full((tokens + 2, h), 7.0, dtype=torch.bfloat16, device="cuda")
    need = moe.moe_ffn_layer_w4_workspace(dims, tokens)
    ws = torch.full((need + 256,), 255, dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    moe.moe_ffn_layer_w4(dims, tokens, x, ids, torch.ones((tokens, k), device="cuda"), *stack.packed, canvas[1:-1], status,
                         ws[:need])
    assert int(status.item()) == moe.MOE_DEV_BAD_EXPERT_ID
    assert (canvas[0] == 7).all() and (canvas[-1] == 7).all() and (ws[need:] == 255).all()


def test_rows_outside_the_offsets_stay(moe):
    """A step call with rows of some experts only: the others' rows of y are left as they were."""
    rng = np.random.default_rng(6)
    h, i, e, k, tokens = 256, 128, 4, 1, 20
    stack = Stack(moe, rng, h, i, e)
    x = torch.from_numpy(rng.standard_normal((tokens, h)).astype(np.float32)).bfloat16()
    offsets = torch.tensor([3, 3, 9, 9, 14], dtype=torch.int32, device="cuda")
    src = torch.from_numpy(rng.permutation(tokens).astype(np.int32))
    y = torch.full((tokens, h), float("nan"), device="cuda")
    dims = moe.MoeDims(h, i, e, k)
    ws = torch.empty(moe.moe_expert_ffn_w4_workspace(dims, tokens), dtype=torch.uint8, device="cuda")
    moe.moe_expert_ffn_w4(dims, tokens, x.cuda(), offsets, src.cuda(), *stack.packed, y, ws)
    got = y.double().cpu()
    assert torch.isnan(got[:3]).all() and torch.isnan(got[14:]).all()
    for ex, lo, hi in ((1, 3, 9), (3, 9, 14)):
        ref, bound = stack.rows(ex, x[src[lo:hi].long()].double())
        assert ((got[lo:hi] - ref).abs() <= bound).all()


def test_refusals_of_the_binding(moe):
    rng = np.random.default_rng(7)
    h, i, e, k, t = 256, 128, 4, 2, 6
    stack = Stack(moe, rng, h, i, e)
    dims = moe.MoeDims(h, i, e, k)
    x = torch.zeros((t, h), dtype=torch.bfloat16, device="cuda")
    ids, p = torch.zeros((t, k), dtype=torch.int32, device="cuda"), torch.zeros((t, k), device="cuda")
    ws = torch.empty(moe.moe_ffn_layer_w4_workspace(dims, t), dtype=torch.uint8, device="cuda")
    args = [dims, t, x, ids, p, *stack.packed, x.clone(), None, ws]
    for at, bad in ((2, x[:3]), (2, x.half()), (2, x[:, :128]), (3, ids.long()), (3, ids[:2]), (4, p.double()), (4, p[:, :1]),
                    (5, stack.packed[0][:2]), (6, stack.packed[1][:64]), (9, stack.packed[4][:1]), (11, x.float()),
                    (11, x[:2]), (12, p)):
        broken = list(args)
        broken[at] = bad
        with pytest.raises(ValueError):
            moe.moe_ffn_layer_w4(*broken)
    with pytest.raises(moe.MoEError):
        moe.moe_ffn_layer_w4(*args[:-1], ws[:256])
    with pytest.raises(moe.MoEError):
        moe.moe_ffn_layer_w4(*args[:-1], None)
    off, src = torch.zeros(e + 1, dtype=torch.int32, device="cuda"), torch.zeros(t * k, dtype=torch.int32, device="cuda")
    y = torch.zeros((t * k, h), device="cuda")
    args = [dims, t, x, off, src, *stack.packed, y, ws]
    for at, bad in ((3, off[:e]), (4, src[:3]), (3, off.float()), (11, y[:3]), (11, y.bfloat16()), (2, x.float())):
        broken = list(args)
        broken[at] = bad
        with pytest.raises(ValueError):
            moe.moe_expert_ffn_w4(*broken)


@pytest.mark.parametrize("tokens", [1, 9, 80])
def test_replayed_graphs_with_a_workspace_each(moe, tokens):
    rng = np.random.default_rng(tokens)
    h, i, e, k = 512, 256, 8, 2
    stack = Stack(moe, rng, h, i, e)
    dims = moe.MoeDims(h, i, e, k)
    x = torch.empty((tokens, h), dtype=torch.bfloat16, device="cuda")
    ids, p = route(rng, tokens, e, k, 0.3).cuda(), weights_of(rng, tokens, k).cuda()
    x.copy_(torch.from_numpy(rng.standard_normal((tokens, h)).astype(np.float32)))
    need = moe.moe_ffn_layer_w4_workspace(dims, tokens)
    outs = [torch.empty_like(x) for _ in range(3)]
    ws = [torch.empty(need, dtype=torch.uint8, device="cuda") for _ in range(3)]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")

    def call(n):
        moe.moe_ffn_layer_w4(dims, tokens, x, ids, p, *stack.packed, outs[n], status, ws[n])
    call(2)
    graphs = [torch.cuda.CUDAGraph() for _ in range(2)]
    for n, graph in enumerate(graphs):
        with torch.cuda.graph(graph):
            call(n)
    for turn in range(4):
        x.copy_(torch.from_numpy(rng.standard_normal((tokens, h)).astype(np.float32)))
        ids.copy_(route(rng, tokens, e, k, 0.3))
        for w in ws:
            w.fill_(255)  # nothing of an earlier call is needed
        for graph in graphs:
            graph.replay()
        call(2)
        torch.cuda.synchronize()
        assert torch.equal(outs[0], outs[2]) and torch.equal(outs[1], outs[2]), turn
    assert int(status.item()) == 0


@pytest.mark.parametrize("tokens", [1, 6, 70])
def test_a_layer_from_norm_to_norm(moe, tokens):
    """Norm, projection, single-token attention, projection, norm with the residual, gate, experts, residual: every step
    against its formula on the inputs that it had."""
    rng = np.random.default_rng(tokens)
    h, i, e, k = 512, 256, 8, 2
    hq, hkv, dim, page = 4, 2, 64, 16
    d = moe.MoeAttnDims(hq, hkv, dim)
    n_qkv = (hq + 2 * hkv) * dim

    def bf16(*shape):
        return torch.from_numpy(rng.standard_normal(shape).astype(np.float32)).bfloat16()
    q_in, s_in = ordinary(rng, n_qkv, h)
    q_out, s_out = ordinary(rng, h, hq * dim)
    w_in, w_out = packed(moe, q_in, s_in), packed(moe, q_out, s_out)
    stack = Stack(moe, rng, h, i, e)
    gate = bf16(e, h).cuda()
    weight = [(1 + 0.1 * bf16(h)).bfloat16() for _ in range(2)]
    stream = torch.from_numpy(rng.standard_normal((tokens, h)).astype(np.float32)).cuda()
    first = stream.clone()

    def near(got, ref, bound):
        assert ((got.double().cpu() - ref).abs() <= bound).all()
    normed = torch.empty((tokens, h), dtype=torch.bfloat16, device="cuda")
    moe.moe_add_norm(stream, weight[0].cuda(), normed)
    _, y = wo.add_norm(first.double().cpu().numpy(), None, weight[0].double().numpy(), 1e-6)
    near(normed, torch.from_numpy(y), (2.0 ** -8 + h * 2.0 ** -24) * torch.from_numpy(np.abs(y)))
    qkv = torch.empty((tokens, n_qkv), dtype=torch.bfloat16, device="cuda")
    scratch = torch.empty(max(256, *(moe.moe_linear_w4_workspace(tokens, a, b) for a, b in ((h, n_qkv), (hq * dim, h)))),
                          dtype=torch.uint8, device="cuda")
    moe.moe_linear_w4(normed, *w_in, qkv, ws=scratch)
    ref_w = values(q_in, s_in).cpu()
    ref = normed.double().cpu() @ ref_w.t()
    near(qkv, ref, 2.0 ** -8 * ref.abs() + h * 2.0 ** -22 * (normed.double().cpu().abs() @ ref_w.abs().t()))
    # the new token's own key is its only one: attention gives its value back, as the cache holds it (e4m3: 2^-4)
    rows = qkv.unflatten(1, (-1, dim))
    q, key, v = rows.split((hq, hkv, hkv), dim=1)
    cache = moe.KVCache.empty(tokens, hkv, page, dim)
    table = torch.empty((16, dim), device="cuda")
    moe.moe_rope_table(table)
    ints = torch.arange(tokens, dtype=torch.int32, device="cuda")
    buf = moe.AttentionBuffers(d, tokens, 1)
    attended = moe.run_attention(buf, q, key, v, torch.zeros_like(ints), table, ints * page, cache, dim ** -0.5,
                                 page_table=ints[:, None].contiguous(), lens=torch.ones_like(ints))
    ref = v.double().cpu().repeat_interleave(hq // hkv, 1)
    near(attended, ref, 2.0 ** -4 * ref.abs() + ref.abs().amax(-1, keepdim=True) * (2.0 ** -10 / 448 + 2.0 ** -8))
    out = torch.empty((tokens, h), dtype=torch.bfloat16, device="cuda")
    moe.moe_linear_w4(attended.flatten(1), *w_out, out, ws=scratch)
    moe.moe_add_norm(out, weight[1].cuda(), normed, residual=stream, sum_out=stream)
    z, y = wo.add_norm(out.double().cpu().numpy(), first.double().cpu().numpy(), weight[1].double().numpy(), 1e-6)
    near(stream, torch.from_numpy(z), 2.0 ** -23 * torch.from_numpy(np.abs(z)) + 2.0 ** -23)
    near(normed, torch.from_numpy(y), (2.0 ** -8 + h * 2.0 ** -24) * torch.from_numpy(np.abs(y)) + 2.0 ** -20)
    ids, p = torch.empty((tokens, k), dtype=torch.int32, device="cuda"), torch.empty((tokens, k), device="cuda")
    ws = torch.empty(max(256, moe.moe_router_workspace(tokens, h, e)), dtype=torch.uint8, device="cuda")
    moe.moe_router(normed, gate, None, ids, p, ws=ws)
    layer = moe.MoELayerBuffers(h, i, e, k, tokens, w4=True, fused=True)
    y = moe.run_layer(layer, normed, ids, p, stack.packed).view(torch.bfloat16)
    x, ids_h, p_h = normed.double().cpu(), ids.cpu(), p.double().cpu()
    ref, bound = torch.zeros((tokens, h), dtype=torch.float64), torch.zeros((tokens, h), dtype=torch.float64)
    for ex in range(e):
        t, j = (ids_h == ex).nonzero(as_tuple=True)
        rows_y, off = stack.rows(ex, x[t])
        ref.index_add_(0, t, rows_y * p_h[t, j][:, None])
        bound.index_add_(0, t, (off + 2.0 ** -21 * rows_y.abs()) * p_h[t, j][:, None])
    near(y, ref, bound + 2.0 ** -8 * (ref.abs() + bound))
    assert int(layer.dev_status.item()) == 0 and int(buf.dev_status.item()) == 0


def test_the_examples_layer_with_such_weights(moe):
    """A token by a step against the same token as its prompt's last: what differs is the cache's e4m3 rows, as with other
    weights, so the hidden states are a few percent off at most."""
    spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(ROOT, "examples", "decoder_layer.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    g = torch.Generator(device="cuda").manual_seed(3)

    def tokens(n):
        return torch.randn((n, ex.HIDDEN), generator=g, device="cuda").bfloat16()
    layer, prefix, prompts = ex.Layer(weights4=True), tokens(100), [tokens(70), tokens(33)]
    new = tokens(2)
    by_step = ex.run(layer, prefix, prompts, [new])[1]
    whole = ex.run(layer, prefix, [torch.cat([p, new[i:i + 1]]) for i, p in enumerate(prompts)], [])[0]
    by_prompt = whole[[70, 70 + 34]]
    off = ((by_step - by_prompt).float().norm() / by_prompt.float().norm()).item()
    log(f"step against prompt: {off:.4f}")
    assert off < 0.1
