"""GPU: scores at the far ends of what fp32 holds."""
import numpy as np
import pytest
import torch

from attention_cases import Cache, bf16, offsets
from gpu_cases import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def weights(n, dim, size):
    """Key factors: all equal, and one that gives the largest score by far (scores are negative)."""
    flat, peak = np.ones(n), np.full(n, 2.0)
    peak[n // 3] = 1.0
    return ((flat * size, None), (peak * size, n // 3))


# 64 or 128 products of 2^60 and 2^44 .. 2^58, times 2^-3 (and log2 e): the scores lie between -2^107 and -2^123
@pytest.mark.parametrize("power", [44, 58])
@pytest.mark.parametrize("max_k", [0, 640, 20000])
@pytest.mark.parametrize("dim", [64, 128])
def test_prompts_of_hugely_negative_scores(moe, dim, max_k, power):
    """Equal scores give the values' mean (numerators of 1, sums of n fp32 terms and one rounding to bf16), one that is far
    larger than the others its own value, however low they all lie."""
    rng = np.random.default_rng(81)
    n = 150
    d = moe.MoeAttnDims(4, 2, dim)
    q, _ = bf16(np.full((7, 4, dim), -2.0 ** 60))
    v, vv = bf16(rng.standard_normal((n, 2, dim)))
    ws = torch.empty(max(256, moe.moe_attn_prefill_workspace(d, 1, 7, max_k)), dtype=torch.uint8, device="cuda")
    for factor, top in weights(n, dim, 2.0 ** power / (dim // 64)):
        k, _ = bf16(np.broadcast_to(factor[:, None, None], (n, 2, dim)).copy())
        out = torch.empty_like(q)
        moe.moe_attn_prefill(d, q, k, v, *(torch.from_numpy(offsets([x])).cuda() for x in (7, n)), max_k, 0.125, out, ws,
                             causal=False)
        got = out.double().cpu().numpy()
        ref = vv.mean(0) if top is None else vv[top]
        tol = 2.0 ** -8 * np.abs(ref) + n * 2.0 ** -24 * np.abs(vv).mean(0) if top is None else 0.0 * ref
        assert np.all(np.abs(got - np.repeat(ref, 2, 0)) <= np.repeat(tol, 2, 0)), (top, power)


@pytest.mark.parametrize("power", [44, 58])
@pytest.mark.parametrize("n,prefix", [(100, 0), (100, 50), (3000, 0), (30, 2500)])
def test_steps_of_hugely_negative_scores(moe, n, prefix, power):
    """As for prompts; the values have 16 bits as numerators, so that the mean is off by 2^-16 of their size more."""
    rng = np.random.default_rng(82)
    dim = 64
    d = moe.MoeAttnDims(4, 2, dim)
    cache = Cache(moe, rng, [n] + ([prefix] if prefix else []), 2, dim, 16)
    q, _ = bf16(np.full((1, 4, dim), -2.0 ** 60))
    values = [np.concatenate([cache.values["v"][b][h] for b in ((1, 0) if prefix else (0,))]).astype(np.float64)
              for h in range(2)]
    total = n + prefix
    pages = torch.from_numpy(cache.table[1, :-(-prefix // 16)].copy()).cuda() if prefix else None
    ws = torch.empty(max(256, moe.moe_attn_decode_workspace(d, 1, n, prefix)), dtype=torch.uint8, device="cuda")
    cache.dev.k.fill_(0x38)  # 1.0
    for factor, top in weights(total, dim, 2.0 ** power):
        scales = np.full(cache.scales["k"].shape, np.nan, np.float32)
        for b, first, m in ((1, 0, prefix), (0, prefix, n)) if prefix else ((0, 0, n),):
            for t in range(m):
                scales[cache.table[b, t // 16], :, t % 16] = factor[first + t]
        cache.dev.k_scale.copy_(torch.from_numpy(scales))
        out = torch.empty_like(q)
        moe.moe_attn_decode(d, q, cache.dev, torch.from_numpy(cache.table[:1].copy()).cuda(),
                            torch.tensor([n], dtype=torch.int32, device="cuda"), n, 0.125, out, ws, prefix_pages=pages,
                            prefix_len=prefix)
        got = out[0].double().cpu().numpy()
        for h in range(4):
            x = values[h // 2]
            ref = x.mean(0) if top is None else x[top]
            tol = 2.0 ** -8 * np.abs(ref) + (2.0 ** -16 + total * 2.0 ** -24) * np.abs(x).mean(0) if top is None else \
                2.0 ** -8 * np.abs(ref)
            assert np.all(np.abs(got[h] - ref) <= tol), (top, power, h)
