"""GPU: the numerators of single-token attention carry 16 bits (two bf16 each): its error within the bound that this gives,
which single bf16 numerators exceed (tests/test_oracle_attention_numerators.py)."""
import math

import numpy as np
import pytest
import torch

from attention_cases import Cache, bf16
from gpu_cases import log, require_gpu
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def worst(moe, dims, cache, lens, prefix, seed):
    rng = np.random.default_rng(seed)
    hq, hkv, dim = dims
    d, n = moe.MoeAttnDims(*dims), len(lens)
    q, qv = bf16(rng.standard_normal((n, hq, dim)))
    scale = 1 / math.sqrt(dim)
    out = torch.empty_like(q)
    ws = torch.empty(max(256, moe.moe_attn_decode_workspace(d, n, max(lens), prefix)), dtype=torch.uint8, device="cuda")
    pages = torch.from_numpy(cache.table[n, :-(-prefix // cache.page)].copy()).cuda() if prefix else None
    moe.moe_attn_decode(d, q, cache.dev, torch.from_numpy(cache.table[:n].copy()).cuda(),
                        torch.tensor(lens, dtype=torch.int32, device="cuda"), max(lens), scale, out, ws, prefix_pages=pages,
                        prefix_len=prefix)
    got, most = out.double().cpu().numpy(), 0.0
    for b in range(n):
        for h in range(hq):
            k, v = (np.concatenate([cache.values[x][i][h // (hq // hkv)] for i in ((n, b) if prefix else (b,))]) for x in "kv")
            ref, bound = ao.attention(qv[b, h][None], k, v, scale, numerators=ao.TWO_BF16_ROUNDOFF)
            most = max(most, float(np.max(np.abs(got[b, h] - ref[0]) / bound[0])))
    return most


@pytest.mark.parametrize("dims,lens,page,prefix", [
    ((8, 2, 128), [1, 2, 3, 17, 40, 300, 129], 16, 0),         # one launch
    ((16, 4, 64), [2, 33, 64, 250], 32, 100),
    ((40, 2, 64), [3, 90], 16, 0),                             # two blocks of columns
    ((8, 2, 128), [3, 40, 1500], 64, 0),                       # pieces and a join
    ((8, 1, 64), [5, 20, 60, 1, 9], 16, 1300),                 # two blocks of columns on the prefix
    ((34, 1, 128), [40, 1100], 32, 0)])
def test_steps(moe, dims, lens, page, prefix):
    cache = Cache(moe, np.random.default_rng(101), lens + ([prefix] if prefix else []), dims[1], dims[2], page)
    ratio = worst(moe, dims, cache, lens, prefix, 102)
    log(f"{dims} {lens} prefix {prefix}: worst error {ratio:.3f} of its bound")
    assert ratio <= 1.0


@pytest.mark.parametrize("n", [60, 2000])
def test_value_rows_of_many_sizes(moe, n):
    """Rows from 2^-40 to 2^0 of the largest, whose scales are in the numerators."""
    rng = np.random.default_rng(103)
    cache = Cache(moe, rng, [n], 1, 64, 16)
    factor = (2.0 ** -rng.integers(0, 41, n)).astype(np.float32)
    for t in range(n):
        cache.scales["v"][cache.table[0, t // 16], 0, t % 16] *= factor[t]
    cache.values["v"][0] = cache.values["v"][0] * factor[None, :, None]
    cache.dev.v_scale.copy_(torch.from_numpy(cache.scales["v"]))
    ratio = worst(moe, (4, 1, 64), cache, [n], 0, 104)
    log(f"{n} value rows of many sizes: worst error {ratio:.3f} of its bound")
    assert ratio <= 1.0
