"""GPU: calls of many sizes in the workspace of the largest."""
import numpy as np
import pytest
import torch

from attention_cases import Cache, bf16, offsets
from gpu_cases import require_gpu
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


def test_chunks_of_a_prompt_in_one_workspace():
    """Full chunks and an odd last one in the workspace of the largest call: 32 heads, the keys in parts for some of them."""
    moe = require_gpu()
    rng = np.random.default_rng(63)
    dims, total = (32, 8, 128), 8701
    d = moe.MoeAttnDims(*dims)
    ws = torch.empty(max(256, moe.moe_attn_prefill_workspace(d, 1, 4096, total)), dtype=torch.uint8, device="cuda")
    k, kv = bf16(rng.standard_normal((total, 8, 128)))
    v, vv = bf16(rng.standard_normal((total, 8, 128)))
    for past, n in ((0, 4096), (4096, 2048), (6144, 2048), (8192, 509), (8700, 1)):
        q, qv = bf16(rng.standard_normal((n, 32, 128)))
        out = torch.empty_like(q)
        cu_q, cu_k = offsets([n]), offsets([past + n])
        moe.moe_attn_prefill(d, q, k[:past + n], v[:past + n], torch.from_numpy(cu_q).cuda(), torch.from_numpy(cu_k).cuda(),
                             past + n, 0.088, out, ws)
        rows = np.unique(np.linspace(0, n - 1, 9).astype(int))
        for h in (0, 31):
            see = np.arange(past + n)[None] <= (past + rows)[:, None]
            ref, bound = ao.attention(qv[rows, h], kv[:past + n, h // 4], vv[:past + n, h // 4], 0.088, see)
            assert np.all(np.abs(out[torch.from_numpy(rows).cuda(), h].double().cpu().numpy() - ref) <= bound), (past, n, h)


def test_a_batch_that_shrinks_in_one_workspace():
    moe = require_gpu()
    rng = np.random.default_rng(64)
    d = moe.MoeAttnDims(32, 8, 128)
    lens = [1024, 700] + [int(n) for n in rng.integers(1, 1024, 46)]
    cache = Cache(moe, rng, lens, 8, 128, 64)
    ws = torch.empty(max(256, moe.moe_attn_decode_workspace(d, 48, 1024, 0)), dtype=torch.uint8, device="cuda")
    for n in (48, 32, 16, 8, 2, 1):
        q, qv = bf16(rng.standard_normal((n, 32, 128)))
        out = torch.empty_like(q)
        moe.moe_attn_decode(d, q, cache.dev, torch.from_numpy(cache.table[:n].copy()).cuda(),
                            torch.tensor(lens[:n], dtype=torch.int32, device="cuda"), 1024, 0.088, out, ws)
        for b in (0, n - 1):
            for h in (0, 31):
                ref, bound = ao.attention(qv[b, h][None], cache.values["k"][b][h // 4], cache.values["v"][b][h // 4], 0.088)
                assert np.all(np.abs(out[b, h].double().cpu().numpy() - ref[0]) <= bound[0]), (n, b, h)
