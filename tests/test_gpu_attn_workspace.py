"""GPU: calls of many sizes in the workspace of the largest."""
import numpy as np
import pytest
import torch

from attention_cases import bf16, offsets
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
