"""GPU: offsets that leave their tensors are reported also where the cut leaves a sequence nothing, and what lies within
the tensors is computed."""
import numpy as np
import pytest
import torch

from attention_cases import bf16
from gpu_cases import require_gpu
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def ints(x):
    return torch.tensor([int(n) for n in x], dtype=torch.int32, device="cuda")


MANY = [0] * 100 + [40] * 51
PROMPTS = [
    # offsets of queries, of keys, those within 40 rows of each
    ([0, 40, 55], [0, 40, 40], [0, 40], [0, 40]),           # a sequence behind the last row
    ([0, 40, 40], [0, 40, 90], [0, 40], [0, 40]),           # its keys alone
    ([-5, 0, 40], [0, 0, 40], [0, 0, 40], [0, 0, 40]),      # a sequence in front of the first
    ([0, 0, 40], [-7, 0, 40], [0, 0, 40], [0, 0, 40]),      # keys of a sequence without queries
    ([40, 50], [0, 40], [40, 40], [0, 40]),                 # nothing is left
    (MANY[:-1] + [41], MANY, MANY, MANY),                   # behind sequences that a wave looks at first
    (MANY, MANY[:-1] + [10 ** 9], MANY, MANY),
    ([-2 ** 31] + MANY[1:], MANY, MANY, MANY),
]


@pytest.mark.parametrize("max_k", [0, 640, 20000])
@pytest.mark.parametrize("cu_q,cu_k,good_q,good_k", PROMPTS)
def test_prompts(moe, cu_q, cu_k, good_q, good_k, max_k):
    """max_k: whole rows, shared rows, keys in parts."""
    rng = np.random.default_rng(51)
    dims = (4, 2, 64)
    d = moe.MoeAttnDims(*dims)
    q, qv = bf16(rng.standard_normal((40, 4, 64)))
    (k, kv), (v, vv) = (bf16(rng.standard_normal((40, 2, 64))) for _ in "kv")
    ws = torch.empty(max(256, moe.moe_attn_prefill_workspace(d, len(cu_q) - 1, 40, max_k)), dtype=torch.uint8, device="cuda")
    ref, bound = ao.packed_attention(qv, kv, vv, good_q, good_k, 0.1, True)
    dead = np.isnan(ref)
    for a, b, want in ((cu_q, cu_k, moe.MOE_DEV_BAD_LENGTH), (good_q, good_k, 0)):
        out = torch.full_like(q, float("nan"))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        moe.moe_attn_prefill(d, q, k, v, ints(a), ints(b), max_k, 0.1, out, ws, dev_status=status)
        got = out.double().cpu().numpy()
        assert np.array_equal(np.isnan(got), dead)
        assert np.all(np.abs(got - ref)[~dead] <= bound[~dead])
        assert int(status.item()) == want
