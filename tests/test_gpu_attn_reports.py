"""GPU: offsets that leave their tensors are reported also where the cut leaves a sequence nothing, and what lies within
the tensors is computed."""
import numpy as np
import pytest
import torch

from attention_cases import Cache, bf16, offsets
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


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("cu,bad", [([0, 20, 40], False), ([0, 20, 45], True), ([0, 40, 41], True), ([-5, 20, 40], True),
                                    ([-30, -3, 40], True), ([0, 60, 40], True), ([20, 10, 40], True), ([50, 60, 70], True)])
def test_cache_read(moe, cu, bad, dim):
    """Token t is token t - cu[b] of its sequence, also where the sequence begins in front of the tensor."""
    rng = np.random.default_rng(52)
    cache = Cache(moe, rng, [64, 64], 2, dim, 16)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    k_out, v_out = (torch.full((40, 2, dim), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    moe.moe_cache_read(moe.MoeAttnDims(2, 2, dim), cache.dev, torch.from_numpy(cache.table).cuda(), ints(cu), k_out, v_out,
                       status)
    torch.cuda.synchronize()
    assert int(status.item()) == (moe.MOE_DEV_BAD_LENGTH if bad else 0)
    if sorted(cu) != cu:
        return
    for name, out in (("k", k_out), ("v", v_out)):
        want = np.full((40, 2, dim), 9.0, np.float32)
        for b in range(2):
            lo, hi = max(cu[b], 0), min(cu[b + 1], 40)
            if lo < hi:
                want[lo:hi] = cache.values[name][b].transpose(1, 0, 2)[lo - cu[b]:hi - cu[b]]
        assert torch.equal(out.cpu(), torch.from_numpy(want).bfloat16()), name


def test_cache_read_of_many_sequences(moe):
    """The offsets of more sequences than a workgroup has threads: the last one's."""
    lens = [1] * 600
    cache = Cache(moe, np.random.default_rng(53), lens, 1, 64, 16)
    k_out, v_out = (torch.empty((600, 1, 64), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    for last, want in ((600, 0), (601, moe.MOE_DEV_BAD_LENGTH)):
        cu = offsets(lens)
        cu[-1] = last
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        moe.moe_cache_read(moe.MoeAttnDims(1, 1, 64), cache.dev, torch.from_numpy(cache.table).cuda(), ints(cu), k_out, v_out,
                           status)
        assert int(status.item()) == want
