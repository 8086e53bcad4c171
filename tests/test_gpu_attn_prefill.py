"""GPU: attention over packed prompts against the fp64 oracle, element by element, within the bound that the
definition's roundings give (oracle/attention_oracle.py)."""
import math

import numpy as np
import pytest
import torch

from attention_cases import bf16, offsets
from gpu_cases import log, require_gpu
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def run(moe, dims, q, k, v, cu_q, cu_k, max_k, scale, causal=True, status=None):
    d = moe.MoeAttnDims(*dims)
    out = torch.full((q.shape[0], dims[0], dims[2]), float("nan"), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(256, moe.moe_attn_prefill_workspace(d, len(cu_q) - 1, q.shape[0], max_k)), dtype=torch.uint8,
                     device="cuda").fill_(0xFF)
    moe.moe_attn_prefill(d, q, k, v, torch.from_numpy(cu_q).cuda(), torch.from_numpy(cu_k).cuda(), max_k, scale, out, ws,
                         causal=causal, dev_status=status)
    torch.cuda.synchronize()
    return out


def check(got, ref, bound, what):
    got = got.double().cpu().numpy()
    dead = np.isnan(ref)
    assert np.array_equal(np.isnan(got), dead), f"{what}: rows written that are in no sequence, or NaN in those that are"
    worst = float(np.max(np.where(dead, 0.0, np.abs(got - ref)) / np.where(dead, 1.0, bound))) if ref.size else 0.0
    log(f"{what}: worst error {worst:.3f} of its bound")
    assert worst <= 1.0


CASES = [
    # heads, lengths of queries, keys more than queries per sequence, causal
    ((4, 4, 64), [1], 0, True),
    ((8, 2, 128), [17], 0, True),
    ((8, 2, 128), [0, 5, 0, 64, 65, 1, 0], 0, True),
    ((4, 1, 64), [31, 32, 33, 63, 127, 128, 129], 0, True),
    ((14, 2, 128), [257, 3], 0, True),                 # a group of 7: rows of a tile start inside a token
    ((16, 1, 128), [40, 9], 0, True),
    ((6, 6, 128), [200], 0, True),
    ((8, 2, 128), [3, 70], 300, True),                 # a chunk behind cached keys
    ((8, 2, 64), [1, 1, 1], 777, True),
    ((8, 2, 128), [50, 200], -37, True),               # fewer keys than queries: the first see none
    ((8, 2, 64), [64, 10], -64, True),                 # no keys at all
    ((8, 2, 128), [77, 130], 0, False),
    ((4, 2, 64), [5, 66], 129, False),
    ((8, 2, 128), [20], -20, False),
]


@pytest.mark.parametrize("dims,lens,more,causal", CASES)
def test_packed_prompts(moe, dims, lens, more, causal):
    rng = np.random.default_rng(5)
    hq, hkv, dim = dims
    keys = [max(0, n + more) if n else 0 for n in lens]
    cu_q, cu_k = offsets(lens), offsets(keys)
    q, qv = bf16(rng.standard_normal((cu_q[-1], hq, dim)))
    k, kv = bf16(rng.standard_normal((cu_k[-1], hkv, dim)) * np.exp(rng.standard_normal((1, 1, dim))))
    v, vv = bf16(rng.standard_normal((cu_k[-1], hkv, dim)))
    scale = 1 / math.sqrt(dim)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(moe, dims, q, k, v, cu_q, cu_k, max(keys), scale, causal, status)
    ref, bound = ao.packed_attention(qv, kv, vv, cu_q, cu_k, scale, causal)
    check(got, ref, bound, f"{dims} {lens} {more:+d} causal={causal}")
    assert int(status.item()) == 0


@pytest.mark.parametrize("dims", [(8, 2, 128), (8, 4, 64)])
def test_strided_views_and_rows_between_sequences(moe, dims):
    """q, k, v are views of one packed projection with padding columns; rows in front of the first sequence and behind the
    last hold NaN and are neither read into a result nor written."""
    rng = np.random.default_rng(6)
    hq, hkv, dim = dims
    lens, pad = [70, 1, 33], 5
    cu = offsets(lens) + pad
    cu[0] = pad
    rows = int(cu[-1]) + pad
    width = (hq + 2 * hkv) * dim + 24
    x = rng.standard_normal((rows, width)).astype(np.float32)
    x[:pad] = np.nan
    x[-pad:] = np.nan
    packed, val = bf16(x)

    def view(t, lo, n):
        return t[:, lo * dim:(lo + n) * dim].unflatten(1, (n, dim)) if isinstance(t, torch.Tensor) else \
            t[:, lo * dim:(lo + n) * dim].reshape(rows, n, dim)
    q, k, v = (view(packed, lo, n) for lo, n in ((0, hq), (hq, hkv), (hq + hkv, hkv)))
    qv, kv, vv = (view(val, lo, n) for lo, n in ((0, hq), (hq, hkv), (hq + hkv, hkv)))
    cu = cu.astype(np.int32)
    got = run(moe, dims, q, k, v, cu, cu, 70, 0.11)
    ref, bound = ao.packed_attention(qv, kv, vv, cu, cu, 0.11, True)
    check(got, ref, bound, f"strided {dims}")


@pytest.mark.parametrize("size", [30.0, 0.0])
def test_peaked_and_flat_scores(moe, size):
    """Scores of hundreds (the running maximum grows many times) and all equal ones (a mean of the values)."""
    rng = np.random.default_rng(7)
    dims, lens = (4, 2, 128), [300]
    cu = offsets(lens)
    q, qv = bf16(rng.standard_normal((300, 4, 128)) * size)
    ramp = np.linspace(0.1, 3.0, 300)[:, None, None]
    k, kv = bf16(rng.standard_normal((300, 2, 128)) * ramp)
    v, vv = bf16(rng.standard_normal((300, 2, 128)) + 1.0)
    got = run(moe, dims, q, k, v, cu, cu, 300, 1 / math.sqrt(128))
    ref, bound = ao.packed_attention(qv, kv, vv, cu, cu, 1 / math.sqrt(128), True)
    check(got, ref, bound, f"scores x {size}")


@pytest.mark.parametrize("dims,n,past", [((8, 2, 128), 2500, 0), ((8, 1, 64), 130, 9000), ((4, 4, 128), 1, 5000)])
def test_long_axes(moe, dims, n, past):
    """Long prompts and few rows over many keys: every row of two heads."""
    rng = np.random.default_rng(8)
    hq, hkv, dim = dims
    cu_q, cu_k = offsets([n]), offsets([n + past])
    q, qv = bf16(rng.standard_normal((n, hq, dim)))
    k, kv = bf16(rng.standard_normal((n + past, hkv, dim)))
    v, vv = bf16(rng.standard_normal((n + past, hkv, dim)))
    scale = 1 / math.sqrt(dim)
    got = run(moe, dims, q, k, v, cu_q, cu_k, n + past, scale)
    heads = [0, hq - 1]
    ref, bound = ao.packed_attention(qv, kv, vv, cu_q, cu_k, scale, True, heads)
    check(got[:, heads], ref[:, heads], bound[:, heads], f"long {dims} {n}+{past}")


def test_the_split_does_not_depend_on_a_wrong_longest_length(moe):
    """max_k decides how the work is split, never what is computed: too small and too large ones give the result."""
    rng = np.random.default_rng(9)
    dims, lens, keys = (4, 1, 128), [3, 20], [3000, 41]
    cu_q, cu_k = offsets(lens), offsets(keys)
    q, qv = bf16(rng.standard_normal((23, 4, 128)))
    k, kv = bf16(rng.standard_normal((cu_k[-1], 1, 128)))
    v, vv = bf16(rng.standard_normal((cu_k[-1], 1, 128)))
    ref, bound = ao.packed_attention(qv, kv, vv, cu_q, cu_k, 0.09, True)
    for max_k in (0, 41, 3000, 100000):
        check(run(moe, dims, q, k, v, cu_q, cu_k, max_k, 0.09), ref, bound, f"max_k={max_k}")


def test_same_inputs_give_the_same_bits(moe):
    rng = np.random.default_rng(10)
    cu = offsets([500, 77])
    q, k, v = (bf16(rng.standard_normal((577, h, 128)))[0] for h in (8, 2, 2))
    first = run(moe, (8, 2, 128), q, k, v, cu, cu, 500, 0.1)
    again = run(moe, (8, 2, 128), q, k, v, cu, cu, 500, 0.1)
    assert torch.equal(first.view(torch.int16), again.view(torch.int16))


def test_offsets_that_leave_the_tensors_are_cut(moe):
    rng = np.random.default_rng(11)
    q, qv = bf16(rng.standard_normal((40, 4, 64)))
    k, kv = bf16(rng.standard_normal((40, 4, 64)))
    v, vv = bf16(rng.standard_normal((40, 4, 64)))
    good, bad = np.array([0, 10, 40], np.int32), np.array([0, 10, 55], np.int32)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(moe, (4, 4, 64), q, k, v, bad, bad, 55, 0.1, True, status)
    ref, bound = ao.packed_attention(qv, kv, vv, good, good, 0.1, True)
    check(got, ref, bound, "cut offsets")
    assert int(status.item()) == moe.MOE_DEV_BAD_LENGTH


def test_more_sequences_than_a_wave_has_lanes(moe):
    """The row tile's sequence is looked up 64 at a time."""
    rng = np.random.default_rng(12)
    lens = [int(n) for n in rng.integers(0, 40, 150)]
    keys = [n + int(m) if n else 0 for n, m in zip(lens, rng.integers(0, 30, 150))]
    dims = (4, 2, 64)
    cu_q, cu_k = offsets(lens), offsets(keys)
    q, qv = bf16(rng.standard_normal((cu_q[-1], 4, 64)))
    k, kv = bf16(rng.standard_normal((cu_k[-1], 2, 64)))
    v, vv = bf16(rng.standard_normal((cu_k[-1], 2, 64)))
    got = run(moe, dims, q, k, v, cu_q, cu_k, max(keys), 0.1)
    ref, bound = ao.packed_attention(qv, kv, vv, cu_q, cu_k, 0.1, True)
    check(got, ref, bound, "150 sequences")


@pytest.mark.parametrize("dims", [(1024, 1, 64), (96, 3, 128)])
def test_wide_groups(moe, dims):
    """Groups of more heads than a tile has rows, and of 32 heads."""
    rng = np.random.default_rng(13)
    hq, hkv, dim = dims
    cu = offsets([7, 3])
    q, qv = bf16(rng.standard_normal((10, hq, dim)))
    k, kv = bf16(rng.standard_normal((10, hkv, dim)))
    v, vv = bf16(rng.standard_normal((10, hkv, dim)))
    got = run(moe, dims, q, k, v, cu, cu, 7, 0.1)
    ref, bound = ao.packed_attention(qv, kv, vv, cu, cu, 0.1, True)
    check(got, ref, bound, f"wide group {dims}")


def test_values_that_are_all_one_stay_one(moe):
    """Numerators and denominators are the same rounded numbers, so a mean of ones is exactly one."""
    rng = np.random.default_rng(14)
    cu = offsets([333])
    q, k = (bf16(rng.standard_normal((333, h, 128)) * 3)[0] for h in (8, 2))
    got = run(moe, (8, 2, 128), q, k, torch.ones_like(k), cu, cu, 333, 0.1)
    assert bool((got == 1).all())


@pytest.mark.parametrize("past", [0, 6000])
def test_replays_from_a_hip_graph(moe, past):
    """A call (with `past`, cut into parts and joined) captured once and replayed on new inputs, eager work in between."""
    d = moe.MoeAttnDims(8, 2, 128)
    q = torch.empty((90, 8, 128), dtype=torch.bfloat16, device="cuda")
    k, v = (torch.empty((90 + 2 * past, 2, 128), dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cu_q, cu_k = (torch.tensor(x, dtype=torch.int32, device="cuda") for x in ([0, 50, 90], [0, 50 + past, 90 + 2 * past]))
    ws = torch.empty(max(256, moe.moe_attn_prefill_workspace(d, 2, 90, 50 + past)), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)

    def call(ws_, out_):
        moe.moe_attn_prefill(d, q, k, v, cu_q, cu_k, 50 + past, 0.1, out_, ws_)
    for t in (q, k, v):
        t.normal_()
    call(ws, out)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(ws, out)
    torch.cuda.synchronize()
    for _ in range(3):
        for t in (q, k, v):
            t.normal_()
        ref = torch.empty_like(q)
        call(torch.empty_like(ws), ref)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), ref.view(torch.int16))


@pytest.mark.parametrize("max_k", [0, 640, 20000])
@pytest.mark.parametrize("dims,lens,more,causal", CASES)
def test_every_way_to_share_the_work(moe, dims, lens, more, causal, max_k):
    """The announced longest length alone chooses between tiles of whole and of shared rows, and cuts keys into parts."""
    rng = np.random.default_rng(35)
    hq, hkv, dim = dims
    keys = [max(0, n + more) if n else 0 for n in lens]
    cu_q, cu_k = offsets(lens), offsets(keys)
    q, qv = bf16(rng.standard_normal((cu_q[-1], hq, dim)))
    k, kv = bf16(rng.standard_normal((cu_k[-1], hkv, dim)))
    v, vv = bf16(rng.standard_normal((cu_k[-1], hkv, dim)))
    scale = 1 / math.sqrt(dim)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(moe, dims, q, k, v, cu_q, cu_k, max_k, scale, causal, status)
    ref, bound = ao.packed_attention(qv, kv, vv, cu_q, cu_k, scale, causal)
    check(got, ref, bound, f"{dims} {lens} {more:+d} causal={causal} max_k={max_k}")
    assert int(status.item()) == 0


@pytest.mark.parametrize("dim", [64, 128])
@pytest.mark.parametrize("keys", [1, 63, 64, 65, 128, 129, 191, 192, 193, 256, 257, 320, 321, 449, 513])
def test_key_tiles_of_both_halves(moe, dim, keys):
    """Odd and even numbers of key tiles, the last one full or not: rows shared by two halves of the waves."""
    rng = np.random.default_rng(keys)
    cu_q, cu_k = offsets([5, 150]), offsets([keys, keys])
    q, qv = bf16(rng.standard_normal((155, 4, dim)))
    k, kv = bf16(rng.standard_normal((2 * keys, 2, dim)))
    v, vv = bf16(rng.standard_normal((2 * keys, 2, dim)))
    for causal in (False, True):
        got = run(moe, (4, 2, dim), q, k, v, cu_q, cu_k, 640, 0.1, causal)
        ref, bound = ao.packed_attention(qv, kv, vv, cu_q, cu_k, 0.1, causal)
        check(got, ref, bound, f"{keys} keys of {dim} causal={causal}")


@pytest.mark.parametrize("max_k", [0, 640, 20000])
@pytest.mark.parametrize("dims,lens,past", [((8, 2, 128), [300], 0), ((4, 4, 64), [70, 200], 0), ((4, 1, 128), [37, 5], 150)])
def test_hidden_keys_and_values_may_hold_anything(moe, dims, lens, past, max_k):
    """Infinite and NaN elements of keys and values stay with the rows that see them; a value's with its column."""
    rng = np.random.default_rng(36)
    hq, hkv, dim = dims
    keys = [n + past for n in lens]
    cu_q, cu_k = offsets(lens), offsets(keys)
    q, qv = bf16(rng.standard_normal((cu_q[-1], hq, dim)))
    k, kv = bf16(rng.standard_normal((cu_k[-1], hkv, dim)))
    v, vv = bf16(rng.standard_normal((cu_k[-1], hkv, dim)))
    scale = 1 / math.sqrt(dim)
    clean_v = vv.copy()
    touched = np.zeros(qv.shape, bool)
    for b, n in enumerate(lens):
        c, a = cu_k[b], cu_q[b]
        # values: an element of a middle token and of the last one
        for j, d, x in ((past + n // 2, 3, np.inf), (past + n - 1, dim - 1, np.nan), (past + n - 2, 40, -np.inf)):
            v[c + j, :, d] = x
            clean_v[c + j, :, d] = 0.0
            touched[a + j - past:cu_q[b + 1], :, d] = True
        # a whole key of the last token: only its own row sees it
        k[c + past + n - 1] = np.nan
        touched[cu_q[b + 1] - 1] = True
    kv = np.nan_to_num(k.double().cpu().numpy())
    got = run(moe, dims, q, k, v, cu_q, cu_k, max_k, scale).double().cpu().numpy()
    ref, bound = ao.packed_attention(qv, kv, clean_v, cu_q, cu_k, scale, True)
    assert np.array_equal(np.isfinite(got), ~touched)
    worst = float(np.max(np.abs(got - ref)[~touched] / np.maximum(bound, 1e-30)[~touched]))
    log(f"{dims} {lens} behind {past}, max_k {max_k}: worst error {worst:.3f} of its bound")
    assert worst <= 1.0
