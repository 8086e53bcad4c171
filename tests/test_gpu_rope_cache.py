"""GPU: rotary positions, the quantized cache's write and its read against the oracle, bit for bit."""
import numpy as np
import pytest
import torch

import oracle
from attention_cases import Cache, bf16, offsets
from gpu_cases import log, require_gpu
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def bits(t):
    return t.contiguous().view(torch.int16).cpu().numpy().view(np.uint16)


@pytest.mark.parametrize("kind,kw", [
    ("PLAIN", {}), ("LINEAR", {"factor": 8.0}),
    ("BY_PARTS", {"factor": 40.0, "original_len": 4096.0, "slow_turns": 1.0, "fast_turns": 32.0, "magnitude": 1.37})])
@pytest.mark.parametrize("rot,base", [(128, 10000.0), (48, 500000.0)])
def test_table(moe, kind, kw, rot, base):
    """Within one fp32 ulp of values of up to `magnitude`: both sides round an fp64 cosine once, and fp64 library functions
    and powers differ by a few fp64 ulps, at angles up to n_pos by n_pos * 2^-50."""
    n = 200_001
    table = torch.full((n, rot), float("nan"), device="cuda")
    moe.moe_rope_table(table, base=base, scaling=getattr(moe, f"MOE_ROPE_{kind}"), **kw)
    torch.cuda.synchronize()
    mag = kw.pop("magnitude", 1.0)
    ref = ao.rope_table(n, ao.rope_frequencies(rot, base, kind.lower(), **kw), mag)
    err = np.abs(table.cpu().numpy().astype(np.float64) - ref)
    log(f"table {kind} {rot}: {err.max():.3e}")
    assert err.max() <= mag * (2.0 ** -23 + n * 2.0 ** -50)


def inputs(rng, T, hq, hkv, dim, packed):
    """q, k, v as device tensors (views of one projection with 8 spare columns, or contiguous) and as fp32 values."""
    x = rng.standard_normal((T, (hq + 2 * hkv) * dim + 8)).astype(np.float32)
    x *= np.exp(2 * rng.standard_normal((T, 1)))
    dev, val = bf16(x)
    out = []
    for lo, n in ((0, hq), (hq, hkv), (hq + hkv, hkv)):
        d = dev[:, lo * dim:(lo + n) * dim].unflatten(1, (n, dim))
        out.append((d if packed else d.contiguous(), val[:, lo * dim:(lo + n) * dim].reshape(T, n, dim).astype(np.float32)))
    return out


CASES = [
    # tokens, heads, rotated, interleaved, packed, page, keep k
    (1, (4, 4, 64), 64, False, False, 16, False),
    (1, (32, 8, 128), 128, True, True, 64, True),
    (17, (8, 2, 128), 64, False, True, 16, True),
    (33, (14, 2, 128), 32, True, True, 32, False),
    (50, (6, 6, 64), 16, False, False, 128, True),
    (200, (16, 1, 128), 112, False, True, 16, True),
    (77, (5, 1, 64), 48, True, False, 64, True),
    (5000, (8, 2, 128), 128, False, True, 64, True),
    (5003, (8, 4, 64), 32, True, True, 16, False),
]


@pytest.mark.parametrize("T,dims,rot,inter,packed,page,keep", CASES)
def test_rope_cache(moe, T, dims, rot, inter, packed, page, keep):
    rng = np.random.default_rng(31)
    hq, hkv, dim = dims
    (q, qv), (k, kv), (v, vv) = inputs(rng, T, hq, hkv, dim, packed)
    n_pos = 9000
    table = ao.rope_table(n_pos, ao.rope_frequencies(rot, 10000.0))
    pos = rng.integers(0, n_pos, T).astype(np.int32)
    n_pages = -(-T // page) + 2
    slots = rng.permutation(n_pages * page)[:T].astype(np.int32)
    skip = rng.random(T) < 0.1 if T > 20 else np.zeros(T, bool)
    slots[skip] = -1 - rng.integers(0, 100, int(skip.sum()))
    cache = moe.KVCache.empty(n_pages, hkv, page, dim)
    for t in (cache.k, cache.v):
        t.fill_(0xAB)
    for t in (cache.k_scale, cache.v_scale):
        t.fill_(-7.0)
    q_out = torch.empty((T, hq, dim), dtype=torch.bfloat16, device="cuda")
    k_out = torch.empty((T, hkv, dim), dtype=torch.bfloat16, device="cuda") if keep else None
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    layout = moe.MOE_ROPE_INTERLEAVED if inter else moe.MOE_ROPE_HALF
    d = moe.MoeAttnDims(*dims)
    moe.moe_rope_cache(d, q, k, v, torch.from_numpy(pos).cuda(), torch.from_numpy(table).cuda(), layout,
                       torch.from_numpy(slots).cuda(), cache, q_out, k_out, status)
    torch.cuda.synchronize()
    assert int(status.item()) == 0
    rq, rk = ao.rotate(qv, table[pos], inter), ao.rotate(kv, table[pos], inter)
    assert np.array_equal(bits(q_out), oracle.f32_to_bf16(rq))
    if keep:
        assert np.array_equal(bits(k_out), oracle.f32_to_bf16(rk))
    live = np.flatnonzero(~skip)
    for name, x in (("k", rk), ("v", vv)):
        want = np.full((n_pages, hkv, page, dim), 0xAB, np.uint8)
        scale = np.full((n_pages, hkv, page), -7.0, np.float32)
        c, s = ao.quantize_head_rows(x)
        want[slots[live] // page, :, slots[live] % page] = c[live]
        scale[slots[live] // page, :, slots[live] % page] = s[live]
        assert np.array_equal(getattr(cache, name).cpu().numpy(), want), name
        assert np.array_equal(getattr(cache, name + "_scale").cpu().numpy(), scale), name
    # moe_rope alone gives the same rotated rows, also in place
    q2, k2 = q.contiguous().clone(), k.contiguous().clone()
    moe.moe_rope(d, q2, k2, torch.from_numpy(pos).cuda(), torch.from_numpy(table).cuda(), layout, q2, k2)
    only = torch.empty_like(k2)
    moe.moe_rope(d, None, k, torch.from_numpy(pos).cuda(), torch.from_numpy(table).cuda(), layout, None, only)
    torch.cuda.synchronize()
    assert np.array_equal(bits(q2), oracle.f32_to_bf16(rq)) and np.array_equal(bits(k2), oracle.f32_to_bf16(rk))
    assert torch.equal(only, k2)


def test_rows_of_zeros_and_of_extreme_sizes(moe):
    """Zero heads (scale 0, signed zero codes), and rows from fp32 subnormals to the largest bf16."""
    rng = np.random.default_rng(32)
    T, dim = 40, 64
    x = rng.standard_normal((T, 1, dim)).astype(np.float32)
    x *= np.float32(2.0) ** np.linspace(-140, 100, T).astype(np.int32)[:, None, None]
    x[3], x[4], x[5, 0, 1:] = 0.0, -0.0, 0.0
    dev, val = bf16(x)
    table = torch.zeros((4, 16), device="cuda")
    moe.moe_rope_table(table)
    cache = moe.KVCache.empty(3, 1, 16, dim)
    out = torch.empty_like(dev)
    moe.moe_rope_cache(moe.MoeAttnDims(1, 1, dim), dev, dev, dev, torch.zeros(T, dtype=torch.int32, device="cuda"), table,
                       moe.MOE_ROPE_HALF, torch.arange(T, dtype=torch.int32, device="cuda"), cache, out)
    torch.cuda.synchronize()
    c, s = ao.quantize_head_rows(val.astype(np.float32))
    # position 0 turns by nothing: x * 1 - y * 0 and x * 1 + y * 0 keep the value, but not the sign of a zero
    for codes, scales, exact in ((cache.v, cache.v_scale, True), (cache.k, cache.k_scale, False)):
        got = codes.cpu().numpy().reshape(48, dim)[:T]
        assert np.array_equal(scales.cpu().numpy().reshape(48)[:T], s[:, 0])
        if exact:
            assert np.array_equal(got, c[:, 0])
        else:
            assert np.array_equal(oracle.e4m3_decode(got), oracle.e4m3_decode(c[:, 0]))


def test_bad_positions_and_slots_are_reported(moe):
    rng = np.random.default_rng(33)
    dims = (4, 2, 64)
    (q, qv), (k, kv), (v, vv) = inputs(rng, 3, *dims, False)
    table = ao.rope_table(10, ao.rope_frequencies(64, 10000.0))
    dt = torch.from_numpy(table).cuda()
    d = moe.MoeAttnDims(*dims)

    def call(pos, slots):
        cache = moe.KVCache.empty(2, 2, 16, 64)
        cache.k.fill_(1)
        out = torch.empty_like(q)
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        moe.moe_rope_cache(d, q, k, v, torch.tensor(pos, dtype=torch.int32, device="cuda"), dt, moe.MOE_ROPE_HALF,
                           torch.tensor(slots, dtype=torch.int32, device="cuda"), cache, out, None, status)
        torch.cuda.synchronize()
        return int(status.item()), out, cache
    for p in (-1, 10, 2 ** 31 - 1):
        st, out, _ = call([9, p, 0], [0, 1, 2])
        assert st == moe.MOE_DEV_BAD_POSITION
        want = oracle.f32_to_bf16(ao.rotate(qv, table[[9, 0, 0]], False))
        assert np.array_equal(bits(out)[[0, 2]], want[[0, 2]])
    for s in (32, 2 ** 31 - 1):
        st, out, cache = call([1, 2, 3], [31, s, 0])
        assert st == moe.MOE_DEV_BAD_SLOT
        codes = cache.k.cpu().numpy()
        want, _ = ao.quantize_head_rows(ao.rotate(kv, table[[1, 2, 3]], False))
        assert np.array_equal(codes[1, :, 15], want[0]) and np.array_equal(codes[0, :, 0], want[2])
        codes[1, :, 15] = codes[0, :, 0] = 1
        assert (codes == 1).all()


@pytest.mark.parametrize("lens,heads,dim,page", [
    ([1], 1, 64, 16), ([0, 17, 0, 300, 1, 64], 8, 128, 64), ([33, 5], 3, 64, 32), ([700, 650, 0], 2, 128, 16),
    ([40] * 70, 2, 64, 16)])
def test_cache_read(moe, lens, heads, dim, page):
    rng = np.random.default_rng(34)
    cache = Cache(moe, rng, lens, heads, dim, page)
    d = moe.MoeAttnDims(heads, heads, dim)
    lead, cu = 3, offsets(lens)
    total = int(cu[-1])
    for shift in (0, lead):   # rows in front of the first sequence and behind the last stay as they are
        k_out, v_out = (torch.full((total + 2 * shift, heads, dim), 9.0, dtype=torch.bfloat16, device="cuda")
                        for _ in range(2))
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        moe.moe_cache_read(d, cache.dev, torch.from_numpy(cache.table).cuda(), torch.from_numpy(cu + shift).cuda(), k_out,
                           v_out, status)
        torch.cuda.synchronize()
        assert int(status.item()) == 0
        for name, t in (("k", k_out), ("v", v_out)):
            want = np.concatenate([x.transpose(1, 0, 2) for x in cache.values[name]])
            got = bits(t)
            assert np.array_equal(got[shift:shift + total], oracle.f32_to_bf16(want)), name
            edge = np.concatenate([got[:shift], got[shift + total:]])
            assert (edge == 0x4110).all()


def test_cache_read_reports_bad_pages_and_lengths(moe):
    rng = np.random.default_rng(35)
    cache = Cache(moe, rng, [40, 20], 2, 64, 16)
    d = moe.MoeAttnDims(2, 2, 64)
    cu = torch.tensor([0, 60, 80], dtype=torch.int32, device="cuda")   # the first row of the table holds 48 tokens
    k_out, v_out = (torch.full((80, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in range(2))
    cache.table[0, 2] = cache.table[1, 0]
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    moe.moe_cache_read(d, cache.dev, torch.from_numpy(cache.table).cuda(), cu, k_out, v_out, status)
    torch.cuda.synchronize()
    assert int(status.item()) == moe.MOE_DEV_BAD_LENGTH
    assert not k_out[48:60].any() and not v_out[48:60].any()
    want = oracle.f32_to_bf16(cache.values["k"][1].transpose(1, 0, 2))
    assert np.array_equal(bits(k_out)[60:80], want)
    for page in (-1, 10 ** 6):
        cache.table[1, 1] = page
        status.zero_()
        moe.moe_cache_read(d, cache.dev, torch.from_numpy(cache.table[1:]).cuda(),
                           torch.tensor([0, 20], dtype=torch.int32, device="cuda"), k_out, v_out, status)
        torch.cuda.synchronize()
        assert int(status.item()) == moe.MOE_DEV_BAD_PAGE
        assert not k_out[16:20].any() and np.array_equal(bits(k_out)[:16], want[:16])
