"""GPU: attention of single tokens over the paged e4m3 cache against the fp64 oracle, element by element, within the
bound that the definition's roundings give.  Every slot that holds no token has NaN codes and NaN or infinite scales."""
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


def reference(cache, qv, n, scale, prefix, heads=None):
    """cache.lens: the sequences' and then, with a prefix, its length."""
    b, hq, dim = qv.shape
    g = hq // cache.heads
    out, bound = np.zeros(qv.shape), np.zeros(qv.shape)
    for i in range(b):
        for h in (range(hq) if heads is None else heads):
            rows = [cache.values[x][n][h // g] for x in "kv"] if prefix else None
            own = [cache.values[x][i][h // g] for x in "kv"]
            k, v = (np.concatenate([r, o]) for r, o in zip(rows, own)) if prefix else own
            o, e = ao.attention(qv[i, h][None], k, v, scale)
            out[i, h], bound[i, h] = o[0], e[0]
    return out, bound


def run(moe, dims, q, cache, lens, scale, prefix=0, max_len=None, status=None, out=None, ws_fill=0xFF):
    d = moe.MoeAttnDims(*dims)
    n = len(lens)
    out = torch.full((n, dims[0], dims[2]), float("nan"), dtype=torch.bfloat16, device="cuda") if out is None else out
    max_len = max(list(lens) + [0]) if max_len is None else max_len
    ws = torch.empty(max(256, moe.moe_attn_decode_workspace(d, n, max_len, prefix)), dtype=torch.uint8,
                     device="cuda").fill_(ws_fill)
    table = torch.from_numpy(cache.table[:n].copy()).cuda()
    pages = torch.from_numpy(cache.table[n, :-(-prefix // cache.page)].copy()).cuda() if prefix else None
    moe.moe_attn_decode(d, q, cache.dev, table, torch.tensor(lens, dtype=torch.int32, device="cuda"), max_len, scale, out,
                        ws, prefix_pages=pages, prefix_len=prefix, dev_status=status)
    torch.cuda.synchronize()
    return out


def check(got, ref, bound, what):
    got = got.double().cpu().numpy()
    assert np.isfinite(got).all(), f"{what}: not finite"
    worst = float(np.max(np.abs(got - ref) / np.maximum(bound, 1e-30)))
    log(f"{what}: worst error {worst:.3f} of its bound")
    assert worst <= 1.0


CASES = [
    # heads, lengths, page, prefix
    ((4, 4, 64), [1], 16, 0),
    ((8, 2, 128), [0], 16, 0),
    ((8, 2, 128), [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255], 16, 0),
    ((8, 2, 64), [0, 1, 15, 16, 17, 31, 32, 33, 63, 64, 65, 127, 128, 129, 255], 64, 0),
    ((14, 2, 128), [300, 7], 32, 0),
    ((16, 1, 128), [500, 100], 128, 0),
    ((40, 2, 64), [90, 200], 64, 0),                      # groups of 20: more than one product's columns
    ((34, 1, 128), [77], 16, 0),                          # 34 = 16 + 16 + 2
    ((8, 2, 128), [0, 1, 40], 16, 1),
    ((8, 2, 128), [0, 0], 32, 33),
    ((8, 2, 64), [5, 200, 0, 64], 64, 500),
    ((8, 1, 128), [5, 90, 0, 64, 1, 1, 1, 300], 16, 257),  # 64 rows on the prefix
    ((28, 4, 128), [30] * 33, 32, 700),                   # 231 rows on the prefix
    ((40, 2, 64), [17, 3], 16, 130),
]


@pytest.mark.parametrize("dims,lens,page,prefix", CASES)
def test_steps(moe, dims, lens, page, prefix):
    rng = np.random.default_rng(21)
    hq, hkv, dim = dims
    cache = Cache(moe, rng, list(lens) + ([prefix] if prefix else []), hkv, dim, page)
    q, qv = bf16(rng.standard_normal((len(lens), hq, dim)))
    scale = 1 / math.sqrt(dim)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(moe, dims, q, cache, lens, scale, prefix, status=status)
    ref, bound = reference(cache, qv, len(lens), scale, prefix)
    check(got, ref, bound, f"{dims} {lens} page {page} prefix {prefix}")
    assert int(status.item()) == 0


@pytest.mark.parametrize("dims,lens,page,prefix", [((8, 2, 128), [9000], 64, 0), ((4, 1, 64), [4097, 3, 2500], 16, 0),
                                                   ((8, 1, 128), [40] * 20, 64, 5000), ((8, 2, 64), [2000], 32, 3001)])
def test_long_axes(moe, dims, lens, page, prefix):
    """Long contexts and prefixes, whose keys many workgroups share: two heads."""
    rng = np.random.default_rng(22)
    hq, hkv, dim = dims
    cache = Cache(moe, rng, list(lens) + ([prefix] if prefix else []), hkv, dim, page)
    q, qv = bf16(rng.standard_normal((len(lens), hq, dim)))
    got = run(moe, dims, q, cache, lens, 0.1, prefix)
    heads = [0, hq - 1]
    ref, bound = reference(cache, qv, len(lens), 0.1, prefix, heads)
    check(got[:, heads], ref[:, heads], bound[:, heads], f"long {dims} {lens} prefix {prefix}")


def test_the_split_does_not_depend_on_a_wrong_longest_length(moe):
    rng = np.random.default_rng(23)
    dims, lens = (8, 2, 128), [3000, 5]
    cache = Cache(moe, rng, lens, 2, 128, 64)
    q, qv = bf16(rng.standard_normal((2, 8, 128)))
    ref, bound = reference(cache, qv, 2, 0.09, 0)
    for max_len in (0, 5, 3000, 1000000):
        check(run(moe, dims, q, cache, lens, 0.09, max_len=max_len), ref, bound, f"max_len={max_len}")


@pytest.mark.parametrize("size", [30.0, 0.0])
def test_peaked_and_flat_scores(moe, size):
    rng = np.random.default_rng(24)
    cache = Cache(moe, rng, [700, 30, 200], 2, 128, 32)
    q, qv = bf16(rng.standard_normal((2, 8, 128)) * size)
    got = run(moe, (8, 2, 128), q, cache, [700, 30], 0.09, 200)
    ref, bound = reference(cache, qv, 2, 0.09, 200)
    check(got, ref, bound, f"scores x {size}")


def test_strided_queries(moe):
    rng = np.random.default_rng(25)
    cache = Cache(moe, rng, [50, 60], 2, 64, 16)
    x, xv = bf16(rng.standard_normal((2, 20, 64)))
    got = run(moe, (8, 2, 64), x[:, 4:12], cache, [50, 60], 0.1)
    ref, bound = reference(cache, xv[:, 4:12], 2, 0.1, 0)
    check(got, ref, bound, "strided queries")


def test_same_inputs_give_the_same_bits(moe):
    rng = np.random.default_rng(26)
    cache = Cache(moe, rng, [2000, 77, 900], 2, 128, 64)
    q, _ = bf16(rng.standard_normal((2, 8, 128)))
    first = run(moe, (8, 2, 128), q, cache, [2000, 77], 0.1, 900)
    again = run(moe, (8, 2, 128), q, cache, [2000, 77], 0.1, 900, ws_fill=0)
    assert torch.equal(first.view(torch.int16), again.view(torch.int16))


def test_bad_lengths_and_pages_are_reported(moe):
    rng = np.random.default_rng(27)
    dims = (8, 2, 128)
    cache = Cache(moe, rng, [64, 64], 2, 128, 16)
    q, qv = bf16(rng.standard_normal((2, 8, 128)))
    ref, bound = reference(cache, qv, 2, 0.1, 0)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(moe, dims, q, cache, [64, 1000], 0.1, status=status)  # cut to the table's 4 pages
    check(got, ref, bound, "cut length")
    assert int(status.item()) == moe.MOE_DEV_BAD_LENGTH
    status.zero_()
    got = run(moe, dims, q, cache, [64, -3], 0.1, status=status)
    assert int(status.item()) == moe.MOE_DEV_BAD_LENGTH
    check(got[:1], ref[:1], bound[:1], "beside a negative length")
    assert not got[1].any()
    for page in (-1, 10 ** 6):
        status.zero_()
        cache.table[1, 2] = page
        got = run(moe, dims, q, cache, [64, 64], 0.1, status=status)
        assert int(status.item()) == moe.MOE_DEV_BAD_PAGE
        check(got[:1], ref[:1], bound[:1], "beside a bad page")


@pytest.mark.parametrize("prefix", [0, 300])
def test_replays_from_a_hip_graph(moe, prefix):
    """A step captured once and replayed with new queries and lengths, eager work in between."""
    rng = np.random.default_rng(28)
    dims = (8, 2, 128)
    cache = Cache(moe, rng, [1500, 40] + ([prefix] if prefix else []), 2, 128, 64)
    d = moe.MoeAttnDims(*dims)
    q = torch.empty((2, 8, 128), dtype=torch.bfloat16, device="cuda").normal_()
    lens = torch.tensor([1500, 40], dtype=torch.int32, device="cuda")
    table = torch.from_numpy(cache.table[:2].copy()).cuda()
    pages = torch.from_numpy(cache.table[2, :-(-prefix // 64)].copy()).cuda() if prefix else None
    ws = torch.empty(max(256, moe.moe_attn_decode_workspace(d, 2, 1500, prefix)), dtype=torch.uint8, device="cuda")
    out = torch.empty_like(q)

    def call(ws_, out_):
        moe.moe_attn_decode(d, q, cache.dev, table, lens, 1500, 0.1, out_, ws_, prefix_pages=pages, prefix_len=prefix)
    call(ws, out)
    torch.cuda.synchronize()
    graph, side = torch.cuda.CUDAGraph(), torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    with torch.cuda.graph(graph, stream=side):
        call(ws, out)
    torch.cuda.synchronize()
    for n in ((1500, 40), (7, 0), (1000, 33)):
        q.normal_()
        lens.copy_(torch.tensor(n, dtype=torch.int32))
        ref = torch.empty_like(q)
        call(torch.empty_like(ws), ref)
        torch.cuda.synchronize()
        graph.replay()
        torch.cuda.synchronize()
        assert torch.equal(out.view(torch.int16), ref.view(torch.int16)), n


def test_on_a_stream_of_its_own(moe):
    rng = np.random.default_rng(29)
    cache = Cache(moe, rng, [300, 90], 2, 128, 64)
    q, qv = bf16(rng.standard_normal((2, 8, 128)))
    d = moe.MoeAttnDims(8, 2, 128)
    out = torch.empty_like(q)
    ws = torch.empty(max(256, moe.moe_attn_decode_workspace(d, 2, 300, 0)), dtype=torch.uint8, device="cuda")
    table, lens = torch.from_numpy(cache.table).cuda(), torch.tensor([300, 90], dtype=torch.int32, device="cuda")
    side = torch.cuda.Stream()
    side.wait_stream(torch.cuda.current_stream())
    moe.moe_attn_decode(d, q, cache.dev, table, lens, 300, 0.1, out, ws, stream=side)
    side.synchronize()
    ref, bound = reference(cache, qv, 2, 0.1, 0)
    check(out, ref, bound, "side stream")


def test_pages_beyond_4_gib(moe):
    """A cache whose arrays are over 4 GiB: pages at its far end, written by moe_rope_cache and read by both readers."""
    rng = np.random.default_rng(30)
    heads, page, dim = 8, 64, 128
    n_pages = (1 << 32) // (heads * page * dim) + 40
    cache = moe.KVCache.empty(n_pages, heads, page, dim)
    d = moe.MoeAttnDims(8, heads, dim)
    n = 100
    x, xv = bf16(rng.standard_normal((n, 8, dim)))
    table = torch.zeros((4, 16), dtype=torch.float32, device="cuda")
    moe.moe_rope_table(table)
    zero = torch.zeros(n, dtype=torch.int32, device="cuda")
    far = [n_pages - 1, n_pages - 7]
    slots = np.array([far[t // page] * page + t % page for t in range(n)], np.int32)
    moe.moe_rope_cache(d, x, x, x, zero, table, moe.MOE_ROPE_HALF, torch.from_numpy(slots).cuda(), cache,
                       torch.empty_like(x))
    pages = torch.tensor([far], dtype=torch.int32, device="cuda")
    ko, vo = torch.empty_like(x), torch.empty_like(x)
    moe.moe_cache_read(d, cache, pages, torch.tensor([0, n], dtype=torch.int32, device="cuda"), ko, vo)
    torch.cuda.synchronize()
    c, s = ao.quantize_head_rows(xv.astype(np.float32))
    want = ao.cached_rows(c, s)
    assert torch.equal(ko.cpu(), torch.from_numpy(want).bfloat16()) and torch.equal(vo.cpu(), ko.cpu())
    out = torch.empty((1, 8, dim), dtype=torch.bfloat16, device="cuda")
    ws = torch.empty(max(256, moe.moe_attn_decode_workspace(d, 1, n, 0)), dtype=torch.uint8, device="cuda")
    moe.moe_attn_decode(d, x[:1].contiguous(), cache, pages, torch.tensor([n], dtype=torch.int32, device="cuda"), n, 0.1, out,
                        ws)
    torch.cuda.synchronize()
    for h in (0, 7):
        ref, bound = ao.attention(xv[:1, h], want[:, h], want[:, h], 0.1)
        check(out[:, h], ref, bound, f"far pages, head {h}")


@pytest.mark.parametrize("dims,prefix", [((4, 2, 64), 0), ((8, 2, 128), 300)])
def test_more_sequences_than_a_wave_has_lanes(moe, dims, prefix):
    """Ragged batches of 150 whose pieces begin and end anywhere; sequences are looked up 64 at a time."""
    rng = np.random.default_rng(31)
    hq, hkv, dim = dims
    lens = [int(n) for n in rng.integers(0, 200, 150)]
    lens[3], lens[70], lens[149] = 1500, 0, 900
    cache = Cache(moe, rng, lens + ([prefix] if prefix else []), hkv, dim, 32)
    q, qv = bf16(rng.standard_normal((150, hq, dim)))
    got = run(moe, dims, q, cache, lens, 0.1, prefix)
    ref, bound = reference(cache, qv, 150, 0.1, prefix)
    check(got, ref, bound, f"150 sequences, prefix {prefix}")


def test_more_heads_than_workgroups(moe):
    rng = np.random.default_rng(32)
    dims, lens = (520, 520, 64), [700, 5]
    cache = Cache(moe, rng, lens, 520, 64, 64)
    q, qv = bf16(rng.standard_normal((2, 520, 64)))
    got = run(moe, dims, q, cache, lens, 0.1)
    heads = [0, 511, 512, 519]
    ref, bound = reference(cache, qv, 2, 0.1, 0, heads)
    check(got[:, heads], ref[:, heads], bound[:, heads], "520 heads")


@pytest.mark.parametrize("power", [-90, -20, 60])
def test_values_of_extreme_sizes(moe, power):
    """Value rows from 2^-40 to 2^0 of the largest in every order, all times 2^power: the reference that the numerators are
    taken against follows the values' scales."""
    rng = np.random.default_rng(33)
    n = 1000
    cache = Cache(moe, rng, [n], 1, 64, 16)
    factor = (2.0 ** (power - rng.integers(0, 41, n))).astype(np.float32)
    for t in range(n):
        p, o = cache.table[0, t // 16], t % 16
        cache.scales["v"][p, 0, o] *= factor[t]
    cache.values["v"][0] = cache.values["v"][0] * factor[None, :, None]
    cache.dev.v_scale.copy_(torch.from_numpy(cache.scales["v"]))
    q, qv = bf16(rng.standard_normal((1, 4, 64)))
    got = run(moe, (4, 1, 64), q, cache, [n], 0.1)
    ref, bound = reference(cache, qv, 1, 0.1, 0)
    check(got, ref, bound, f"values times 2^{power}")


def one_launch(moe, dims, batch, longest, prefix):
    return moe.moe_attn_decode_workspace(moe.MoeAttnDims(*dims), batch, longest, prefix) == 0


@pytest.mark.parametrize("dims", [(8, 2, 128), (40, 2, 64), (4, 1, 64)])
@pytest.mark.parametrize("prefix,longest,one", [
    (1, 512, True), (127, 1, True), (129, 384, True), (300, 256, True), (512, 128, True), (513, 0, True), (512, 129, True),
    (1024, 300, False), (512, 700, False), (1290, 0, False), (0, 1024, False)])
def test_one_launch_and_two(moe, dims, prefix, longest, one):
    """Few steps of 128 keys, the prefix's among them, take one launch and no workspace."""
    rng = np.random.default_rng(prefix + longest)
    hq, hkv, dim = dims
    lens = [longest, 0, min(longest, 1), longest // 2]
    assert one_launch(moe, dims, len(lens), longest, prefix) == one
    cache = Cache(moe, rng, lens + [prefix], hkv, dim, 32)
    q, qv = bf16(rng.standard_normal((len(lens), hq, dim)))
    scale = 1 / math.sqrt(dim)
    out = run(moe, dims, q, cache, lens, scale, prefix, max_len=longest)
    ref, bound = reference(cache, qv, len(lens), scale, prefix)
    check(out, ref, bound, f"{dims} prefix {prefix} longest {longest}")


ODD = [0, 1, 15, 16, 17, 31, 33, 127, 128, 129]
TWO = [
    ((8, 2, 128), ODD, 16, 1100),
    ((8, 2, 64), ODD, 64, 1500),
    ((8, 1, 128), [5, 90, 0, 64, 1, 1, 1, 300], 16, 1157),   # 64 rows on the prefix
    ((28, 4, 128), [30] * 33, 32, 1700),                     # 231 rows on the prefix
    ((40, 2, 64), [17, 3], 16, 1300),                        # more than one product's columns for one sequence
    ((34, 1, 128), [77, 2000], 16, 0),
    ((4, 2, 64), [7 * i % 90 for i in range(150)] + [4000], 16, 0),
    ((8, 2, 128), [5 * i % 70 for i in range(130)] + [3000, 0], 32, 300),
]


@pytest.mark.parametrize("dims,lens,page,prefix", TWO)
def test_pieces_of_a_line(moe, dims, lens, page, prefix):
    assert not one_launch(moe, dims, len(lens), max(lens), prefix)
    rng = np.random.default_rng(33)
    hq, hkv, dim = dims
    cache = Cache(moe, rng, list(lens) + ([prefix] if prefix else []), hkv, dim, page)
    q, qv = bf16(rng.standard_normal((len(lens), hq, dim)))
    scale = 1 / math.sqrt(dim)
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    got = run(moe, dims, q, cache, lens, scale, prefix, status=status)
    ref, bound = reference(cache, qv, len(lens), scale, prefix)
    check(got, ref, bound, f"{dims} {len(lens)} sequences page {page} prefix {prefix}")
    assert int(status.item()) == 0


def test_a_longer_call_never_needs_less_workspace(moe):
    """A workspace for the longest context serves shorter ones."""
    for dims in ((8, 2, 128), (32, 8, 128), (40, 2, 64), (16, 16, 64), (64, 1, 128)):
        for batch in (1, 7, 64, 500, 4000):
            for prefix in (0, 100, 5000):
                need = [moe.moe_attn_decode_workspace(moe.MoeAttnDims(*dims), batch, n, prefix) for n in range(0, 9000, 64)]
                assert need == sorted(need), (dims, batch, prefix)


def test_a_bad_page_of_a_short_prefix_is_reported(moe):
    rng = np.random.default_rng(5)
    cache = Cache(moe, rng, [20, 3, 100], 2, 64, 32)
    q, _ = bf16(rng.standard_normal((2, 4, 64)))
    for page in (-1, cache.dev.n_pages, 1 << 30):
        cache.table[2, 1] = page
        status = torch.zeros(1, dtype=torch.int32, device="cuda")
        run(moe, (4, 2, 64), q, cache, [20, 3], 0.125, 100, status=status)
        assert int(status.item()) == moe.MOE_DEV_BAD_PAGE
