"""GPU: arguments that the attention calls' binding has to refuse, or to take."""
import numpy as np
import pytest
import torch

from attention_cases import Cache, bf16
from gpu_cases import require_gpu
from oracle import attention_oracle as ao
from test_gpu_attn_binding import NAMES, Call

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


@pytest.fixture(scope="module")
def call(moe):
    return Call(moe)


@pytest.mark.parametrize("name", NAMES)
def test_types_of_the_same_size(call, name):
    """An fp32 length, page, position or slot, and an int32 rotary table, are no bits to be taken as they stand."""
    tried = 0
    for key, value in call.args[name].items():
        if not isinstance(value, torch.Tensor) or value.dtype not in (torch.int32, torch.float32):
            continue
        other = value.float() if value.dtype == torch.int32 else value.int()
        with pytest.raises(ValueError, match=key):
            call(name, **{key: other})
        tried += 1
    assert tried
    with pytest.raises(ValueError, match="dev_status"):
        call(name, dev_status=torch.zeros(1, device="cuda"))


def test_types_of_the_cache_and_the_table(moe):
    codes, scales = torch.zeros((3, 2, 16, 64), dtype=torch.uint8, device="cuda"), torch.zeros((3, 2, 16), device="cuda")
    moe.KVCache(codes, codes.view(torch.float8_e4m3fn), scales, scales)
    with pytest.raises(ValueError, match="k_scale"):
        moe.KVCache(codes, codes, scales.int(), scales)
    with pytest.raises(ValueError, match="v_scale"):
        moe.KVCache(codes, codes, scales, scales.int())
    for other in (torch.bool, torch.float8_e5m2):
        with pytest.raises(ValueError, match="^v "):
            moe.KVCache(codes, codes.view(other), scales, scales)
    with pytest.raises(ValueError, match="table"):
        moe.moe_rope_table(torch.zeros((8, 64), dtype=torch.int32, device="cuda"))


def test_an_output_without_its_input(call, moe):
    """As the C call: queries and their output, and keys and theirs, are given together."""
    for changed in (dict(q=None), dict(k=None), dict(q=None, k=None)):
        with pytest.raises(moe.MoEError) as e:
            call("moe_rope", **changed)
        assert e.value.status == moe.MOE_ERR_INVALID_ARG
    call("moe_rope", q=None, q_out=None)
    call("moe_rope", k=None, k_out=None)


def test_a_flag_that_has_no_truth_value(call):
    class Vague:
        def __bool__(self):
            raise RuntimeError("neither")
    with pytest.raises(RuntimeError, match="neither"):
        call("moe_attn_prefill", causal=Vague())
    call("moe_attn_prefill", causal=0)
    call("moe_attn_prefill", causal=np.True_)


class Elsewhere(torch.Tensor):
    @classmethod
    def __torch_dispatch__(cls, func, types, args=(), kwargs=None):
        raise NotImplementedError(func)


def elsewhere(t):
    """A tensor like t that says it is on another device (and has no memory)."""
    return torch.Tensor._make_wrapper_subclass(Elsewhere, t.shape, strides=t.stride(), dtype=t.dtype,
                                               device=torch.device("cuda:1"))


@pytest.mark.parametrize("name", NAMES)
def test_tensors_of_another_device(call, name):
    """A call runs on its stream's device, the current one's if none is given."""
    assert torch.cuda.current_device() == 0
    streams = (None, torch.cuda.current_stream())
    for stream in streams:
        for key, value in call.args[name].items():
            if isinstance(value, torch.Tensor):
                with pytest.raises(ValueError, match=f"{key} is on another device"):
                    call(name, **{key: elsewhere(value)}, stream=stream)
        call(name, stream=stream)

    class Handle:
        cuda_stream = torch.cuda.current_stream().cuda_stream
    call(name, stream=Handle())


def test_caches_and_tables_of_another_device(call, moe):
    codes, scales = torch.zeros((3, 2, 16, 64), dtype=torch.uint8, device="cuda"), torch.zeros((3, 2, 16), device="cuda")
    for i in range(4):
        parts = [codes, codes, scales, scales]
        parts[i] = elsewhere(parts[i])
        with pytest.raises(ValueError, match="different devices"):
            moe.KVCache(*parts)
    cache = moe.KVCache(codes, codes, scales, scales)
    cache.on_device.device = 1
    for name in ("moe_rope_cache", "moe_cache_read", "moe_attn_decode"):
        with pytest.raises(ValueError, match="cache is on another device"):
            call(name, cache=cache)
    with pytest.raises(ValueError, match="table is on another device"):
        moe.moe_rope_table(elsewhere(torch.zeros((8, 64), device="cuda")))
    with pytest.raises(ValueError, match="table is on another device"):
        moe.moe_rope_table(elsewhere(torch.zeros((8, 64), device="cuda")), stream=torch.cuda.current_stream())


@pytest.mark.parametrize("prefix", [40, 2000])
def test_tables_without_columns(moe, prefix):
    """Sequences that have nothing of their own yet: a table of no pages, which has no address."""
    rng = np.random.default_rng(71)
    cache = Cache(moe, rng, [prefix], 2, 64, 16)
    q, qv = bf16(rng.standard_normal((3, 4, 64)))
    d = moe.MoeAttnDims(4, 2, 64)
    none = torch.empty((3, 0), dtype=torch.int32, device="cuda")
    zero = torch.zeros(3, dtype=torch.int32, device="cuda")
    out, status = torch.empty_like(q), torch.zeros(1, dtype=torch.int32, device="cuda")
    ws = torch.empty(max(256, moe.moe_attn_decode_workspace(d, 3, 0, prefix)), dtype=torch.uint8, device="cuda")
    moe.moe_attn_decode(d, q, cache.dev, none, zero, 0, 0.1, out, ws, prefix_pages=torch.from_numpy(cache.table[0]).cuda(),
                        prefix_len=prefix, dev_status=status)
    for h in range(4):
        ref, bound = ao.attention(qv[:, h], cache.values["k"][0][h // 2], cache.values["v"][0][h // 2], 0.1)
        assert np.all(np.abs(out[:, h].double().cpu().numpy() - ref) <= bound)
    assert int(status.item()) == 0
    moe.moe_attn_decode(d, q, cache.dev, none, zero, 0, 0.1, out, ws)
    assert not out.any()
    rows = [torch.full((5, 2, 64), 9.0, dtype=torch.bfloat16, device="cuda") for _ in "kv"]
    moe.moe_cache_read(d, cache.dev, none, torch.zeros(4, dtype=torch.int32, device="cuda"), *rows, status)
    assert int(status.item()) == 0 and all(bool((r == 9).all()) for r in rows)
    moe.moe_cache_read(d, cache.dev, none, torch.tensor([0, 0, 2, 2], dtype=torch.int32, device="cuda"), *rows, status)
    assert int(status.item()) == moe.MOE_DEV_BAD_LENGTH
    assert all(not r[:2].any() and bool((r[2:] == 9).all()) for r in rows)


def test_a_call_within_a_call(call, moe):
    """A stream whose handle comes from Python code, which makes calls of its own on another: each call has its own stream."""
    class Far:
        cuda_stream, device_index = 0, 1

    class Nested:
        device_index = 0

        @property
        def cuda_stream(self):
            with pytest.raises(ValueError, match="another device"):
                call("moe_attn_decode", stream=Far())
            return torch.cuda.current_stream().cuda_stream
    for name in NAMES:
        call(name, stream=Nested())
        with pytest.raises(ValueError, match="another device"):
            call(name, stream=Far())


def test_the_cache_and_its_structure_are_one(moe):
    cache = moe.KVCache.empty(3, 2, 16, 64)
    assert bytes(cache.c) == bytes(cache.on_device)[:len(bytes(cache.c))]
    cache.c.n_pages = 2
    assert cache.on_device.cache.n_pages == 2
