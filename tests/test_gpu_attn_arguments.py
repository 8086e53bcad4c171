"""GPU: arguments that the attention calls' binding has to refuse, or to take."""
import numpy as np
import pytest
import torch

from gpu_cases import require_gpu
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
