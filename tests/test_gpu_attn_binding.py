"""GPU: what the attention calls' binding refuses before the library is called, and that it takes what it should."""
import pytest
import torch

from gpu_cases import require_gpu

pytestmark = pytest.mark.gpu


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


class Call:
    """Good arguments of every call, by name; a test replaces some."""

    def __init__(self, moe):
        def bf(*shape):
            return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")

        def i32(*values):
            return torch.tensor(values, dtype=torch.int32, device="cuda")
        d = moe.MoeAttnDims(4, 2, 64)
        cache = moe.KVCache(*(torch.zeros((3, 2, 16, 64), dtype=torch.uint8, device="cuda") for _ in "kv"),
                            *(torch.zeros((3, 2, 16), device="cuda") for _ in "kv"))
        table = torch.zeros((8, 64), device="cuda")
        ws = torch.zeros(1 << 20, dtype=torch.uint8, device="cuda")
        self.args = {
            "moe_rope": dict(dims=d, q=bf(3, 4, 64), k=bf(3, 2, 64), positions=i32(0, 1, 2), table=table, layout=0,
                             q_out=bf(3, 4, 64), k_out=bf(3, 2, 64)),
            "moe_rope_cache": dict(dims=d, q=bf(3, 4, 64), k=bf(3, 2, 64), v=bf(3, 2, 64), positions=i32(0, 1, 2),
                                   table=table, layout=1, slots=i32(0, 1, 2), cache=cache, q_out=bf(3, 4, 64),
                                   k_out=bf(3, 2, 64)),
            "moe_cache_read": dict(dims=d, cache=cache, page_table=i32(0, 1).view(2, 1), cu=i32(0, 2, 3), k_out=bf(3, 2, 64),
                                   v_out=bf(3, 2, 64)),
            "moe_attn_prefill": dict(dims=d, q=bf(3, 4, 64), k=bf(5, 2, 64), v=bf(5, 2, 64), cu_q=i32(0, 2, 3),
                                     cu_k=i32(0, 2, 5), max_k=3, scale=0.1, out=bf(3, 4, 64), ws=ws),
            "moe_attn_decode": dict(dims=d, q=bf(2, 4, 64), cache=cache, page_table=i32(0, 1).view(2, 1), lens=i32(3, 16),
                                    max_len=16, scale=0.1, out=bf(2, 4, 64), ws=ws, prefix_pages=i32(2), prefix_len=9),
        }
        self.moe = moe

    def __call__(self, name, **changed):
        args = {**self.args[name], **changed}
        getattr(self.moe, name)(**args)
        torch.cuda.synchronize()


@pytest.fixture(scope="module")
def call(moe):
    return Call(moe)


NAMES = ("moe_rope", "moe_rope_cache", "moe_cache_read", "moe_attn_prefill", "moe_attn_decode")


@pytest.mark.parametrize("name", NAMES)
def test_good_arguments_and_every_wrong_tensor(call, name):
    call(name)
    call(name, stream=torch.cuda.current_stream())
    for key, value in call.args[name].items():
        if not isinstance(value, torch.Tensor):
            continue
        wrong = [value.cpu(), value.double()]
        if value.dim() > 1:
            wrong.append(value.flatten(0, 1))                               # a dimension less
        if value.dtype == torch.bfloat16:
            wrong += [value.half(), value[..., ::2], value[:, :1], value.transpose(1, 2).contiguous().transpose(1, 2)]
        if key not in ("table", "page_table", "ws", "prefix_pages", "out", "q_out", "k_out", "v_out"):
            wrong.append(value[:-1])                                        # an entry less
        for w in wrong:
            with pytest.raises((ValueError, RuntimeError)):
                call(name, **{key: w})
        with pytest.raises(TypeError):
            call(name, **{key: [1, 2, 3]})
    torch.cuda.synchronize()


def test_structures_and_numbers(call, moe):
    with pytest.raises(ValueError, match="another structure"):
        call("moe_attn_prefill", dims=moe.MoeDims(1, 1, 1, 1))
    with pytest.raises(ValueError, match="the cache has"):
        call("moe_attn_decode", dims=moe.MoeAttnDims(4, 4, 64))
    with pytest.raises(ValueError, match="32 bits"):
        call("moe_attn_decode", max_len=1 << 40)
    with pytest.raises(ValueError, match="prefix"):
        call("moe_attn_decode", prefix_len=17)
    with pytest.raises(TypeError):
        call("moe_attn_prefill", scale="0.1")
    with pytest.raises(AttributeError):
        call("moe_attn_prefill", stream=3)
    with pytest.raises(moe.MoEError) as e:
        call("moe_attn_prefill", scale=-1.0)
    assert e.value.status == moe.MOE_ERR_INVALID_ARG


def test_bits_and_views_are_taken(call):
    """16-bit integer views of bf16, a token's stride that is not the heads', one token of any stride, no optional parts."""
    a = call.args["moe_rope_cache"]
    wide = torch.zeros((3, 9, 64), dtype=torch.bfloat16, device="cuda")
    call("moe_rope_cache", q=wide[:, 1:5], k=wide[:, 5:7].view(torch.int16), v=wide[:, 7:], k_out=None)
    one = torch.zeros((1, 4, 640), dtype=torch.bfloat16, device="cuda")[..., :256].as_strided((1, 4, 64), (1, 64, 1))
    call("moe_rope", q=one, k=None, k_out=None, positions=a["positions"][:1],
         q_out=torch.empty((1, 4, 64), dtype=torch.bfloat16, device="cuda"))
    call("moe_attn_decode", prefix_pages=None, prefix_len=0, ws=None)
