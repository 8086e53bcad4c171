"""GPU: streams that the norm and the calls with 4-bit weights take: torch's, or an object with a handle alone, as the other calls
do; and tensors of another device than the stream's."""
import numpy as np
import pytest
import torch

from gpu_cases import require_gpu
from oracle import w4_oracle as wo
from test_gpu_attn_arguments import elsewhere

pytestmark = pytest.mark.gpu


class Handle:
    """A stream of the current device by its handle."""

    def __init__(self, stream):
        self.cuda_stream = stream.cuda_stream


@pytest.mark.parametrize("bare", [False, True])
def test_quantized_and_packed_on_a_stream(bare):
    moe = require_gpu()
    own = torch.cuda.Stream()
    stream = Handle(own) if bare else own
    w = np.random.default_rng(3).standard_normal((32, 256)).astype(np.float32)
    dev = torch.from_numpy(w).cuda()
    q, s = (torch.empty((32, n), dtype=torch.uint8, device="cuda") for n in (128, 8))
    packed, packed_s = torch.empty_like(q), torch.empty(moe.moe_w4_scale_bytes(1, 32, 256), dtype=torch.uint8, device="cuda")
    own.wait_stream(torch.cuda.current_stream())
    moe.moe_quant_weight_w4(dev, q, s, stream=stream)
    moe.moe_pack_weight_w4(q, s, packed, packed_s, stream=stream)
    torch.cuda.synchronize()
    ref, ref_s = wo.pack(*wo.quantize(w))
    assert np.array_equal(packed.cpu().numpy().reshape(-1), ref) and np.array_equal(packed_s.cpu().numpy(), ref_s)


@pytest.mark.parametrize("bare", [False, True])
def test_tensors_of_another_device(bare):
    """Every tensor of every call has to be on the device of the call's stream."""
    moe = require_gpu()
    stream = Handle(torch.cuda.current_stream()) if bare else torch.cuda.current_stream()
    h, t = 128, 2

    def bytes_(*shape):
        return torch.zeros(shape, dtype=torch.uint8, device="cuda")

    def bf16(*shape):
        return torch.zeros(shape, dtype=torch.bfloat16, device="cuda")

    def f32(*shape):
        return torch.zeros(shape, device="cuda")

    def ints(*shape):
        return torch.zeros(shape, dtype=torch.int32, device="cuda")
    scales = moe.moe_w4_scale_bytes(1, h, h)
    dims = moe.MoeDims(h, h, 1, 1)
    stacks = {f"{kind}_{part}": bytes_(1, h, h // 2) if kind == "w" else bytes_(scales)
              for part in ("gate", "up", "down") for kind in "ws"}
    ws = bytes_(1 << 16)
    calls = {
        "moe_quant_weight_w4": dict(w=f32(h, h), q=bytes_(h, h // 2), s=bytes_(h, h // 32)),
        "moe_pack_weight_w4": dict(q=bytes_(h, h // 2), s=bytes_(h, h // 32), packed=bytes_(h, h // 2), packed_s=bytes_(scales),
                                   dev_status=ints(1)),
        "moe_add_norm": dict(x=bf16(t, h), weight=bf16(h), out=bf16(t, h), q=bytes_(t, h), s=f32(t, 1), residual=f32(t, h),
                             sum_out=f32(t, h)),
        "moe_linear_w4": dict(x=bf16(t, h), w=bytes_(h, h // 2), w_s=bytes_(scales), out=f32(t, h), bias=bf16(h), ws=ws),
        "moe_expert_ffn_w4": dict(dims=dims, T=t, x_bf16=bf16(t, h), expert_offsets=ints(2), sorted_src=ints(t), **stacks,
                                  y_rows=f32(t, h), ws=ws),
        "moe_ffn_layer_w4": dict(dims=dims, T=t, x_bf16=bf16(t, h), topk_ids=ints(t, 1), topk_w=f32(t, 1), **stacks,
                                 out_bf16=bf16(t, h), dev_status=ints(1), ws=ws)}
    for name, args in calls.items():
        call = getattr(moe, name)
        for key, value in args.items():
            if isinstance(value, torch.Tensor):
                with pytest.raises(ValueError, match="is on another device"):
                    call(**dict(args, **{key: elsewhere(value)}), stream=stream)
        call(**args, stream=stream)
    torch.cuda.synchronize()
