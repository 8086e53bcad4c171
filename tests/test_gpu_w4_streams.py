"""GPU: streams that the set-up of 4-bit weights takes: torch's, or an object with a handle alone, as the other calls do."""
import numpy as np
import pytest
import torch

from gpu_cases import require_gpu
from oracle import w4_oracle as wo

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
