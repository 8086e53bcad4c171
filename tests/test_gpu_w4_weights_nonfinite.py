"""GPU: 4-bit weights from groups that hold a NaN or an infinity: marked by the quantizer and reported by the
packing; the other groups are as they are without them, and so are the products' columns that hold no such group."""
import numpy as np
import pytest
import torch

from gpu_cases import require_gpu
from oracle import w4_oracle as wo

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("value", [float("nan"), float("inf"), -float("inf")])
def test_marked_and_reported(value):
    moe = require_gpu()
    rows, cols = 48, 256
    w = np.random.default_rng(3).standard_normal((rows, cols)).astype(np.float32)
    q, s = wo.quantize(w)
    places = [(0, 0), (17, 31), (17, 100), (30, 255), (47, 64)]
    for row, col in places:
        w[row, col] = value
    w[30, 224:256] = value  # a whole group
    dq, ds = torch.empty((rows, cols // 2), dtype=torch.uint8, device="cuda"), torch.empty((rows, cols // 32), dtype=torch.uint8, device="cuda")
    moe.moe_quant_weight_w4(torch.from_numpy(w).cuda(), dq, ds)
    marked = np.zeros((rows, cols // 32), bool)
    for row, col in places:
        marked[row, col // 32] = True
    got = ds.cpu().numpy()
    assert (got[marked] == 255).all() and np.array_equal(got[~marked], s[~marked])
    same = np.repeat(~marked, 16, 1)
    assert np.array_equal(dq.cpu().numpy()[same], q[same])
    packed, packed_s = torch.empty_like(dq), torch.empty(moe.moe_w4_scale_bytes(1, rows, cols), dtype=torch.uint8, device="cuda")
    status = torch.zeros(1, dtype=torch.int32, device="cuda")
    moe.moe_pack_weight_w4(dq, ds, packed, packed_s, status)
    assert int(status.item()) == moe.MOE_DEV_BAD_SCALE
    hit = torch.from_numpy(marked.any(1)).cuda()
    values = torch.from_numpy(wo.values(q, s)).cuda()
    for tokens in (1, 16, 40, 200):
        x = torch.from_numpy(np.random.default_rng(tokens).choice([-1.0, 1.0], (tokens, cols)).astype(np.float32)).bfloat16().cuda()
        out = torch.empty((tokens, rows), device="cuda")
        moe.moe_linear_w4(x, packed, packed_s, out, ws=torch.empty(1 << 20, dtype=torch.uint8, device="cuda"))
        ref = x.double() @ values.t()
        size = x.double().abs() @ values.abs().t()
        assert ((out.double() - ref).abs() <= cols * 2.0 ** -23 * size)[:, ~hit].all()
