"""GPU: moe_add_norm over rows that hold NaN or infinities, beside rows that do not.

What the formula gives in 64 bits is what the outputs have to show: a NaN makes its whole row NaN, an infinity itself
alone (its quotient by the root is NaN, that of the row's other values 0).  Where a block of 128 values holds a NaN its
scale is one, so that no product with its codes is a number.  Other rows are what they are without such neighbours, bit
for bit.
"""
import numpy as np
import pytest
import torch

from gpu_cases import require_gpu
from oracle import w4_oracle as wo

pytestmark = pytest.mark.gpu
TYPES = {"bf16": torch.bfloat16, "f32": torch.float32}
NANS = [0x7fffffff, 0xffffffff, 0x7fc00000, 0x7f800001, 0x7fff8000]  # fp32; bf16 takes the upper halves, where these are NaN


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def bits(values, dtype):
    words = np.array(values, np.uint32)
    if dtype == torch.float32:
        return torch.from_numpy(words.view(np.float32).copy())
    return torch.from_numpy((words >> 16 | (words & 0xffff != 0) * np.uint32(0x40)).astype(np.uint16).view(np.int16).copy()).view(torch.bfloat16)


def spoil(x, r, where):
    """Rows 1, 4, 7, ... of x, or of r, get a value that is not finite."""
    h = x.shape[-1]
    flat_x, flat_r = x.view(-1, h), None if r is None else r.view(-1, h)
    nan = bits(NANS, x.dtype)
    kinds = [nan[0], nan[1], nan[2], nan[3], nan[4], float("inf"), -float("inf")]
    bad = list(range(1, flat_x.shape[0], 3))
    for n, row in enumerate(bad):
        kind, at = n % (len(kinds) + (r is not None)), (where * (n + 1)) % h
        if kind < len(kinds):
            target = flat_x if r is None or n % 2 else flat_r
            target[row, at] = kinds[kind] if not torch.is_tensor(kinds[kind]) else bits(NANS[kind:kind + 1], target.dtype)[0]
        else:  # infinities that cancel
            flat_x[row, at], flat_r[row, at] = float("inf"), -float("inf")
    return bad


CASES = [  # tokens, H, heads, x, stream, residual, codes: rows of 8 to 1024 lanes
    (22, 64, 3, "bf16", "bf16", False, False), (22, 128, 2, "f32", "f32", True, True), (22, 72, 1, "bf16", "f32", True, False),
    (23, 512, 1, "f32", "bf16", True, True), (23, 1024, 1, "bf16", "bf16", True, True), (300, 4096, 1, "bf16", "f32", True, True),
    (25, 7168, 1, "f32", "f32", True, True), (25, 7168, 1, "bf16", "bf16", False, True), (24, 16384, 1, "f32", "f32", False, True)]


@pytest.mark.parametrize("tokens,h,heads,xt,st,residual,codes", CASES)
def test_nan_and_infinities_show(moe, tokens, h, heads, xt, st, residual, codes):
    g = torch.Generator().manual_seed(tokens + h)
    shape = (tokens, heads, h) if heads > 1 else (tokens, h)
    x = torch.randn(shape, generator=g).to(TYPES[xt])
    r = torch.randn(shape, generator=g).to(TYPES[st]) if residual else None
    w = (1 + 0.3 * torch.randn(h, generator=g)).bfloat16().cuda()
    rows = tokens * heads

    def call(x, r):
        out = torch.empty(shape, dtype=torch.bfloat16, device="cuda")
        total = torch.empty(shape, dtype=TYPES[st], device="cuda")
        q = torch.empty((rows, h), dtype=torch.uint8, device="cuda") if codes else None
        s = torch.empty((rows, h // 128), dtype=torch.float32, device="cuda") if codes else None
        moe.moe_add_norm(x.cuda(), w, out, q, s, residual=None if r is None else r.cuda(), sum_out=total)
        return out.view(rows, h), total.view(rows, h), q, s
    clean = call(x, r)
    bad = spoil(x, r, 131)
    got = call(x, r)
    good = torch.ones(rows, dtype=torch.bool)
    good[bad] = False
    for a, b in zip(clean, got):
        if a is not None:
            assert torch.equal(a[good.cuda()], b[good.cuda()])
    with np.errstate(invalid="ignore"):
        z, y = wo.add_norm(x.double().numpy(), None if r is None else r.double().numpy(), w.double().cpu().numpy(), 1e-6)
    z, y = z.reshape(rows, h)[bad], y.reshape(rows, h)[bad]
    assert np.isnan(y).any(-1).all()  # every one of them has something to show
    out, total, q, s = (None if a is None else a[bad].cpu() for a in got)
    assert np.array_equal(torch.isnan(out).numpy(), np.isnan(y))
    assert (out[~torch.isnan(out)] == 0).all()
    assert np.array_equal(torch.isnan(total).numpy(), np.isnan(z))
    assert np.array_equal(torch.isinf(total).numpy(), np.isinf(z))
    if codes:
        v = q.view(torch.float8_e4m3fn).float().view(len(bad), -1, 128) * s[..., None]
        blocks = np.isnan(y).reshape(len(bad), -1, 128).any(-1)
        assert np.array_equal(torch.isnan(s).numpy(), blocks)
        assert (s[~torch.isnan(s)] == 0).all()
        assert np.array_equal(torch.isnan(v).all(-1).numpy(), blocks) and np.array_equal(torch.isnan(v).any(-1).numpy(), blocks)
