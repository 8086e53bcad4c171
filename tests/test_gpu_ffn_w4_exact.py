"""GPU: routed experts with 4-bit weights bit for bit, on numbers that fp32 holds at every step, and the error of ordinary
numbers row by row.

Exact cases.  All weights are whole numbers of -2 .. 2 (as codes under scales of 1/2, 1 and 2), x is +-1 but for one
column of 256, which meets a weight of 1 in the gate projection and 0 in the up projection.  So G is a whole number about
256 and U one about 0; with G >= 32 the sigmoid rounds to 1 in fp32 (exp(-32) < 2^-25), G * U is whole and below 2^24,
h is its rounding to bf16 and whole too, y is a sum of whole numbers below 2^24 and the combine's weights are 1, 1/2 or
1/4 of them, with sums below 2^22.  No order of additions rounds, so the layer's output is known bit for bit: a column,
a block of K, a group's scale or a row that is left out or taken twice shows.

Ordinary numbers.  Roundings of h and of the output are independent and at most 2^-8 of a value each, evenly spread within
half a step, so 2^-8 / sqrt(3) in the root of the mean square: sqrt(2 / 3) 2^-8 = 3.2e-3 of a row's norm together.  A row's
own error scatters about that (a hundred columns or more; h's few largest values count most): half as much again is
allowed.  A column of h left out of 2048 is 2.2e-2.
"""
import numpy as np
import pytest
import torch

from gpu_cases import log, require_gpu
from test_gpu_ffn_w4 import Stack, route, run, weights_of
from w4_cases import packed

pytestmark = pytest.mark.gpu
BIG = 5  # the column of 256


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def whole_matrix(g, rows, cols):
    """Codes, scale bytes and values [rows, cols] (fp32, on the device): about 256 values of +-1 and +-2 a row, zeros else."""
    some = torch.rand((rows, cols), generator=g, device="cuda") < min(0.5, 256 / cols)
    two = torch.randint(0, 2, (rows, cols), generator=g, device="cuda", dtype=torch.uint8)
    sign = torch.randint(0, 2, (rows, cols), generator=g, device="cuda", dtype=torch.uint8)
    up = torch.randint(0, 3, (rows, cols // 32), generator=g, device="cuda", dtype=torch.uint8)  # scale 2^(up - 1)
    return some, two, sign, up


def coded(some, two, sign, up):
    """1 and 2 under a scale of 1/2: 2, 4; of 1: 1, 2; of 2: 1/2, 1."""
    codes = torch.tensor([[4, 6], [2, 4], [1, 2]], dtype=torch.uint8, device="cuda")
    c = codes[up.repeat_interleave(32, 1).long(), two.long()] | sign << 3
    c = torch.where(some, c, torch.zeros_like(c))
    value = (1.0 + two.float()) * (1.0 - 2.0 * sign.float()) * some.float()
    return (c[:, 0::2] | c[:, 1::2] << 4).contiguous(), (126 + up).contiguous(), value


class WholeStack:
    def __init__(self, moe, seed, h, i, e):
        self.dims = (h, i, e)
        g = torch.Generator(device="cuda").manual_seed(seed)
        self.packed, self.values = [], []
        for name, rows, cols in (("gate", i, h), ("up", i, h), ("down", h, i)):
            q, s, v = [], [], []
            for _ in range(e):
                some, two, sign, up = whole_matrix(g, rows, cols)
                if name != "down":
                    some[:, BIG] = name == "gate"
                    two[:, BIG], sign[:, BIG] = 0, 0
                one = coded(some, two, sign, up)
                for to, what in zip((q, s, v), one):
                    to.append(what)
            self.packed += packed(moe, torch.stack(q).cpu().numpy(), torch.stack(s).cpu().numpy())
            self.values.append(v)

    def rows(self, e, x):
        """y [n, H] (fp64, whole) of x [n, H] through expert e."""
        wg, wu, wd = (v[e].double() for v in self.values)
        g, u = x @ wg.t(), x @ wu.t()
        assert (g >= 32).all() and ((g * u).abs() < 2 ** 24).all()
        h = (g * u).float().bfloat16().double()
        assert (h.abs() @ wd.abs().t() < 2 ** 24).all()
        return h @ wd.t()


def exact_case(moe, h, i, e, k, tokens, skew):
    rng = np.random.default_rng(h + 3 * i + e + tokens)
    stack = WholeStack(moe, h + i + tokens, h, i, e)
    x = torch.from_numpy(rng.integers(0, 2, (tokens, h)).astype(np.float32) * 2 - 1)
    x[:, BIG] = 256.0
    ids = route(rng, tokens, e, k, skew)
    p = torch.from_numpy(2.0 ** -rng.integers(0, 3, (tokens, k)).astype(np.float32))
    ref, size = torch.zeros((tokens, h), dtype=torch.float64), torch.zeros((tokens, h), dtype=torch.float64)
    for ex in ids.unique().tolist():
        t, j = (ids == ex).nonzero(as_tuple=True)
        y = stack.rows(ex, x[t].double().cuda()).cpu() * p[t, j].double()[:, None]
        ref.index_add_(0, t, y)
        size.index_add_(0, t, y.abs())
    assert (size < 2 ** 22).all() and float(ref.abs().mean()) > 100
    ref = ref.float().bfloat16()
    x = x.bfloat16()
    print(f"H={h} I={i} E={e} k={k} T={tokens}", flush=True)
    for fused in (True, False):
        out, buf = run(moe, stack, x, ids, p, fused)
        differs = (out.cpu() != ref).nonzero()
        assert len(differs) == 0, (fused, len(differs), differs[:4].tolist())
    assert torch.isfinite(buf.y_rows).all()


FEW = [  # slots up to 64: sorted by the gate/up launch, down and combine in one where the slots' h fits LDS
    (7168, 2048, 4, 3, 1, 0.0), (7168, 2048, 4, 2, 8, 0.5), (7168, 2048, 3, 2, 12, 0.0), (4224, 640, 4, 2, 3, 0.0),
    (4352, 384, 3, 1, 9, 1.0), (8064, 256, 3, 2, 5, 0.0), (8192, 1152, 2, 2, 2, 0.0), (640, 4224, 3, 2, 2, 0.0),
    (256, 8064, 2, 1, 2, 0.0), (384, 8192, 2, 2, 1, 0.0), (128, 128, 2, 1, 1, 0.0), (512, 2176, 4, 2, 4, 0.0),
    (1152, 896, 5, 4, 16, 0.3), (2048, 768, 16, 8, 8, 0.0), (256, 128, 64, 32, 2, 0.0)]


@pytest.mark.parametrize("h,i,e,k,tokens,skew", FEW)
def test_a_few_slots(moe, h, i, e, k, tokens, skew):
    exact_case(moe, h, i, e, k, tokens, skew)


# More slots: up to eight rows an expert by the few-rows kernel (all its lengths of K), above it by the GEMM, narrow and wide
# tiles of every number of rows up to 160.
MORE = [(7168, 2048, 4, 2, 13, 0.0), (7168, 2048, 6, 2, 24, 1.0), (4224, 640, 12, 4, 24, 1.5), (4352, 384, 12, 4, 23, 0.5),
        (8064, 256, 9, 8, 9, 0.0), (8192, 1152, 9, 8, 9, 0.0), (512, 2176, 17, 8, 17, 0.5), (256, 8064, 9, 8, 9, 0.0),
        (128, 8192, 9, 8, 9, 0.0), (7168, 2048, 4, 2, 100, 0.0), (7168, 1280, 3, 1, 450, 0.1), (4224, 640, 4, 2, 310, 0.0),
        (1152, 896, 4, 2, 130, 1.0), (640, 4224, 3, 2, 240, 0.0), (8064, 384, 2, 1, 50, 0.5), (512, 8192, 2, 1, 300, 0.0),
        (384, 256, 40, 8, 150, 0.2), (2048, 768, 24, 8, 200, 0.0), (2048, 768, 24, 8, 440, 0.0), (1024, 512, 64, 8, 250, 0.05),
        (1024, 1024, 64, 8, 460, 0.02), (1024, 512, 64, 8, 700, 0.01), (1024, 512, 64, 8, 1100, 0.0), (1024, 2048, 64, 8, 1240, 0.0)]


@pytest.mark.parametrize("h,i,e,k,tokens,skew", MORE)
def test_more_slots(moe, h, i, e, k, tokens, skew):
    exact_case(moe, h, i, e, k, tokens, skew)


LONG = [(8320, 256, 3, 2), (256, 8320, 3, 2), (8448, 8320, 2, 1), (12288, 384, 2, 2), (384, 16384, 2, 1)]


@pytest.mark.parametrize("tokens", [1, 5, 33, 90])
@pytest.mark.parametrize("h,i,e,k", LONG)
def test_rows_longer_than_the_few_rows_kernel_holds(moe, h, i, e, k, tokens):
    """Experts whose hidden or inner size is above 8192: any number of slots goes by the sort and the GEMM there."""
    exact_case(moe, h, i, e, k, tokens, 0.3)


ORDINARY = [(7168, 2048, 4, 2, 1, 0.0), (7168, 2048, 4, 2, 16, 0.0), (7168, 1280, 3, 1, 40, 0.5), (4096, 2176, 2, 2, 7, 0.0),
            (256, 2048, 8, 8, 2, 0.0), (2048, 768, 16, 8, 70, 0.3), (2048, 4096, 5, 2, 150, 0.3), (4352, 640, 3, 2, 400, 0.0),
            (8320, 1152, 2, 1, 60, 0.0)]


@pytest.mark.parametrize("h,i,e,k,tokens,skew", ORDINARY)
def test_the_error_of_every_row(moe, h, i, e, k, tokens, skew):
    rng = np.random.default_rng(h + i + tokens)
    stack = Stack(moe, rng, h, i, e)
    x = torch.from_numpy(rng.standard_normal((tokens, h)).astype(np.float32)).bfloat16()
    ids, p = route(rng, tokens, e, k, skew), weights_of(rng, tokens, k)
    ref, kept = (torch.zeros((tokens, h), dtype=torch.float64) for _ in range(2))
    for ex in ids.unique().tolist():
        t, j = (ids == ex).nonzero(as_tuple=True)
        wg, wu, wd = (v[ex] for v in stack.values)
        rows = x[t].double().cuda()
        g, u = rows @ wg.t(), rows @ wu.t()
        mid = g * torch.sigmoid(g) * u
        w = p[t, j].double()[:, None]
        ref.index_add_(0, t, (mid @ wd.t()).cpu() * w)
        kept.index_add_(0, t, (mid.bfloat16().double() @ wd.t()).cpu() * w)

    def error(a, b):
        return float(((a - b).norm(dim=1) / b.norm(dim=1)).max())
    for fused in (True, False):
        out = run(moe, stack, x, ids, p, fused)[0].double().cpu()
        off, own = error(out, ref), error(out, kept)
        log(f"H={h} I={i} E={e} k={k} T={tokens}: {off:.2e} of a row, {own:.2e} with h rounded in the formula too")
        assert off <= 1.5 * (2 / 3) ** 0.5 * 2.0 ** -8
        # what is left beside h's rounding is the output's, and an h here and there that falls to the other side
        assert own <= 1.5 * 3 ** -0.5 * 2.0 ** -8
