"""GPU: the attention calls put together as a layer uses them, against the oracle chained the same way; and the example."""
import importlib.util
import math
import os

import numpy as np
import pytest
import torch

import oracle
from attention_cases import bf16, offsets
from gpu_cases import log, require_gpu
from oracle import attention_oracle as ao

pytestmark = pytest.mark.gpu
ROOT = os.path.dirname(os.path.dirname(os.path.abspath(__file__)))


@pytest.fixture(scope="module")
def moe():
    return require_gpu()


def ints(x):
    return torch.from_numpy(np.asarray(x, np.int32)).cuda()


def test_prompts_then_steps(moe):
    """run_attention on two packed prompts and then three steps.  The oracle rotates in fp32 (bit for bit the library's
    rows), takes bf16 rows for the prompt and the cached e4m3 rows for the steps."""
    rng = np.random.default_rng(41)
    hq, hkv, dim, page = 8, 2, 64, 16
    d = moe.MoeAttnDims(hq, hkv, dim)
    lens, n_steps = [37, 18], 3
    cu, scale = offsets(lens), 1 / math.sqrt(dim)
    table = ao.rope_table(100, ao.rope_frequencies(32, 10000.0))
    dev_table = torch.from_numpy(table).cuda()
    width = 4
    pages = rng.permutation(2 * width).reshape(2, width).astype(np.int32)
    cache = moe.KVCache.empty(2 * width, hkv, page, dim)
    cache.k.fill_(0x7F)
    cache.v.fill_(0x7F)

    def qkv(n):
        return [bf16(rng.standard_normal((n, h, dim))) for h in (hq, hkv, hkv)]

    def slot(b, t):
        return pages[b, t // page] * page + t % page
    (q, qv), (k, kv), (v, vv) = qkv(sum(lens))
    pos = np.concatenate([np.arange(n) for n in lens])
    buf = moe.AttentionBuffers(d, 2, max(lens), tokens=sum(lens))
    out = moe.run_attention(buf, q, k, v, ints(pos), dev_table, ints([slot(b, t) for b in range(2) for t in range(lens[b])]),
                            cache, scale, cu=ints(cu))
    torch.cuda.synchronize()

    def rounded(x):
        return oracle.bf16_to_f32(oracle.f32_to_bf16(x)).astype(np.float64)
    rq, rk = (ao.rotate(x.astype(np.float32), table[pos], False) for x in (qv, kv))
    ref, bound = ao.packed_attention(rounded(rq), rounded(rk), vv, cu, cu, scale, True)
    worst = float(np.max(np.abs(out.double().cpu().numpy() - ref) / bound))
    log(f"prompts: {worst:.3f} of the bound")
    assert worst <= 1 and int(buf.dev_status.item()) == 0
    held = [[list(x) for x in np.split(ao.cached_rows(*ao.quantize_head_rows(y.astype(np.float32))), cu[1:-1])]
            for y in (rk, vv)]

    step = moe.AttentionBuffers(d, 2, max(lens) + n_steps)
    for i in range(n_steps):
        (q, qv), (k, kv), (v, vv) = qkv(2)
        at = np.array([n + i for n in lens])
        out = moe.run_attention(step, q, k, v, ints(at), dev_table, ints([slot(b, at[b]) for b in range(2)]), cache, scale,
                                page_table=ints(pages), lens=ints(at + 1))
        torch.cuda.synchronize()
        rq, rk = (ao.rotate(x.astype(np.float32), table[at], False) for x in (qv, kv))
        for h, y in zip(held, (rk, vv)):
            rows = ao.cached_rows(*ao.quantize_head_rows(y.astype(np.float32)))
            for b in range(2):
                h[b].append(rows[b])
        for b in range(2):
            keys, values = (np.stack(h[b]) for h in held)
            for head in range(hq):
                g = head // (hq // hkv)
                ref, bound = ao.attention(rounded(rq)[b, head][None], keys[:, g], values[:, g], scale)
                err = np.abs(out[b, head].double().cpu().numpy() - ref[0]) / bound[0]
                assert err.max() <= 1, (i, b, head, err.max())
    assert int(step.dev_status.item()) == 0


def test_example_steps_agree_with_its_prompts(moe):
    """The example's layer: a token computed by a step, behind a shared prefix in the cache, against the same token as the
    last of its prompt.  The step's own part is the cache's e4m3 rows where the prompt's was bf16: a row is off by 2.6 % of
    its norm (uniform rounding within e4m3's 3 bits), scores of unit size by as much of themselves, and the layer adds the
    attention's result to a residual of its own size, so the hidden states differ by a few percent at most."""
    spec = importlib.util.spec_from_file_location("decoder_layer", os.path.join(ROOT, "examples", "decoder_layer.py"))
    ex = importlib.util.module_from_spec(spec)
    spec.loader.exec_module(ex)
    g = torch.Generator(device="cuda").manual_seed(3)

    def tokens(n):
        return torch.randn((n, ex.HIDDEN), generator=g, device="cuda").bfloat16()
    layer, prefix, prompts = ex.Layer(), tokens(100), [tokens(70), tokens(33)]
    new = tokens(2)
    by_step = ex.run(layer, prefix, prompts, [new])[1]
    longer = [torch.cat([p, new[i:i + 1]]) for i, p in enumerate(prompts)]
    whole = ex.run(layer, prefix, longer, [])[0]
    by_prompt = whole[[70, 70 + 34]]
    off = ((by_step - by_prompt).float().norm() / by_prompt.float().norm()).item()
    log(f"step against prompt: {off:.4f}")
    assert off < 0.1
