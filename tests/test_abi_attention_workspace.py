"""The attention calls' workspace queries: one that serves the largest call serves every smaller one (CPU)."""
import math
import random

import pytest

import paper_2606_10493_amd as moe

HEADS = [(32, 8, 128), (8, 2, 128), (64, 8, 128), (16, 16, 64), (16, 1, 128), (40, 2, 64), (1024, 8, 128), (1, 1, 64)]


def log_uniform(rng, most):
    return int(round(math.exp(rng.uniform(0.0, math.log(most)))))


@pytest.mark.parametrize("dims", HEADS)
def test_a_larger_prompt_call_never_needs_less(dims):
    d, rng = moe.MoeAttnDims(*dims), random.Random(61)

    def need(batch, tokens, longest):
        return moe.moe_attn_prefill_workspace(d, batch, tokens, longest)
    for longest in (63, 64, 1000, 8701, 100000):
        sizes = [need(1, t, longest) for t in [*range(1, 700), *range(700, 9000, 37)]]
        assert sizes == sorted(sizes), longest
    for tokens in (1, 64, 509, 2048, 8192):
        sizes = [need(1, tokens, n) for n in range(0, 12000, 16)]
        assert sizes == sorted(sizes), tokens
        sizes = [need(b, tokens, 3000) for b in range(1, 130)]
        assert sizes == sorted(sizes), tokens
    for _ in range(3000):
        a = [log_uniform(rng, m) for m in (300, 60000, 1000000)]
        b = [x + rng.choice((0, 0, 1, log_uniform(rng, m))) for x, m in zip(a, (300, 60000, 1000000))]
        assert need(*a) <= need(*b), (a, b)


@pytest.mark.parametrize("dims", HEADS)
def test_a_larger_batch_or_prefix_never_needs_less(dims):
    d, rng = moe.MoeAttnDims(*dims), random.Random(62)

    def need(batch, longest, prefix):
        return moe.moe_attn_decode_workspace(d, batch, longest, prefix)
    for longest in (0, 100, 500, 768, 1024, 1500, 2048, 4000, 9000):
        for prefix in (0, 120, 1500, 8191):
            sizes = [need(b, longest, prefix) for b in [*range(1, 129), 200, 384, 500, 1000, 5000]]
            assert sizes == sorted(sizes), (longest, prefix)
        for batch in (1, 8, 48):
            sizes = [need(batch, longest, p) for p in range(0, 3000, 43)]
            assert sizes == sorted(sizes), (longest, batch)
    for _ in range(3000):
        a = [log_uniform(rng, m) for m in (300, 20000, 20000)]
        b = [x + rng.choice((0, 0, 1, log_uniform(rng, m))) for x, m in zip(a, (300, 20000, 20000))]
        assert need(*a) <= need(*b), (a, b)
        assert need(a[0], a[1], 0) <= need(*a)
