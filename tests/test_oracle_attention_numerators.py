"""The oracle's bound for numerators of two bf16 each tells them from single ones (CPU)."""
import numpy as np
import pytest
import torch

from oracle import attention_oracle as ao


def bf16(x):
    return torch.from_numpy(x).bfloat16().double().numpy()


@pytest.mark.parametrize("n", [3, 40, 300])
def test_two_bf16_stay_within_the_bound_and_one_does_not(n):
    rng = np.random.default_rng(n)
    q, k, v = (rng.standard_normal((m, 64)) for m in (60, n, n))
    ref, bound = ao.attention(q, k, v, 0.125, numerators=ao.TWO_BF16_ROUNDOFF)
    assert np.array_equal(ref, ao.attention(q, k, v, 0.125)[0]) and np.all(bound < ao.attention(q, k, v, 0.125)[1])
    s = 0.125 * q @ k.T
    p = np.exp(s - s.max(1, keepdims=True))
    total = p.sum(1, keepdims=True)
    one = bf16(p)
    two = one + bf16(p - one)
    ratio = {name: np.max(np.abs(bf16(x @ v / total) - ref) / bound) for name, x in (("one", one), ("two", two))}
    assert ratio["two"] <= 1.0 < ratio["one"], ratio
