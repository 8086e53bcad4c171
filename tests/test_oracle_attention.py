"""The attention-side oracle against something other than itself (CPU)."""
import numpy as np
import pytest
import torch

import oracle
from oracle import attention_oracle as ao


def test_plain_and_linear_frequencies():
    f = ao.rope_frequencies(8, 10000.0)
    assert np.allclose(f, [1.0, 0.1, 0.01, 0.001], rtol=1e-15)
    assert np.allclose(ao.rope_frequencies(8, 10000.0, "linear", factor=4.0), f / 4, rtol=1e-15)


def test_frequencies_by_parts_have_their_limits():
    """Pairs that turn often over the original context keep their frequency, those that hardly turn are interpolated, and
    the mix is linear in the number of turns."""
    kw = dict(factor=8.0, original_len=2 * np.pi * 100, slow_turns=1.0, fast_turns=33.0)
    plain, mixed = ao.rope_frequencies(32, 1e6), ao.rope_frequencies(32, 1e6, "by_parts", **kw)
    turns = 100 * plain
    assert np.array_equal(mixed[turns >= 33], plain[turns >= 33]) and (turns >= 33).any()
    assert np.allclose(mixed[turns <= 1], plain[turns <= 1] / 8, rtol=1e-15) and (turns <= 1).any()
    between = (turns > 1) & (turns < 33)
    assert between.any()
    w = (turns[between] - 1) / 32
    assert np.allclose(mixed[between], plain[between] * (w + (1 - w) / 8), rtol=1e-14)


@pytest.mark.parametrize("interleaved", [False, True])
def test_rotation_is_a_rotation(interleaved):
    """Against complex products in 64 bits; the rest of the head is kept; scores depend on distance alone."""
    rng = np.random.default_rng(0)
    table = ao.rope_table(500, ao.rope_frequencies(16, 10000.0))
    x = rng.standard_normal((6, 3, 24)).astype(np.float32)
    pos = np.array([0, 1, 7, 100, 499, 3])
    y = ao.rotate(x, table[pos], interleaved)
    assert np.array_equal(y[..., 16:], x[..., 16:]) and np.array_equal(y[0], x[0])
    a, b = (x[..., 0:16:2], x[..., 1:16:2]) if interleaved else (x[..., :8], x[..., 8:16])
    z = (a + 1j * b) * np.exp(1j * pos[:, None, None] * ao.rope_frequencies(16, 10000.0))
    u, w = (y[..., 0:16:2], y[..., 1:16:2]) if interleaved else (y[..., :8], y[..., 8:16])
    assert np.abs(u - z.real).max() < 1e-5 and np.abs(w - z.imag).max() < 1e-5
    q, k = x[:1, :1], x[1:2, :1]

    def score(m, n):
        return float(np.sum(ao.rotate(q, table[[m]], interleaved) * ao.rotate(k, table[[n]], interleaved)))
    assert abs(score(17, 5) - score(412, 400)) < 1e-4


def test_head_rows_are_the_activation_quantizers_at_its_block():
    """At 128 elements a head's row is one block of the activation quantizer."""
    rng = np.random.default_rng(1)
    x = (rng.standard_normal((40, 128)) * np.exp(3 * rng.standard_normal((40, 1)))).astype(np.float32)
    x[3] = 0
    q, s = ao.quantize_head_rows(x)
    q2, s2 = oracle.quantize_rows(x)
    assert np.array_equal(q, q2) and np.array_equal(s, s2[:, 0])
    err = np.abs(ao.cached_rows(q, s).astype(np.float64) - x)
    assert np.all(err <= np.maximum(np.abs(x) * 2.0 ** -4, s[:, None] * 2.0 ** -10) * (1 + 1e-6))


@pytest.mark.parametrize("causal", [False, True])
def test_attention_against_torch(causal):
    rng = np.random.default_rng(2)
    q, k, v = (rng.standard_normal((n, h, 8)) for n, h in ((9, 4), (12, 2), (12, 2)))
    cu_q, cu_k = [0, 5, 9], [0, 7, 12]
    out, bound = ao.packed_attention(q, k, v, cu_q, cu_k, 0.4, causal)
    for b in range(2):
        a, z, c, e = cu_q[b], cu_q[b + 1], cu_k[b], cu_k[b + 1]
        tq = torch.from_numpy(q[a:z]).transpose(0, 1)
        tk, tv = (torch.from_numpy(np.repeat(x[c:e], 2, axis=1)).transpose(0, 1) for x in (k, v))
        mask = torch.ones(z - a, e - c, dtype=torch.bool).tril((e - c) - (z - a)) if causal else None
        ref = torch.nn.functional.scaled_dot_product_attention(tq, tk, tv, attn_mask=mask, scale=0.4)
        assert np.allclose(out[a:z], ref.transpose(0, 1).numpy(), atol=1e-13)
    assert (bound > 0).all()


def test_rows_without_keys_give_zeros_and_rows_outside_are_marked():
    rng = np.random.default_rng(3)
    q, k = rng.standard_normal((6, 1, 8)), rng.standard_normal((2, 1, 8))
    out, _ = ao.packed_attention(q, k, k, [1, 5], [0, 2], 1.0, True)
    assert np.isnan(out[[0, 5]]).all()
    assert not out[1:3].any() and np.allclose(out[3, 0], k[0, 0])
    assert not ao.attention(q[:, 0], k[:0, 0], k[:0, 0], 1.0)[0].any()


def test_the_bound_covers_its_roundings_and_little_more():
    """An attention with the definition's roundings (bf16 numerators and result) stays within the bound and comes near."""
    rng = np.random.default_rng(4)
    q, k, v = (rng.standard_normal((n, 64)) for n in (50, 300, 300))
    ref, bound = ao.attention(q, k, v, 0.125)
    s = 0.125 * q @ k.T
    p = torch.from_numpy(np.exp(s - s.max(1, keepdims=True)))
    out = (p.bfloat16().double() @ torch.from_numpy(v) / p.sum(1, keepdim=True)).bfloat16().double().numpy()
    ratio = np.abs(out - ref) / bound
    assert 0.1 < ratio.max() <= 1
