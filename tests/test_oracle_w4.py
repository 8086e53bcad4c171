"""The oracle of the 4-bit weights against their format (CPU)."""
import numpy as np
import pytest

from oracle import w4_oracle as wo


def test_e2m1_values_follow_the_format():
    """Sign, two bits of exponent with bias 1, one of mantissa, subnormals at exponent 0."""
    for code in range(16):
        exponent, mantissa = code >> 1 & 3, code & 1
        size = mantissa / 2 if exponent == 0 else (1 + mantissa / 2) * 2.0 ** (exponent - 1)
        assert wo.E2M1[code] == (-size if code & 8 else size)


def test_quantized_groups_take_the_smallest_scale_and_the_nearest_code():
    rng = np.random.default_rng(3)
    w = (rng.standard_normal((40, 64)) * np.exp(3 * rng.standard_normal((40, 1)))).astype(np.float32)
    q, s = wo.quantize(w)
    v = wo.values(q, s).reshape(40, 2, 32)
    x = w.astype(np.float64).reshape(40, 2, 32)
    scale = 2.0 ** (s.astype(np.float64) - 127)
    top = np.abs(x).max(-1)
    assert (top <= 7 * scale).all() and (top > 3.5 * scale).all()
    # nearest, and never more than half a step of the codes' grid off (steps of 2 up to 8, where 7 is the last)
    grid = np.unique(wo.E2M1)
    near = np.abs(x[..., None] - grid * scale[..., None, None]).min(-1)
    assert np.array_equal(np.abs(v - x), near)
    assert (np.abs(v - x) <= scale[..., None]).all()


@pytest.mark.parametrize("value,code", [(0.25, 0), (0.75, 2), (1.25, 2), (1.75, 4), (2.5, 4), (3.5, 6), (5.0, 6), (7.0, 7),
                                        (-0.25, 8), (-0.0, 8), (-7.0, 15)])
def test_ties_and_ends(value, code):
    w = np.zeros((1, 32), np.float32)
    w[0, 0], w[0, 31] = value, 7.0   # scale 1
    q, s = wo.quantize(w)
    assert s[0, 0] == 127 and q[0, 0] & 15 == code and q[0, 15] >> 4 == 7


def test_scales_end_at_their_limits():
    w = np.zeros((3, 32), np.float32)
    w[1, 0], w[2, 0] = 2.0 ** -149, 3e38
    q, s = wo.quantize(w)
    assert s[:, 0].tolist() == [7, 7, 247] and q[1, 0] & 15 == 0 and q[2, 0] & 15 == 7


def test_packed_places_are_a_permutation():
    rows, cols = 32, 640
    q = np.arange(rows * cols // 2, dtype=np.int64)
    rng = np.random.default_rng(4)
    q = rng.integers(0, 256, (rows, cols // 2)).astype(np.uint8)
    s = rng.integers(0, 253, (rows, cols // 32)).astype(np.uint8)
    packed, scales = wo.pack(q, s)
    assert np.array_equal(np.sort(packed), np.sort(q.reshape(-1)))
    assert scales.size == rows // 16 * 2 * 256
    # lane 16 kq + r of tile (1, 3), dword 2: row 16 + r, columns 128 * 3 + 64 + 8 kq
    kq, r, j = 3, 5, 2
    at = (1 * 5 + 3) * 1024 + 16 * (16 * kq + r) + 4 * j
    assert np.array_equal(packed[at:at + 4], q[21, (384 + 64 + 24) // 2:][:4])
    assert scales[(1 * 2 + 1) * 256 + 16 * 5 + 3] == s[21, 19]
    assert (scales[(1 * 2 + 1) * 256 + 16 * 5 + 4:][:12] == 127).all()


def test_norm_against_its_parts():
    rng = np.random.default_rng(5)
    x, r, w = rng.standard_normal((3, 7, 64))
    z, y = wo.add_norm(x, r, w[0], 1e-5, 1.0)
    assert np.array_equal(z, x + r)
    for t in range(7):
        mean = sum(float(v) ** 2 for v in z[t]) / 64
        assert np.allclose(y[t], z[t] / (mean + 1e-5) ** 0.5 * (1 + w[0]), rtol=1e-14)
