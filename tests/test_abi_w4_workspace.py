"""What moe_linear_w4_workspace asks for, against what calls need (CPU; nothing is launched).

A call looks at the workspace's size before its alignment, so that one with a misaligned workspace is refused for its size
(MOE_ERR_WORKSPACE) or, where that is enough, for its alignment (MOE_ERR_INVALID_ARG).
"""
import ctypes
import random

import pytest

import paper_2606_10493_amd as moe

P = ctypes.c_void_p
A, ODD = P(0x10000), P(0x10080)  # stand-ins for device addresses, never followed


def enough(t, k, n, size):
    st = moe.lib.moe_linear_w4(A, k, t, k, A, A, n, None, A, n + n % 8, moe.MOE_F32, ODD, size, None)
    assert st in (moe.MOE_ERR_WORKSPACE, moe.MOE_ERR_INVALID_ARG)
    return st == moe.MOE_ERR_INVALID_ARG


def needed(t, k, n):
    """The smallest size that a call takes."""
    low, high = 0, 16 * max(t, 1024) * n * 4 + 256
    assert enough(t, k, n, high)
    while low < high:
        mid = (low + high) // 2
        low, high = (low, mid) if enough(t, k, n, mid) else (mid + 1, high)
    return low


@pytest.mark.parametrize("k", [128, 256, 640, 2048, 4096, 7168, 8192])
@pytest.mark.parametrize("n", [65536, 129280])
def test_nothing_is_asked_where_k_stays_whole(k, n):
    for t in (1, 16, 17, 24, 33, 64, 65, 100, 128, 200, 256, 257, 400, 512, 513, 1000, 8192):
        assert moe.moe_linear_w4_workspace(t, k, n) == 0
        assert enough(t, k, n, 0)


@pytest.mark.parametrize("n", [16, 1536, 4096, 7168])
def test_nothing_is_asked_for_a_short_k(n):
    """Parts have three blocks of K at least, so that six are the fewest that are cut."""
    for k in (128, 512, 640):
        for t in (17, 40, 100, 512, 2000):
            assert moe.moe_linear_w4_workspace(t, k, n) == 0


def test_what_is_asked_is_enough_and_nearly_needed():
    """For every smaller call too; and some call of up to that many rows needs most of it: 15 rows more at most are counted
    for a call of 17 rows or more."""
    rng = random.Random(5)
    for _ in range(60):
        k = 128 * int(2 ** rng.uniform(0, 10))
        n = 16 * int(2 ** rng.uniform(0, 12))
        top = rng.choice((rng.randint(1, 16), rng.randint(17, 128), rng.randint(129, 520), 4000))
        asked = moe.moe_linear_w4_workspace(top, k, n)
        most, most_rows = 0, 0
        for t in sorted({rng.randint(1, top) for _ in range(20)} | {1, min(top, 16), top}):
            assert enough(t, k, n, asked), (t, k, n)
            assert moe.moe_linear_w4_workspace(t, k, n) <= asked
            most = max(most, needed(t, k, n))
        for t in range(1, min(top, 512) + 1) if asked else ():
            if moe.moe_linear_w4_workspace(t, k, n) == asked:
                most_rows = max(most_rows, t)
                most = max(most, needed(t, k, n))
                break
        assert most <= asked and (asked == 0 or asked <= 2 * most), (top, k, n, asked, most)


def test_sizes_of_ordinary_projections():
    """4096 x 4096 asked for 16.8 MB at 64 rows."""
    for t in (17, 64, 100, 201, 512, 4096):
        assert moe.moe_linear_w4_workspace(t, 4096, 4096) <= 16.8e6 / 3
    assert moe.moe_linear_w4_workspace(24, 7168, 65536) == 0
    # 16 parts of a long K, a launch behind the first joins them
    assert needed(2, 65536, 32) == 16 * 2 * 32 * 4 <= moe.moe_linear_w4_workspace(2, 65536, 32)
    assert needed(17, 65536, 32) == 16 * 17 * 32 * 4
