"""Sizes at the ends of their types, through the C ABI (CPU; every call returns before anything is launched)."""
import ctypes

import pytest

import paper_2606_10493_amd as moe

A = ctypes.c_void_p(0x10000)  # a stand-in for device addresses, never followed
MOST = 2 ** 31 - 16           # the most columns


@pytest.mark.parametrize("tokens", [100000, 2 ** 31 - 1])
def test_too_many_rows_and_columns(tokens):
    """More workgroups than a launch has; the number of column tiles is not taken round the end of 32 bits."""
    st = moe.lib.moe_linear_w4(A, 128, tokens, 128, A, A, MOST, None, A, MOST, moe.MOE_BF16, A, 1 << 62, None)
    assert st == moe.MOE_ERR_UNSUPPORTED_SHAPE, moe.moe_last_error()
    d = moe.MoeDims(128, 2 ** 31 - 128, 1024, 8)
    rows = min(tokens, (2 ** 31 - 1) // 8)
    st = moe.lib.moe_expert_ffn_w4(d, rows, A, A, A, A, A, A, A, A, A, A, A, 1 << 63, None)
    assert st == moe.MOE_ERR_UNSUPPORTED_SHAPE, moe.moe_last_error()
