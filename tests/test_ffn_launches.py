"""How large the launches of the feed-forward calls can be (no GPU needed)."""
import ctypes

import pytest

import mm_routes as R


def check_sum_blocks(rows, cols):
    f = R._lib().fp8lin_check_sum_blocks
    f.restype, f.argtypes = ctypes.c_int64, [ctypes.c_int64] * 2
    return f(rows, cols)


@pytest.mark.parametrize("rows", [1, 17, 4096])
@pytest.mark.parametrize("cols", [1, 64, 65, 5120, 1 << 22, 1 << 30, (1 << 31) - 512])
def test_the_launch_that_checks_codes_and_adds_sums_can_be_counted(rows, cols):
    """Fewer than 2^32 threads whatever the columns, and a workgroup for every 64 of them up to 2^22."""
    blocks = check_sum_blocks(rows, cols)
    assert blocks * 256 < 1 << 32
    assert blocks > (-(-cols // 64) if cols <= 1 << 22 else 0)
