"""Sizes that the many-class entry points refuse because no launch holds them, seen on the host: the refusal comes before any work on a device."""
import ctypes

import pytest

from paper_1708_04801_amd import api

GB = 1 << 30            # addresses that no call gets as far as using


@pytest.mark.parametrize("rows_a,rows_b", [(4, 1 << 33), (1 << 33, 4), (1, 1 << 32), (100, 1 << 33), (1 << 33, 3000)])
@pytest.mark.parametrize("dtype", [api.F32, api.BF16])
def test_products_of_more_workgroups_than_a_launch_has(rows_a, rows_b, dtype):
    a, b = (api._CBlocks(r, 128, GB, 128, GB, 4) for r in (rows_a, rows_b))
    assert api.load().wpsgd_block_matmul(ctypes.byref(a), ctypes.byref(b), GB, rows_b, dtype, None, 0, None) == api.UNSUPPORTED


def test_products_of_wide_rows_on_both_sides():
    a, b = (api._CBlocks(5_000_000, 128, GB, (1 << 22) + 16, GB, 4) for _ in range(2))
    assert api.load().wpsgd_block_matmul(ctypes.byref(a), ctypes.byref(b), GB, 5_000_000, api.F32, None, 0, None) == api.UNSUPPORTED
