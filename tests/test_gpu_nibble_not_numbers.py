"""Rows times 4-bit matrices: what is not a number stays none, in every kernel."""
import math

import pytest
import torch

from paper_1708_04801_amd import api
from test_gpu_nibble_parts import matrix

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("n,classes,d", [(3, 33000, 300), (5, 4200, 4093), (7, 17000, 300), (6, 17000, 2305), (20, 33000, 300), (70, 17000, 300), (3, 40, 300), (37, 40, 300)])
def test_what_is_not_a_number_stays_none(n, classes, d):
    """whichever bits say so, the quiet one or one among the lowest: such a row has no numbers, one with an infinity as its only such element infinities (beside weights that are
    not 0), and the others are what they are"""
    q, value = matrix(classes, d, 64, d)
    g = torch.Generator().manual_seed(n)
    x = torch.randn(n, d, generator=g)
    want = api.wpsgd_nibble_matmul(api.Matrix(n, d, dense=x.cuda()), q, dtype=torch.float32)
    for column in (3, 200, d - 1):
        for bits in (0x7F800001, 0x7F80FFFF, 0x7FC00000, 0x7FFFFFFF, 0x7FBF0000, 0xFF800001 - (1 << 32), 0xFFC00001 - (1 << 32)):
            y = x.clone()
            y.view(torch.int32)[1, column] = bits
            y = api.wpsgd_nibble_matmul(api.Matrix(n, d, dense=y.cuda()), q, dtype=torch.float32)
            assert torch.isnan(y[1]).all() and torch.equal(y[0], want[0]) and torch.equal(y[2:], want[2:])
        y = x.clone()
        y[1, column] = -math.inf
        y = api.wpsgd_nibble_matmul(api.Matrix(n, d, dense=y.cuda()), q, dtype=torch.float32)
        w = value[:, column]
        assert torch.isnan(y[1][w == 0]).all() and torch.equal(y[1][w > 0], torch.full_like(y[1][w > 0], -math.inf)) and torch.equal(y[1][w < 0], torch.full_like(y[1][w < 0], math.inf))
        assert torch.equal(y[0], want[0]) and torch.equal(y[2:], want[2:])


@pytest.mark.parametrize("n,classes,d", [(3, 33000, 300), (12, 4200, 4093), (7, 17000, 9000), (20, 33000, 300), (70, 17000, 300), (3, 40, 300), (37, 40, 300)])
def test_what_is_not_a_number_in_bfloat16_stays_none(n, classes, d):
    q, _ = matrix(classes, d, 32, d)
    x = torch.randn(n, d, generator=torch.Generator().manual_seed(n)).bfloat16()
    want = api.wpsgd_nibble_matmul(api.Matrix(n, d, dense=x.cuda()), q, dtype=torch.float32)
    for column in (3, 200, d - 1):
        for bits in (0x7F81, 0x7FC0, 0x7FFF, 0x7FA0, 0xFF81 - (1 << 16), 0xFFC1 - (1 << 16)):
            y = x.clone()
            y.view(torch.int16)[1, column] = bits
            y = api.wpsgd_nibble_matmul(api.Matrix(n, d, dense=y.cuda()), q, dtype=torch.float32)
            assert torch.isnan(y[1]).all() and torch.equal(y[0], want[0]) and torch.equal(y[2:], want[2:])
