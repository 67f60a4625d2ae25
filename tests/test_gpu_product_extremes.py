"""Products of blocks at the ends of fp32's exponents, through every kernel: exact where the elements' values and the result are exact, infinite where fp32 cannot
hold the result, and not a number only where an operand is none."""
import numpy as np
import pytest
import torch

import product_shapes as shapes
from paper_1708_04801_amd import api
from test_gpu_product_kernels import DTYPES, blocks, gen, values, whole

pytestmark = pytest.mark.gpu

MOST = float(np.finfo(np.float32).max)
CASES = [(m, n, k, t) for m, n, k, *_ in shapes.ROWS[1::3] + shapes.TILES_128[:7] for t in DTYPES] + [(*shapes.TILES_256[3], "f32"), (*shapes.TILES_256[5], "f32"),
                                                                                                     (*shapes.FAST_256[4], "bf16"), (*shapes.FAST_256[8], "bf16")]
every = pytest.mark.parametrize("m,n,k,dtype", CASES)


def rounded(want, dtype):
    return want.float().to(DTYPES[dtype])


@every
def test_the_largest_values_meet_zeros_and_small_ones(m, n, k, dtype):
    g = gen(m, n, k, 3)
    x, y = whole(m, k, g), whole(n, k, g) * 2.0 ** -24
    x[m // 2] = 0.0
    x[m // 2, k // 3] = MOST                          # a code of 256 at 2^120
    y[::2, k // 3] = 0.0
    a, b = blocks(x), blocks(y)
    assert int(a.exps[m // 2, :-(-k // 128)].max()) == 247 and float(values(a).max()) == 2.0 ** 128
    want = values(a) @ values(b).t()
    assert torch.equal(api.wpsgd_block_matmul(a, b, dtype=DTYPES[dtype]), rounded(want, dtype))
    assert torch.equal(api.wpsgd_block_matmul(b, a, dtype=DTYPES[dtype]), rounded(want, dtype).t())
    a.codes.view(torch.uint8)[m // 2, k // 3] = 0x7E  # 448 at 2^120, which no fp32 value needs
    want = values(a) @ values(b).t()
    assert torch.equal(api.wpsgd_block_matmul(a, b, dtype=DTYPES[dtype]), rounded(want, dtype))


@every
@pytest.mark.parametrize("power", [-128, -132])
def test_the_smallest_values_count(m, n, k, dtype, power):
    g = gen(m, n, k, 4)
    x, y = whole(m, k, g) * 2.0 ** power, whole(n, k, g) * 2.0 ** 100
    a, b = blocks(x), blocks(y)
    assert int(a.exps[:, :-(-k // 128)].min()) == 1
    want = x.double() @ y.double().t()
    assert torch.equal(api.wpsgd_block_matmul(a, b, dtype=DTYPES[dtype]), rounded(want, dtype))
    assert torch.equal(api.wpsgd_block_matmul(b, a, dtype=DTYPES[dtype]), rounded(want, dtype).t())


@every
def test_values_finer_than_the_spacing_are_off_by_half_of_it(m, n, k, dtype):
    g = gen(m, n, k, 5)
    x, y = whole(m, k, g) * 2.0 ** -135, whole(n, k, g) * 2.0 ** 100
    want = x.double() @ y.double().t()
    got = api.wpsgd_block_matmul(blocks(x), blocks(y), dtype=DTYPES[dtype]).double()
    assert bool(((got - want).abs() <= 2.0 ** -133 * y.double().abs().sum(1)[None, :] * 1.001 + 2.0 ** -8 * want.abs()).all())


@every
def test_results_that_fp32_cannot_hold_are_infinite(m, n, k, dtype):
    g = gen(m, n, k, 6)
    x, y = (whole(m, k, g).abs() + 1) * 2.0 ** 80, (whole(n, k, g).abs() + 1) * 2.0 ** 80
    x[0], y[0] = -x[0], y[0] * 2.0 ** -80
    got = api.wpsgd_block_matmul(blocks(x), blocks(y), dtype=DTYPES[dtype])
    want = rounded(x.double() @ y.double().t(), dtype)
    assert bool(torch.isinf(want[:, 1:]).all()) and bool(torch.isfinite(want[:, 0]).all())
    assert torch.equal(got, want)
