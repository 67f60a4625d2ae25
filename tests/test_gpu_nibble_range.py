"""Products with 4-bit matrices at the ends of the number range: results that fp32 holds come out, however large the rows' elements, and small ones are off by next to nothing."""
import pytest
import torch

from paper_1708_04801_amd import api
from test_gpu_nibble_parts import SHAPES, matrix, values

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
# Each product is exact; 12 additions of 33 numbers in a block, one for each of d / 32 groups, 16 waves: so many roundings of 2^-24 of the sum of all sizes, and the result's own.
ROUNDINGS = 12 * 33 + 16


def check(x, value, y, least):
    exact = x.double() @ value.t()
    sizes = x.double().abs() @ value.abs().t()
    slack = (ROUNDINGS + x.shape[1] / 32) * 2.0 ** -24 * sizes + least
    most = torch.finfo(torch.float32).max
    inside, beyond = exact.abs() + slack < most, exact.abs() - slack > 2 * most
    y = y.double()
    assert inside.any() and ((y - exact).abs() <= slack + 2.0 ** -24 * exact.abs())[inside].all()
    assert torch.equal(y[beyond], torch.sign(exact[beyond]) * float("inf"))


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("n,classes,d", SHAPES)
def test_rows_as_large_as_they_can_be(n, classes, d, group, dtype):
    q, value = matrix(classes, d, group, d + n)
    q.scales.mul_(2.0 ** -12)                         # sums of 2^128 times 6, a thousand of them, and they fit
    value = values(q)
    g = torch.Generator(device="cuda").manual_seed(n)
    most = torch.finfo(DTYPES[dtype]).max
    alike = torch.full((n, d), most, device="cuda", dtype=DTYPES[dtype])
    either = alike * torch.randint(0, 2, (n, d), generator=g, device="cuda").mul_(2).sub_(1)
    some = (torch.randn(n, d, generator=g, device="cuda") * 2.0 ** 125).to(DTYPES[dtype])
    for x in (alike, either, some):
        check(x, value, api.wpsgd_nibble_matmul(api.Matrix(n, d, dense=x), q, dtype=torch.float32), 0.0)


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,classes,d", SHAPES)
def test_small_weights_and_small_rows(n, classes, d, dtype):
    """What is under 2^-126 on the way may be lost: 2^-116 of a group's sum before its scale, of which there are d / 64, and of a result."""
    for rows, weights in ((1.0, 2.0 ** -100), (2.0 ** -60, 2.0 ** -50), (2.0 ** -100, 1.0)):
        q, _ = matrix(classes, d, 64, d + n)
        q.scales.mul_(weights)
        value = values(q)
        x = (torch.randn(n, d, generator=torch.Generator(device="cuda").manual_seed(n), device="cuda") * rows).to(DTYPES[dtype])
        least = 2.0 ** -116 * (1 + float(q.scales[:, :-(-d // 64)].double().max()) * d / 64)
        y = api.wpsgd_nibble_matmul(api.Matrix(n, d, dense=x), q, dtype=torch.float32)
        check(x, value, y, least)
