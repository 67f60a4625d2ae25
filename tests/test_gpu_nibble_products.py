"""Products with 4-bit matrices: results that depend neither on timing nor on a row's place or company, in every kernel."""
import pytest
import torch

from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu

# rows in registers (few rows, many classes), rows in LDS, rows asked for by each wave; whole blocks and rows that end inside one
SHAPES = [(1, 65600, 512), (4, 20000, 4096), (5, 20000, 4093), (16, 33000, 1000), (3, 5000, 9000), (7, 20000, 300), (12, 17000, 2050), (20, 40000, 384), (50, 34000, 260), (130, 17000, 256),
          (24, 33000, 2300), (70, 17000, 2305), (1, 64, 4096), (9, 700, 1111), (30, 3000, 640), (64, 1000, 200), (37, 5003, 301)]


@pytest.mark.parametrize("group", [32, 64, 128])
@pytest.mark.parametrize("dtype", [torch.float32, torch.bfloat16])
@pytest.mark.parametrize("n,classes,d", SHAPES)
def test_a_rows_products_do_not_depend_on_its_place(n, classes, d, dtype, group):
    g = torch.Generator(device="cuda").manual_seed(n + d)
    x = torch.randn(200, d, generator=g, device="cuda").to(dtype)
    W = torch.randn(classes, d, generator=g, device="cuda")
    q = api.wpsgd_quantize_nibbles(api.Matrix(classes, d, dense=W), group=group)
    X = api.Matrix(200, d, dense=x)
    rows = torch.randint(0, 200, (n,), generator=g, device="cuda")
    y = api.wpsgd_nibble_matmul(X, q, rows=rows, dtype=torch.float32)
    # against fp32 products: either side adds d numbers, each off by d 2^-24 of their sizes at most
    at = torch.arange(d, device="cuda")
    byte = at // 128 * 64 + at % 32 // 8 * 16 + at % 128 // 32 * 4 + at % 8 // 2
    code = (q.codes[:, byte] >> (4 * (at % 2)).to(torch.uint8)) & 15
    value = torch.tensor([0, 0.5, 1, 1.5, 2, 3, 4, 6, 0, -0.5, -1, -1.5, -2, -3, -4, -6], device="cuda")
    w = value[code.int()] * q.scales.float()[:, at // group]
    xs = x[rows].float()
    assert ((y - xs @ w.t()).abs() <= 2 * (d + 400) * 2.0 ** -24 * (xs.abs() @ w.abs().t())).all()
    order = torch.randperm(n, generator=torch.Generator().manual_seed(n)).cuda()
    for _ in range(3):
        assert torch.equal(api.wpsgd_nibble_matmul(X, q, rows=rows[order], dtype=torch.float32), y[order])
    assert torch.equal(api.wpsgd_nibble_matmul(X, q, rows=rows, dtype=torch.bfloat16), y.bfloat16())
