"""Sums in fp32 for bfloat16 results, asked for where the sizes would take the 8-bit matrix instructions."""
import ctypes

import pytest
import torch

import product_shapes as shapes
from paper_1708_04801_amd import api
from test_gpu_product_kernels import blocks, gen, values, whole

pytestmark = pytest.mark.gpu


@pytest.mark.parametrize("m,n,k", [*shapes.FAST_256, *shapes.TILES_256, *shapes.SUMS_256, (129, 257, 520), (5, 3001, 129), (200, 200, 65536)])
def test_small_products_beside_large_ones_that_cancel(m, n, k):
    """a pair of products 2^16 and -2^16 in every block, and whole numbers up to 16 beside them: exact in fp32"""
    g = gen(m, n, k, 7)
    x, y = whole(m, k, g), whole(n, k, g)
    at = torch.arange(0, k - 1, 128, device="cuda") if k > 1 else torch.arange(0, device="cuda")
    x[:, at], x[:, at + 1] = 256.0, -256.0
    y[:, at], y[:, at + 1] = 256.0, 256.0
    a, b = blocks(x), blocks(y)
    got = api.wpsgd_block_matmul(a, b, fp32_sums=True)
    want = x.double() @ y.double().t()
    assert got.dtype == torch.bfloat16 and torch.equal(got, want.float().bfloat16())
    exact = api.wpsgd_block_matmul(a, b, dtype=torch.float32, fp32_sums=True)
    assert torch.equal(exact, want.float())


@pytest.mark.parametrize("m,n,k", shapes.FAST_256 + shapes.TILES_256[2:6] + shapes.SUMS_256)
def test_random_rows(m, n, k):
    """the bound of fp32 sums (sqrt(K) roundings by 2^-24 of |a| |b|, six standard deviations) and half of bfloat16's last place"""
    g = gen(m, n, k, 8)
    a, b = (blocks(torch.randn(r, k, generator=g, device="cuda")) for r in (m, n))
    A, B = values(a), values(b)
    want = A @ B.t()
    size = A.norm(dim=1)[:, None] * B.norm(dim=1)[None, :]
    got = api.wpsgd_block_matmul(a, b, fp32_sums=True)
    assert bool(((got.double() - want).abs() <= 4 * k ** 0.5 * 2.0 ** -24 * size + 2.0 ** -8 * want.abs()).all())
    room = torch.full((m + 2, n + 13), 7.0, dtype=torch.bfloat16, device="cuda")
    assert torch.equal(api.wpsgd_block_matmul(a, b, out=room[1:-1, 5:n + 5], fp32_sums=True), got)
    assert bool((room[0] == 7).all()) and bool((room[-1] == 7).all()) and bool((room[:, :5] == 7).all()) and bool((room[:, n + 5:] == 7).all())


def test_types_with_sums():
    a = blocks(torch.randn(4, 200, device="cuda"))
    L, out = api.load(), torch.empty(4, 4, device="cuda")
    call = lambda t: L.wpsgd_block_matmul(ctypes.byref(a.c_struct()), ctypes.byref(a.c_struct()), out.data_ptr(), 4, t, None, 0, None)  # noqa: E731
    assert call(api.F32 | api.FP32_SUMS) == call(api.BF16 | api.FP32_SUMS) == api.OK
    assert call(2 | api.FP32_SUMS) == call(32) == call(api.F32 | 8) == api.INVALID_ARG
    torch.cuda.synchronize()
