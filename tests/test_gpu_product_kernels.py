"""Every kernel of the products of 8-bit blocks, at the shapes that take it: whole numbers, whose products are exact in any order, random rows against 64
bits, rows that are not numbers, operands and results with strides of their own, and the same bits twice."""
import numpy as np
import pytest
import torch

import product_shapes as shapes
from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}
CASES = [(m, n, k, t) for m, n, k, _ in shapes.ROWS + shapes.TILES_128 for t in DTYPES] + [(m, n, k, "f32") for m, n, k in shapes.TILES_256] + \
    [(m, n, k, "bf16") for m, n, k in shapes.FAST_256]
FEW = [c for c in CASES if c[0] * c[1] < 6_000_000 or c[:3] in (shapes.TILES_256[3], shapes.TILES_256[5], shapes.FAST_256[4])]


def blocks(t, **how):
    return api.wpsgd_quantize(api.Matrix(t.shape[0], t.shape[1], dense=t), **how)


def values(q):
    """what the blocks stand for, in 64 bits"""
    b = q.codes.shape[1] // 128
    power = ((q.exps[:, :b].to(torch.int64) + (1023 - 127)) << 52).view(torch.float64)
    return (q.codes.to(torch.float64).view(q.rows, b, 128) * power[..., None]).view(q.rows, b * 128)


def whole(r, k, gen):
    """whole numbers from -4 to 4, whose products over 65536 elements stay below 2^24 in any order"""
    return torch.randint(-4, 5, (r, k), generator=gen, device="cuda").float()


def gen(*seed):
    return torch.Generator(device="cuda").manual_seed(hash(seed) % (1 << 31))


@pytest.mark.parametrize("m,n,k,dtype", CASES)
def test_whole_numbers_are_exact(m, n, k, dtype):
    g = gen(m, n, k)
    x, y = whole(m, k, g), whole(n, k, g)
    a, b = blocks(x), blocks(y)
    got = api.wpsgd_block_matmul(a, b, dtype=DTYPES[dtype])
    want = x.double() @ y.double().t()
    assert float(want.abs().max()) < 2 ** 24
    assert torch.equal(got, want.float().to(DTYPES[dtype]))
    assert torch.equal(got, api.wpsgd_block_matmul(a, b, dtype=DTYPES[dtype]))


@pytest.mark.parametrize("m,n,k,dtype", CASES)
def test_random_rows(m, n, k, dtype):
    """fp32 sums: K roundings of partial sums, none over |a| |b|, by 2^-24 of them at most and either way: six standard deviations are 6 / sqrt(3) sqrt(K) 2^-24 |a| |b|.  The
    8-bit instruction loses what lies 2^-14 under the largest of 64 products, which are ten times their mean |a| |b| / K at most.  bfloat16 adds half of its last place."""
    g = gen(m, n, k, 1)
    x = torch.randn(m, k, generator=g, device="cuda") * torch.exp(torch.randn(m, 1, generator=g, device="cuda"))
    y = torch.randn(n, k, generator=g, device="cuda").bfloat16()
    a, b = blocks(x), blocks(y)
    got = api.wpsgd_block_matmul(a, b, dtype=DTYPES[dtype]).double()
    A, B = values(a), values(b)
    want = A @ B.t()
    size = A.norm(dim=1)[:, None] * B.norm(dim=1)[None, :]
    bound = 4 * k ** 0.5 * 2.0 ** -24 * size
    if dtype == "bf16":
        bound += 2.0 ** -8 * want.abs() + (10 * 2.0 ** -14 / k ** 0.5 * size if (m, n, k) in shapes.FAST_256 else 0)
    assert bool(((got - want).abs() <= bound).all())


@pytest.mark.parametrize("m,n,k,dtype", FEW)
def test_rows_that_are_not_numbers_and_what_lies_beside(m, n, k, dtype):
    g = gen(m, n, k, 2)
    x, y = whole(m, k, g), whole(n, k, g)
    x[m // 2, k - 1] = float("inf")
    y[n - 1, 0] = float("nan")
    pad = 128 * (-(-k // 128)) + 48
    codes = torch.full((n, pad), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    exps = torch.full((n, -(-(-(-k // 128)) // 4) * 4 + 8), 255, dtype=torch.uint8, device="cuda")
    a, b = blocks(x), blocks(y, codes=codes[:, :pad - 48], exps=exps[:, :-8])
    room = torch.full((m + 2, n + 13), 7.0, dtype=DTYPES[dtype], device="cuda")
    got = api.wpsgd_block_matmul(a, b, out=room[1:-1, 5:n + 5], dtype=DTYPES[dtype])
    bad = torch.isnan(got)
    assert bool(bad[m // 2].all()) and bool(bad[:, n - 1].all()) and int(bad.sum()) == m + n - 1
    x[m // 2] = y[n - 1] = 0.0
    want = (x.double() @ y.double().t()).float().to(DTYPES[dtype])
    assert torch.equal(got.masked_fill(bad, 0.0), want.masked_fill(bad, 0.0))
    assert bool((room[0] == 7).all()) and bool((room[-1] == 7).all()) and bool((room[:, :5] == 7).all()) and bool((room[:, n + 5:] == 7).all())


@pytest.mark.parametrize("dtype", list(DTYPES))
@pytest.mark.parametrize("wide", ["codes", "exps"])
def test_rows_too_far_apart_for_32_bits(wide, dtype):
    m, n, k = 131, 90, 700
    g = gen(9)
    x, y = whole(m, k, g), whole(n, k, g)
    a = blocks(x)
    far = torch.zeros((m, (1 << 22) + 16), dtype=torch.uint8, device="cuda")
    if wide == "codes":
        far[:, :768] = a.codes.view(torch.uint8)
        a = api.BlockMatrix(m, k, far[:, :768].view(torch.float8_e4m3fn), a.exps)
    else:
        far[:, :8] = a.exps
        a = api.BlockMatrix(m, k, a.codes, far[:, :8])
    b = blocks(y)
    want = (x.double() @ y.double().t()).float().to(DTYPES[dtype])
    assert torch.equal(api.wpsgd_block_matmul(a, b, dtype=DTYPES[dtype]), want)
    assert torch.equal(api.wpsgd_block_matmul(b, a, dtype=DTYPES[dtype]), want.t())


@pytest.mark.parametrize("n,c,d", [(2749, 2751, 1100), (8192, 3120, 3135)])
def test_gradients_at_sizes_of_the_large_tiles(n, c, d):
    """<G, x W^T> = <G^T x, W> = <G W, x> in whole numbers, by the transposed forms"""
    g = gen(n, c)
    x, W = whole(n, d, g), whole(c, d, g)
    G = torch.randint(-1, 2, (n, c), generator=g, device="cuda").float()
    scores = api.wpsgd_block_matmul(blocks(x), blocks(W), dtype=torch.float32)
    dW = api.wpsgd_block_matmul(blocks(G, transpose=True), blocks(x, transpose=True), dtype=torch.float32)
    dx = api.wpsgd_block_matmul(blocks(G), blocks(W, transpose=True), dtype=torch.float32)
    assert torch.equal(dW, (G.double().t() @ x.double()).float()) and torch.equal(dx, (G.double() @ W.double()).float())
    inner = lambda a, b: float((a.double() * b.double()).sum())  # noqa: E731
    assert inner(G, scores) == inner(dW, W) == inner(dx, x)
