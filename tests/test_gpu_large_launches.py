"""Calls of more workgroups than one launch may have (2^32 threads along x): rows on both sides of where the next launch begins, and the last ones, are
what a call on them alone gives."""
import pytest
import torch

from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu

GROUPS = (1 << 24) - 1            # of 256 threads, in one launch


def places(edge, n, width=200):
    return [(0, width), (edge - width, edge + width), (n - width, n)]


def test_draws():
    n, c = GROUPS + 300, 3
    z = torch.randn(n, c, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda")
    u = torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    k = torch.randint(0, 4, (n,), generator=torch.Generator(device="cuda").manual_seed(3), device="cuda", dtype=torch.int32)
    drawn, probs = torch.full((n,), -7, dtype=torch.int64, device="cuda"), torch.full((n,), -7.0, device="cuda")
    api.wpsgd_draw_classes(z, u, top_k=k, top_p=0.9, drawn=drawn, probs=probs)
    assert bool((drawn >= 0).all()) and bool((drawn < c).all()) and bool((probs > 0).all())
    for lo, hi in places(GROUPS, n):
        d, p = api.wpsgd_draw_classes(z[lo:hi], u[lo:hi], top_k=k[lo:hi], top_p=0.9)
        assert torch.equal(d, drawn[lo:hi]) and torch.equal(p, probs[lo:hi])


def test_losses_of_short_rows():
    n, c = 4 * GROUPS + 301, 2
    z = torch.randn(n, c, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16()
    labels = torch.randint(0, c, (n,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    w = torch.rand(n, generator=torch.Generator(device="cuda").manual_seed(3), device="cuda")
    loss, grad = torch.full((n,), -7.0, device="cuda"), torch.full((n, c), -7.0, dtype=torch.bfloat16, device="cuda")
    api.wpsgd_softmax_loss(z, labels, row_weights=w, loss=loss, grad=grad)
    assert bool((loss >= 0).all()) and bool((grad.abs() <= 1).all())
    for lo, hi in places(4 * GROUPS, n):
        one = api.wpsgd_softmax_loss(z[lo:hi], labels[lo:hi], row_weights=w[lo:hi])
        assert torch.equal(one[0], loss[lo:hi]) and torch.equal(one[1], grad[lo:hi])


def test_rows_in_blocks():
    n = 16 * GROUPS + 303                             # rows of one block
    x = torch.randn(1000, 3, generator=torch.Generator().manual_seed(1)).cuda()
    X = api.Matrix(1000, 3, dense=x)
    picked = torch.randint(0, 1000, (n,), generator=torch.Generator(device="cuda").manual_seed(2), device="cuda")
    q = api.wpsgd_quantize(X, rows=picked)
    for lo, hi in places(16 * GROUPS, n):
        one = api.wpsgd_quantize(X, rows=picked[lo:hi].clone())
        assert torch.equal(one.codes.view(torch.uint8), q.codes[lo:hi].view(torch.uint8)) and torch.equal(one.exps[:, 0], q.exps[lo:hi, 0])


def test_columns_in_blocks():
    n = 1 << 31                                       # one column: 2^24 blocks
    x = torch.randn(n // 64, generator=torch.Generator(device="cuda").manual_seed(1), device="cuda").bfloat16().repeat(64).view(n, 1)
    x[-500:] *= 3
    q = api.wpsgd_quantize(api.Matrix(n, 1, dense=x), transpose=True)
    blocks = n // 128
    for lo, hi in ((0, 5), (GROUPS - 5, GROUPS + 1), (blocks - 3, blocks)):
        one = api.wpsgd_quantize(api.Matrix((hi - lo) * 128, 1, dense=x[lo * 128:hi * 128]), transpose=True)
        assert torch.equal(one.codes.view(torch.uint8), q.codes[:, lo * 128:hi * 128].view(torch.uint8)) and torch.equal(one.exps[:, :hi - lo], q.exps[:, lo:hi])


def test_products_of_few_rows():
    """a thousand million rows of one block against one and against sixteen: 2^23 workgroups of 512 threads and more"""
    torch.cuda.empty_cache()
    edge = ((1 << 23) - 1) * 128                      # rows of the first launch
    n = edge + 1000
    if torch.cuda.mem_get_info()[0] < n * 170:
        pytest.skip("not enough memory free for 143 GB of operands and 34 GB of results")
    codes = torch.zeros((n, 128), dtype=torch.uint8, device="cuda")
    exps = torch.full((n, 4), 127, dtype=torch.uint8, device="cuda")
    for lo, hi in places(edge, n):
        codes[lo:hi] = torch.randint(0, 126, (hi - lo, 128), dtype=torch.uint8, device="cuda")
    many = api.BlockMatrix(n, 128, codes.view(torch.float8_e4m3fn), exps)
    for few in (1, 16):
        x = torch.randn(few, 128, generator=torch.Generator().manual_seed(few)).cuda()
        a = api.wpsgd_quantize(api.Matrix(few, 128, dense=x))
        out = torch.full((n, few), 7.0, dtype=torch.bfloat16, device="cuda")
        api.wpsgd_block_matmul(many, a, out=out)
        for lo, hi in places(edge, n):
            part = api.BlockMatrix(hi - lo, 128, codes[lo:hi].view(torch.float8_e4m3fn), exps[lo:hi])
            want = api.wpsgd_block_matmul(part, a)
            assert bool(want.any()) and torch.equal(out[lo:hi], want)
        assert not bool(out[200:edge - 200].any()) and not bool(out[edge + 200:n - 200].any())
        del out
    torch.cuda.empty_cache()
