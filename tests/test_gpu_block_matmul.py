"""Rows in 8-bit blocks and products of them, against the definition in 64 bits."""
import numpy as np
import pytest
import torch

import class_reference as ref
from paper_1708_04801_amd import api

pytestmark = pytest.mark.gpu

DTYPES = {"f32": torch.float32, "bf16": torch.bfloat16}


def rows_of(n, c, dtype, seed, pad=0, spread=3.0):
    rng = np.random.default_rng(seed)
    x = torch.from_numpy(rng.standard_normal((n, c + pad)) * np.exp(spread * rng.standard_normal((n, 1)))).to(DTYPES[dtype])
    return x.cuda()[:, :c]


def same_blocks(q, want):
    codes, exps = ref.codes_of(q)
    wc, we = ref.quantize(want)
    assert np.array_equal(exps, we)
    nan = np.isnan(ref.E4M3[wc])
    assert np.array_equal(np.isnan(ref.E4M3[codes]), nan)
    assert np.array_equal(codes[~nan], wc[~nan])


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("n,d,pad", [(1, 1, 0), (1, 127, 0), (3, 128, 0), (5, 129, 0), (2, 520, 8), (67, 1000, 1), (130, 300, 3), (128, 64, 0), (1, 4096, 0),
                                     (300, 65, 5)])
def test_quantize_matches_the_definition_bit_for_bit(n, d, pad, dtype):
    x = rows_of(n, d, dtype, n * 1000 + d, pad)
    X = api.Matrix(n, d, dense=x)
    host = x.double().cpu().numpy()
    same_blocks(api.wpsgd_quantize(X), host)
    same_blocks(api.wpsgd_quantize(X, transpose=True), host.T)
    picked = torch.from_numpy(np.random.default_rng(d).integers(0, n, size=2 * n + 3)).cuda()
    same_blocks(api.wpsgd_quantize(X, rows=picked), host[picked.cpu().numpy()])
    same_blocks(api.wpsgd_quantize(X, rows=picked, transpose=True), host[picked.cpu().numpy()].T)


@pytest.mark.parametrize("transpose", [False, True])
def test_quantize_special_values(transpose):
    x = np.zeros((9, 260))
    x[0, 3] = 448.0                                   # the largest code with e = 0
    x[1, 5] = np.nextafter(np.float32(448), np.float32(1e9))
    x[2, :] = 1e-38 * np.arange(260) / 260            # below the smallest power kept: subnormal codes
    x[3, 7], x[3, 130], x[3, 131] = np.inf, -np.inf, 2.0
    x[4, 9], x[4, 10] = np.nan, 1.0
    x[5, :] = np.finfo(np.float32).max
    x[6, 0] = -0.0
    x[7, :] = 2.0 ** np.linspace(-20, 8, 260)         # codes of every size in one block
    x[8, :] = np.float32(1e-42)                       # subnormal inputs
    x = x.astype(np.float32)
    t = torch.from_numpy(x.T.copy() if transpose else x).cuda()
    same_blocks(api.wpsgd_quantize(api.Matrix(t.shape[0], t.shape[1], dense=t), transpose=transpose), x.astype(np.float64))


def test_rows_outside_the_data_set_are_zero_and_nothing_is_asked_of_no_rows():
    x = rows_of(4, 200, "f32", 1)
    X = api.Matrix(4, 200, dense=x)
    picked = torch.tensor([2, -1, 4, 1 << 40, 0], device="cuda")
    want = np.zeros((5, 200))
    want[0], want[4] = x[2].cpu().numpy(), x[0].cpu().numpy()
    same_blocks(api.wpsgd_quantize(X, rows=picked), want)
    same_blocks(api.wpsgd_quantize(X, rows=picked, transpose=True), want.T)
    none = torch.empty(0, dtype=torch.int64, device="cuda")
    q = api.wpsgd_quantize(X, rows=none)
    assert q.codes.shape == (0, 256)
    w = api.wpsgd_quantize(X)
    assert api.wpsgd_block_matmul(q, w).shape == (0, 4)
    t = api.wpsgd_quantize(X, rows=none, transpose=True)          # 200 x 0: a sum over nothing
    assert torch.equal(api.wpsgd_block_matmul(t, t, dtype=torch.float32), torch.zeros(200, 200, device="cuda"))


def check_product(a, b, dtype, out=None):
    got = api.wpsgd_block_matmul(a, b, out=out, dtype=DTYPES[dtype])
    A, B = (torch.from_numpy(ref.values(*ref.codes_of(q))) for q in (a, b))
    want, size = A @ B.t(), A.abs() @ B.abs().t()
    # every order of summing K products in fp32 is within K 2^-24 of the sum of their sizes; bfloat16 adds half of its last place
    bound = A.shape[1] * 2.0 ** -24 * size + (2.0 ** -8 * want.abs() if dtype == "bf16" else 0) + 1e-37
    assert ((got.double().cpu() - want).abs() <= bound).all()
    return got


SHAPES = [(1, 1, 1), (1, 64, 128), (2, 17, 129), (16, 256, 640), (17, 100, 4096), (33, 1000, 1000), (64, 64, 2048), (100, 33, 260), (128, 128, 128),
          (129, 257, 520), (255, 511, 1100), (256, 256, 4096), (300, 700, 384), (513, 130, 896), (1, 5003, 512), (5003, 1, 512), (7, 3000, 8200),
          (200, 200, 65536)]


@pytest.mark.parametrize("dtype", ["f32", "bf16"])
@pytest.mark.parametrize("m,n,k", SHAPES)
def test_product_matches_the_definition(m, n, k, dtype):
    a = api.wpsgd_quantize(api.Matrix(m, k, dense=rows_of(m, k, "bf16", m + k, spread=1.0)))
    b = api.wpsgd_quantize(api.Matrix(n, k, dense=rows_of(n, k, "f32", n + k, spread=1.0)))
    check_product(a, b, dtype)


@pytest.mark.parametrize("m,n,k", [(1, 50, 300), (48, 500, 1300), (700, 900, 2000)])
def test_product_of_whole_numbers_is_exact(m, n, k):
    """products of small whole numbers are exact in fp32 in any order: every element in its place"""
    rng = np.random.default_rng(k)
    x, y = (torch.from_numpy(rng.integers(-4, 5, size=(r, k)).astype(np.float32)).cuda() for r in (m, n))
    a, b = (api.wpsgd_quantize(api.Matrix(t.shape[0], k, dense=t)) for t in (x, y))
    got = api.wpsgd_block_matmul(a, b, dtype=torch.float32)
    assert torch.equal(got.double().cpu(), x.double().cpu() @ y.double().cpu().t())


def test_strided_operands_and_output_and_nothing_written_beside_it():
    m, n, k = 77, 301, 500
    x, y = rows_of(m, k, "f32", 5, spread=1.0), rows_of(n, k, "bf16", 6, pad=3, spread=1.0)
    codes = torch.full((m, 512 + 48), 0x7F, dtype=torch.uint8, device="cuda").view(torch.float8_e4m3fn)
    exps = torch.full((m, 12), 255, dtype=torch.uint8, device="cuda")
    a = api.wpsgd_quantize(api.Matrix(m, k, dense=x), codes=codes[:, :512], exps=exps[:, :4])
    assert (codes[:, 512:].view(torch.uint8) == 0x7F).all() and (exps[:, 4:] == 255).all()
    b = api.wpsgd_quantize(api.Matrix(n, k, dense=y))
    for dtype in DTYPES:
        whole = torch.full((m, n + 5), 7.0, dtype=DTYPES[dtype], device="cuda")
        got = check_product(a, b, dtype, out=whole[:, 2:n + 2])
        assert (whole[:, :2] == 7).all() and (whole[:, n + 2:] == 7).all()
        assert torch.equal(got, api.wpsgd_block_matmul(a, b, dtype=DTYPES[dtype]))


def test_not_a_number_stays_in_its_row_and_column():
    m, n, k = 40, 70, 400
    x, y = rows_of(m, k, "f32", 8, spread=0.1), rows_of(n, k, "f32", 9, spread=0.1)
    x[3, 399] = float("inf")
    y[65, 0] = float("nan")
    got = api.wpsgd_block_matmul(api.wpsgd_quantize(api.Matrix(m, k, dense=x)), api.wpsgd_quantize(api.Matrix(n, k, dense=y)), dtype=torch.float32)
    bad = torch.isnan(got)
    assert bad[3].all() and bad[:, 65].all() and int(bad.sum()) == m + n - 1


@pytest.mark.parametrize("n,c,d", [(5, 40, 130), (300, 200, 96)])
def test_gradients_are_the_scores_adjoint(n, c, d):
    """<G, x W^T> = <G^T x, W> = <G W, x>, exactly in whole numbers: gradients of W and x by the transposed forms; and scores are linear in W:
    what a change of W adds is what the gradient says"""
    rng = np.random.default_rng(n)
    x, W, G, step = (torch.from_numpy(rng.integers(-3, 4, size=s).astype(np.float32)).cuda() for s in ((n, d), (c, d), (n, c), (c, d)))
    q = lambda t, transpose=False: api.wpsgd_quantize(api.Matrix(t.shape[0], t.shape[1], dense=t), transpose=transpose)  # noqa: E731
    mm = lambda a, b: api.wpsgd_block_matmul(a, b, dtype=torch.float32)  # noqa: E731
    scores, moved = mm(q(x), q(W)), mm(q(x), q(W + step))
    dW, dx = mm(q(G, True), q(x, True)), mm(q(G), q(W, True))
    assert dW.shape == W.shape and dx.shape == x.shape
    inner = lambda a, b: float((a.double() * b.double()).sum())  # noqa: E731
    assert inner(G, scores) == inner(dW, W) == inner(dx, x)
    assert inner(G, moved - scores) == inner(dW, step)


def test_long_operands_pass_32_bit_offsets():
    rows, k, n = 1_100_000, 4096, 40                 # 4.5e9 bytes of codes
    codes = torch.zeros((rows, k), dtype=torch.uint8, device="cuda")
    exps = torch.full((rows, 32), 127, dtype=torch.uint8, device="cuda")
    codes[-3:] = torch.randint(0, 126, (3, k), dtype=torch.uint8, device="cuda")
    b = api.wpsgd_quantize(api.Matrix(n, k, dense=rows_of(n, k, "bf16", 3, spread=0.5)))
    big = api.BlockMatrix(rows, k, codes.view(torch.float8_e4m3fn), exps)
    last = api.BlockMatrix(3, k, codes[-3:].clone().view(torch.float8_e4m3fn), exps[-3:].clone())
    got = api.wpsgd_block_matmul(big, b)
    want = check_product(last, b, "bf16")
    assert torch.equal(got[-3:], want) and not got[:-3].any()
    got = api.wpsgd_block_matmul(b, big)
    assert torch.equal(got[:, -3:], api.wpsgd_block_matmul(b, last)) and not got[:, :-3].any()
    del codes, big
    x = torch.zeros((700_000, 4096), dtype=torch.bfloat16, device="cuda")      # 5.7e9 bytes
    x[-2:] = 1.5
    q = api.wpsgd_quantize(api.Matrix(x.shape[0], x.shape[1], dense=x), rows=torch.tensor([699_999, 5, 699_998], device="cuda"))
    assert (q.codes[[0, 2]].float() * 2.0 ** (float(q.exps[0, 0]) - 127) == 1.5).all() and not q.codes[1].float().any()


def test_refusals():
    x = rows_of(4, 200, "f32", 1)
    X = api.Matrix(4, 200, dense=x)
    a = api.wpsgd_quantize(X)

    def status(f):
        with pytest.raises(api.WpsgdError) as e:
            f()
        return e.value.status

    csr = api.Matrix(4, 200, row_ptr=torch.zeros(5, dtype=torch.int64, device="cuda"), col_idx=torch.zeros(1, dtype=torch.int32, device="cuda"),
                     vals=torch.zeros(1, device="cuda"))
    assert status(lambda: api.wpsgd_quantize(csr, codes=a.codes, exps=a.exps)) == api.UNSUPPORTED
    skewed = torch.empty(4 * 272 + 8, dtype=torch.uint8, device="cuda")[8:].view(4, 272)[:, :256].view(torch.float8_e4m3fn)
    assert status(lambda: api.wpsgd_quantize(X, codes=skewed)) == api.INVALID_ARG                       # codes not on a 16-byte boundary
    narrow = torch.empty((4, 3), dtype=torch.uint8, device="cuda")
    assert status(lambda: api.wpsgd_quantize(X, exps=narrow)) == api.INVALID_ARG                        # a stride that is no whole words
    other = api.wpsgd_quantize(api.Matrix(4, 100, dense=x[:, :100]))
    assert status(lambda: api.wpsgd_block_matmul(a, other)) == api.INVALID_ARG                          # different lengths
    assert status(lambda: api.wpsgd_block_matmul(a, a, out=torch.empty(4, device="cuda").expand(4, 4))) == api.INVALID_ARG      # rows on top of each other
    with pytest.raises(AssertionError):
        api.wpsgd_block_matmul(a, a, out=torch.empty((4, 5), device="cuda"))
    with pytest.raises(AssertionError):
        api.wpsgd_block_matmul(a, a, out=torch.empty((4, 4), device="cuda", dtype=torch.float16))
    torch.cuda.synchronize()
